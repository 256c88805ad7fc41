"""What the cache in 8 bits and the attention operators refuse, on the host and before anything is enqueued (no GPU: pointers are
only checked)."""
import ctypes
import math

import pytest

from paper_2607_12287_amd import incvit

ARG, SHAPE, UNSUPPORTED, OK = (incvit.INCVIT_ERR_ARG, incvit.INCVIT_ERR_SHAPE, incvit.INCVIT_ERR_UNSUPPORTED, incvit.INCVIT_OK)
A, B, C, D, E = 1 << 32, 1 << 33, 1 << 34, 1 << 35, 1 << 36   # addresses that are never read


def kv(**kw):
    c = incvit.incvit_kv(100, 16, 4, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_KV = [dict(blocks=0), dict(blocks=-1), dict(block=0), dict(block=8), dict(block=48), dict(block=256), dict(heads=0), dict(heads=1025),
          dict(head_dim=0), dict(head_dim=4), dict(head_dim=12), dict(head_dim=264), dict(blocks=2 ** 27), dict(blocks=2 ** 31 - 1, block=128)]


@pytest.mark.parametrize("kw", BAD_KV)
def test_caches_out_of_range(kw):
    c = kv(**kw)
    assert incvit.incvit_kv_bytes(c) == 0
    assert incvit.incvit_kv_write(c, 1, 1, A, 256, 64, B, 256, 64, C, 0, D) == UNSUPPORTED
    assert incvit.incvit_kv_read(c, D, 1, 1, C, 0, A, 256, 64, B, 256, 64) == UNSUPPORTED
    assert "cache" in incvit.incvit_last_error()


def test_cache_sizes():
    f = incvit.incvit_kv_bytes
    assert incvit.lib().incvit_kv_bytes(None) == 0
    for d, stored in ((8, 32), (32, 32), (40, 64), (64, 64), (72, 80), (80, 80), (88, 96), (96, 96), (104, 128), (128, 128),
                      (136, 192), (192, 192), (200, 256), (256, 256)):
        want = 100 * 4 * 2 * 16 * stored
        assert want + 100 * 4 * 8 <= f(kv(head_dim=d)) <= want + 100 * 4 * 8 + 512
    # past 32 bits
    assert f(kv(blocks=2 ** 24, heads=16, head_dim=128)) > 2 ** 24 * 16 * 2 * 16 * 128


OK_ROWS = dict(dtype=1, rows=5, k=A, k_row=256, k_head=64, v=B, v_row=256, v_head=64, slots=C, begin=0, cache=D)
BAD_ROWS = [(dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(rows=-1), ARG), (dict(rows=2 ** 22 + 1), ARG), (dict(k=0), ARG),
            (dict(v=0), ARG), (dict(k=A + 2), ARG), (dict(v=B + 8), ARG), (dict(k_row=260), ARG), (dict(v_head=68), ARG), (dict(k_row=-256), ARG),
            (dict(v_row=2 ** 40 + 8), ARG), (dict(slots=0), ARG), (dict(slots=C + 2), ARG), (dict(cache=0), ARG), (dict(cache=D + 128), ARG)]


@pytest.mark.parametrize("kw,status", BAD_ROWS)
def test_rows_of_the_cache(kw, status):
    d = {**OK_ROWS, **kw}
    write = list(d.values())
    assert incvit.incvit_kv_write(kv(), *write) == status
    begin, cache = d.pop("begin"), d.pop("cache")
    assert incvit.incvit_kv_read(kv(), cache, d["dtype"], d["rows"], d["slots"], 0, *[d[x] for x in ("k", "k_row", "k_head", "v", "v_row", "v_head")]) == status
    assert incvit.incvit_last_error() != ""


def test_cache_calls():
    w, r = incvit.incvit_kv_write, incvit.incvit_kv_read
    assert w(kv(), *{**OK_ROWS, "begin": 2}.values()) == ARG and w(kv(), *{**OK_ROWS, "begin": -1}.values()) == ARG
    assert w(None, *OK_ROWS.values()) == ARG and r(None, D, 1, 5, C, 0, A, 256, 64, B, 256, 64) == ARG
    assert r(kv(), D, 1, 5, C, 2, A, 256, 64, B, 256, 64) == ARG and r(kv(), D, 1, 5, C, -1, A, 256, 64, B, 256, 64) == ARG
    # heads of the output that overlap
    for k_row, k_head in ((0, 64), (256, 0), (256, 56), (248, 64), (64, 64)):
        assert r(kv(), D, 1, 5, C, 0, A, k_row, k_head, B, 256, 64) == SHAPE
        assert r(kv(), D, 1, 5, C, 0, A, 256, 64, B, k_row, k_head) == SHAPE
    # nothing to do: nothing is looked at or enqueued
    assert w(kv(), 1, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) == OK and r(kv(), 0, 1, 0, 0, 0, 0, 0, 0, 0, 0, 0) == OK


def attention(**kw):
    a = incvit.incvit_attention(1, 8, 4, 64, 1, 0, 0, 0, 0.125)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def rows(p=A, row=512, head=64):
    return incvit.incvit_rows(p, row, head)


def cached(a=None, c=None, cache=D, n=2, rows_=6, q_start=0, table=B, table_stride=50, width=50, lens=C, max_len=0, q=None, out=None,
           workspace=E):
    return incvit.incvit_kv_attend(a or attention(), c or kv(), cache, n, rows_, q_start, table, table_stride, width, lens, max_len,
                                   q or rows(), out or rows(E), workspace)


def plain(a=None, n=2, rows_=6, q_start=0, key_rows=100, k_start=0, max_len=0, q=None, k=None, v=None, out=None, workspace=E):
    return incvit.incvit_attend(a or attention(), n, rows_, q_start, key_rows, k_start, max_len, q or rows(), k or rows(B, 256), v or rows(C, 256),
                                out or rows(E), workspace)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=264), UNSUPPORTED),
    (dict(q_heads=0), ARG), (dict(q_heads=1028), ARG), (dict(q_heads=9), ARG), (dict(kv_heads=0), ARG), (dict(kv_heads=-4), ARG),
    (dict(causal=2), ARG), (dict(window=-1), ARG), (dict(window=2 ** 30 + 1), ARG), (dict(sinks=-1), ARG), (dict(sinks=2 ** 30 + 1), ARG),
    (dict(fill=2), ARG), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG), (dict(scale=math.nan), ARG), (dict(scale=math.inf), ARG)])
def test_attentions_out_of_range(kw, status):
    a = attention(**kw)
    assert cached(a) == status and plain(a) == status
    assert incvit.incvit_last_error() != ""
    assert incvit.incvit_attention_workspace_bytes(a, 1, 2, 6, 0, 10 ** 6) == 0


def test_scales_that_are_infinite_in_units_of_log2():
    """Infinity times a score of 0 would be NaN."""
    for scale, status in ((3.4e38, ARG), (2.4e38, ARG), (2.35e38, OK)):
        a = attention(scale=scale)
        assert cached(a, rows_=0) == status and plain(a, rows_=0) == status
        assert (incvit.incvit_attention_workspace_bytes(a, 1, 2, 6, 0, 10 ** 6) > 0) == (status == OK)


@pytest.mark.parametrize("call", [cached, plain])
def test_what_both_attentions_refuse(call):
    for kw, status in [(dict(n=-1), ARG), (dict(n=2 ** 24 + 1, rows_=2 ** 24 + 1), ARG), (dict(rows_=-1), ARG), (dict(rows_=2 ** 29), ARG),
                       (dict(rows_=7), SHAPE), (dict(max_len=-1), ARG), (dict(max_len=2 ** 41), ARG), (dict(q_start=A + 2), ARG),
                       (dict(q=rows(0)), ARG), (dict(q=rows(A + 8)), ARG), (dict(q=rows(A, 516)), ARG), (dict(q=rows(A, 512, -64)), ARG),
                       (dict(out=rows(0)), ARG), (dict(out=rows(E + 2)), ARG), (dict(out=rows(E, 504)), SHAPE), (dict(out=rows(E, 0)), SHAPE),
                       (dict(out=rows(E, 512, 56)), SHAPE), (dict(rows_=2 ** 28, n=1), UNSUPPORTED)]:
        assert call(**kw) == status, kw
        assert incvit.incvit_last_error() != ""
    f = incvit.lib().incvit_kv_attend if call is cached else incvit.lib().incvit_attend
    one = f.argtypes
    assert f(*[None if t is ctypes.c_void_p else 1 for t in one]) == ARG
    # nothing to do
    assert call(n=0, rows_=0) == OK and call(rows_=0) == OK and call(n=0) == OK


def test_what_the_cached_attention_refuses():
    for kw, status in [(dict(c=kv(heads=8)), SHAPE), (dict(c=kv(head_dim=72)), SHAPE), (dict(c=kv(block=24)), UNSUPPORTED),
                       (dict(cache=0), ARG), (dict(cache=D + 16), ARG), (dict(table=0), ARG), (dict(table=B + 1), ARG), (dict(lens=0), ARG),
                       (dict(lens=C + 2), ARG), (dict(table_stride=-1), ARG), (dict(table_stride=2 ** 41), ARG), (dict(width=-1), ARG),
                       (dict(width=10 ** 5, workspace=0), ARG), (dict(width=10 ** 5, workspace=E + 64), ARG)]:
        assert cached(**kw) == status, kw


def test_what_the_plain_attention_refuses():
    for kw, status in [(dict(key_rows=-1), ARG), (dict(key_rows=2 ** 30 + 1), ARG), (dict(key_rows=101), SHAPE), (dict(k_start=B + 2), ARG),
                       (dict(k=rows(B, 2 ** 23 + 8)), UNSUPPORTED), (dict(v=rows(C, 2 ** 24)), UNSUPPORTED), (dict(k=rows(0)), ARG), (dict(k=rows(B + 2)), ARG), (dict(v=rows(C, 257)), ARG), (dict(v=rows(C, 2 ** 41)), ARG),
                       (dict(key_rows=2 ** 20, workspace=0), ARG)]:
        assert plain(**kw) == status, kw


def test_workspaces():
    f = incvit.incvit_attention_workspace_bytes
    a = attention()
    assert f(a, 1, 1, 1, 0, 1024) == 0 and f(a, 1, 4096, 4096, 0, 10 ** 6) == 0  # one workgroup's keys; rows enough
    assert f(a, 1, 1, 1, 0, 10 ** 5) > f(a, 1, 1, 1, 0, 10 ** 4) > 0
    assert f(a, 0, 1, 1, 0, 10 ** 5) > 0
    assert f(attention(window=512), 1, 1, 1, 0, 10 ** 9) == f(attention(window=512), 1, 1, 1, 0, 10 ** 5)
    for bad in ((0, 1, 0, 5), (1, 0, 0, 5), (1, 1, 0, -1), (1, 2 ** 30, 0, 5), (2 ** 25, 1, 0, 5)):
        n, r, ragged, most = bad
        assert f(a, 1, n, r, ragged, most) == 0
    assert incvit.lib().incvit_attention_workspace_bytes(None, 1, 1, 1, 0, 5) == 0


@pytest.mark.parametrize("most", [2 ** 30, 2 ** 31 + 5, 2 ** 36, 2 ** 39, 2 ** 40])
def test_hints_past_the_most_keys_plan_as_those(most):
    """A hint may be any number to 2^40; a sequence has 2^30 keys at most, and the split is made for no more."""
    f = incvit.incvit_attention_workspace_bytes
    forms = set()
    for dtype in (0, 1):
        for hk in (1, 2, 3, 4, 7, 16, 64, 255, 1000):
            for cached in (0, 1):
                for n, rows, ragged in [(1, 1, 0), (1, 40, 0), (1, 4096, 0), (1, 8192, 0), (1, 8192, 1), (180, 180, 0), (180, 180, 1), (60, 60, 0)]:
                    a = attention(dtype=dtype, q_heads=hk, kv_heads=hk)
                    got = f(a, cached, n, rows, ragged, most)
                    assert got == f(a, cached, n, rows, ragged, 2 ** 30), (dtype, hk, cached, n, rows, ragged)
                    forms.add(got > 0)
                    # partial results of 128 rows at most: of 1536 shares, or of as many (one for each head) and one for each sequence
                    assert got <= (max(1536, hk) + 64 * hk) * 128 * (64 + 2) * 4
    assert forms == {False, True}


def test_the_widest_tables_are_planned():
    """Without a hint the table's width stands for it, up to 2^38 keys: shared, so that a call without a workspace is refused."""
    for block, width, n, rows_ in ((128, 2 ** 31 - 1, 1, 1), (128, 2 ** 31 - 1, 1, 1000), (16, 2 ** 31 - 1, 3, 3), (128, 2 ** 31 - 1, 31, 62)):
        assert cached(c=kv(block=block), n=n, rows_=rows_, width=width, workspace=0) == ARG


def test_sizes_past_32_bits_are_refused_in_python():
    for kw in (dict(blocks=2 ** 32 + 1), dict(heads=2 ** 32 + 1), dict(head_dim=2 ** 32 + 64), dict(block=2 ** 32 + 16), dict(blocks=-1)):
        with pytest.raises(ValueError):
            incvit.KVCache(**{**dict(blocks=4, heads=1, head_dim=64), **kw})
    with pytest.raises(incvit.IncvitError):
        incvit.KVCache(4, 1, 60)
