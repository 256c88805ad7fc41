"""What the stand-alone operators refuse, on the host and before anything is enqueued (no GPU: pointers are only checked)."""
import ctypes
import math

import pytest

from paper_2607_12287_amd import incvit

ARG, SHAPE, UNSUPPORTED, OK = (incvit.INCVIT_ERR_ARG, incvit.INCVIT_ERR_SHAPE, incvit.INCVIT_ERR_UNSUPPORTED, incvit.INCVIT_OK)
A, B, T, X = 1 << 32, 1 << 33, 1 << 34, 1 << 35   # addresses that are never read


def rope(**kw):
    r = incvit.make_rope(128, (16, 24, 24))
    for k, v in kw.items():
        if isinstance(v, tuple):
            for i, x in enumerate(v):
                getattr(r, k)[i] = x
        else:
            setattr(r, k, v)
    return r


@pytest.mark.parametrize("kw", [dict(axes=0), dict(axes=4), dict(pairs=(0, 24, 24)), dict(pairs=(64, 64, 1)), dict(pairs=(-1, 3, 3)),
                                dict(ladder=2), dict(layout=-1), dict(theta=0.5), dict(theta=math.nan), dict(theta=math.inf),
                                dict(scale=(0.0, 1.0, 1.0)), dict(scale=(1.0, math.nan, 1.0)), dict(scale=(1.0, 1.0, math.inf)),
                                dict(scale=(-2.0 ** 21, 1.0, 1.0))])
def test_ropes_out_of_range(kw):
    assert incvit.incvit_rope_table(rope(**kw), 5, A, 5, 1, T) == ARG
    assert incvit.incvit_rope_table_grids(rope(**kw), [(1, 2, 2)], 1, T) == ARG
    assert "rope" in incvit.incvit_last_error()


def test_rope_table_arguments():
    f = incvit.incvit_rope_table
    for args in [(-1, A, 5, 1, T), (5, 0, 5, 1, T), (5, A, 5, 1, 0), (5, A + 2, 5, 1, T), (5, A, 5, 1, T + 4), (5, A, -1, 1, T),
                 (5, A, 5, -1, T), (5, A, 2 ** 41, 1, T), (2 ** 31 // 64, A, 5, 1, T), (2 ** 40, A, 5, 1, T)]:
        assert f(rope(), *args) == ARG, args
    assert incvit.lib().incvit_rope_table(None, 5, A, 5, 1, T, None) == ARG
    assert f(rope(), 0, 0, 0, 0, 0) == OK


def test_rope_grid_arguments():
    f = incvit.incvit_rope_table_grids
    for grids, merge, status in [([(0, 2, 2)], 1, ARG), ([(1, 2, 2), (1, -2, 2)], 1, ARG), ([(1, 2, 2)], 0, ARG),
                                 ([(1, 2, 3)], 2, SHAPE), ([(1, 3, 2)], 2, SHAPE), ([(2 ** 30, 2 ** 30, 2 ** 30)], 1, ARG),
                                 ([(1, 5000, 5000)] * 3, 1, ARG)]:
        assert f(rope(), grids, merge, T) == status, grids
    assert f(rope(), [(1, 2, 2)], 1, 0) == ARG
    assert f(rope(), [(1, 2, 2)], 1, T + 4) == ARG
    assert incvit.lib().incvit_rope_table_grids(ctypes.addressof(rope()), -1, None, 1, T, None) == ARG
    assert incvit.lib().incvit_rope_table_grids(ctypes.addressof(rope()), 1, None, 1, T, None) == ARG
    assert f(rope(), [], 1, 0) == OK


def qk(**kw):
    c = incvit.incvit_qk(incvit.INCVIT_BF16, 64, 64, 0, 1, 1e-6)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def heads(**kw):
    h = incvit.incvit_heads(A, B, None, None, 256, 64, 256, 64, 4)
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def call(c=None, rows=8, q=None, k=None, table=T, table_rows=8, index=0, k_rows=0, k_out_rows=0):
    return incvit.incvit_qk_norm_rope(c or qk(), rows, q, k, table, table_rows, index, k_rows, k_out_rows)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(head_dim=258), UNSUPPORTED),
    (dict(head_dim=63), UNSUPPORTED), (dict(rot_dim=66), SHAPE), (dict(rot_dim=31), SHAPE), (dict(rot_dim=-2), SHAPE),
    (dict(pairing=2), ARG), (dict(norm=3), ARG), (dict(eps=-1.0), ARG), (dict(eps=math.nan), ARG), (dict(eps=math.inf), ARG)])
def test_qk_configurations(kw, status):
    assert call(qk(**kw), q=heads()) == status
    assert incvit.incvit_last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(in_=0), ARG), (dict(out=0), ARG), (dict(in_=A + 1), ARG), (dict(gamma=X + 1), ARG), (dict(beta=X), ARG), (dict(heads=-1), ARG),
    (dict(heads=70000), ARG), (dict(in_row=-1), ARG), (dict(out_head=2 ** 41), ARG), (dict(out_head=63), SHAPE), (dict(out_row=255), SHAPE),
    (dict(out_row=0), SHAPE), (dict(out_row=64, out_head=64 * 7), SHAPE), (dict(out=A, in_row=512, out_row=256), SHAPE),
    (dict(out=A, in_head=128), SHAPE)])
def test_qk_rows(kw, status):
    assert call(q=heads(**kw)) == status, kw
    assert call(k=heads(**kw)) == status, kw


def test_qk_arguments():
    assert incvit.lib().incvit_qk_norm_rope(None, 8, None, None, T, 8, None, None, 0, None) == ARG
    assert call(rows=-1, q=heads()) == ARG
    assert call(table=0, q=heads()) == ARG
    assert call(table=T + 4, q=heads()) == ARG
    assert call(table_rows=0, q=heads()) == ARG
    assert call(table_rows=2 ** 31, q=heads()) == ARG
    assert call(index=X + 2, q=heads()) == ARG
    assert call(k_rows=X + 1, k_out_rows=9, k=heads()) == ARG
    assert call(k_rows=X, k_out_rows=0, k=heads()) == ARG
    assert call(k_rows=X, k_out_rows=9, k=heads(out=A)) == SHAPE
    assert call(rows=2 ** 30, q=heads()) == ARG
    # transposed outputs that do not overlap for 8 rows do for the cache's 9
    assert call(k_rows=X, k_out_rows=9, k=heads(out_row=64, out_head=64 * 8)) == SHAPE
    # nothing to do: nothing is looked at or enqueued
    assert call(rows=0, q=heads(in_=0, out=0), table=0) == OK
    assert call() == OK


def test_make_rope_checks_its_sizes():
    for args in [(64, ()), (64, (1, 1, 1, 1)), (64, (20, 20))]:
        with pytest.raises(ValueError):
            incvit.make_rope(*args)
    with pytest.raises(ValueError):
        incvit.make_rope(64, (16, 16), scale=(1.0,))
    with pytest.raises(KeyError):
        incvit.make_rope(64, (16, 16), ladder="both")


def test_qlinear_sizes():
    w, r = incvit.incvit_qlinear_weights_bytes, incvit.incvit_qlinear_rows_bytes
    for K, N in [(0, 5), (5, 0), (65537, 5), (5, 2 ** 20 + 1), (65536, 65536), (-1, 5)]:
        assert w(K, N) == 0
        assert incvit.incvit_qlinear_pack_weights(0, K, N, A, N, 1, 0, 0, B) == UNSUPPORTED
        assert incvit.incvit_qlinear(0, 5, K, N, A, K, B, 0, 0, 0, T, N, X) == UNSUPPORTED
    assert w(64, 16) >= 64 * 16 + 2 * 64 and w(65, 17) >= 2 * 128 * 16
    for rows, K in [(-1, 5), (5, 0), (5, 65537), (2 ** 31, 5)]:
        assert r(rows, K) == 0
    assert r(0, 64) == 0 and r(1, 64) >= 1024 + 64 and r(17, 65) >= 2 * 2048


def test_qlinear_pack_refusals():
    f = incvit.incvit_qlinear_pack_weights
    ok = dict(dtype=0, K=64, N=16, w=A, k_stride=16, n_stride=1, scales=0, bias=0, weights=B)
    for kw, status in [(dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(w=0), ARG), (dict(weights=0), ARG),
                       (dict(weights=B + 64), ARG), (dict(scales=T), ARG), (dict(dtype=2), ARG), (dict(w=A + 2), ARG),
                       (dict(bias=T + 2), ARG), (dict(dtype=2, scales=T + 2), ARG), (dict(k_stride=-1), ARG),
                       (dict(n_stride=2 ** 41), ARG)]:
        assert f(*{**ok, **kw}.values()) == status, kw


def test_qlinear_row_refusals():
    f = incvit.incvit_qlinear_quantize_rows
    ok = dict(dtype=1, rows=5, K=64, x=A, x_stride=64, gamma=0, beta=0, eps=1e-6, qrows=B)
    for kw, status in [(dict(dtype=2), UNSUPPORTED), (dict(rows=-1), ARG), (dict(rows=2 ** 31), ARG), (dict(x=0), ARG), (dict(x=A + 1), ARG),
                       (dict(x_stride=-1), ARG), (dict(qrows=0), ARG), (dict(qrows=B + 128), ARG), (dict(beta=T), ARG),
                       (dict(gamma=T + 1), ARG), (dict(gamma=T, eps=-1.0), ARG), (dict(gamma=T, eps=math.nan), ARG)]:
        assert f(*{**ok, **kw}.values()) == status, kw
    assert f(1, 0, 64, 0, 64, 0, 0, 1e-6, 0) == OK


def test_qlinear_product_refusals():
    two, one = incvit.incvit_qlinear_multiply, incvit.incvit_qlinear
    ok = dict(dtype=1, rows=5, K=64, N=16, x=A, weights=B, gelu=0, residual=0, res_stride=0, out=T, out_stride=16)
    for kw, status in [(dict(dtype=2), UNSUPPORTED), (dict(rows=-1), ARG), (dict(x=0), ARG), (dict(x=A + 1), ARG), (dict(weights=0), ARG),
                       (dict(weights=B + 16), ARG), (dict(gelu=2), ARG), (dict(residual=X + 1, res_stride=16), ARG),
                       (dict(residual=X, res_stride=-1), ARG), (dict(out=0), ARG), (dict(out=T + 1), ARG), (dict(out_stride=15), SHAPE),
                       (dict(residual=T, res_stride=32), SHAPE)]:
        d = {**ok, **kw}
        assert two(*d.values()) == status, kw
        v = list(d.values())
        assert one(*v[:5], 64, *v[5:], X) == status, kw
    assert one(1, 5, 64, 16, A, 64, B, 0, 0, 0, T, 16, X + 16) == ARG
    assert one(1, 5, 64, 16, A, -1, B, 0, 0, 0, T, 16, X) == ARG
    assert two(1, 0, 64, 16, 0, 0, 0, 0, 0, 0, 0) == OK and one(1, 0, 64, 16, 0, 0, 0, 0, 0, 0, 0, 0, 0) == OK


@pytest.mark.parametrize("kw,status", [(dict(rope=3, rope_theta=10.0), ARG), (dict(rope=-1), ARG), (dict(rope=1), ARG),
                                       (dict(rope=1, rope_theta=math.nan), ARG), (dict(rope=2, rope_theta=0.5), ARG),
                                       (dict(qk_norm=3), ARG), (dict(mlp_int8=2), ARG), (dict(mlp_int8=1, mlp_dim=65537), UNSUPPORTED)])
def test_encoder_options_out_of_range(kw, status):
    from paper_2607_12287_amd import synth
    cfg = incvit.make_config(synth.small_model(dtype="bf16"), 1)
    cfg.rope_theta = 0.0
    for k, v in kw.items():
        setattr(cfg, k, v)
    assert incvit.incvit_canonical_weights_bytes(cfg) == 0
    assert incvit.incvit_pack_weights(cfg, 256, 256, 0) == status


def test_encoder_options_in_the_sizes():
    from paper_2607_12287_amd import synth
    for o in (dict(), dict(rope="halves"), dict(qk_norm="rms"), dict(qk_norm="layer", mlp_int8=True)):
        m = synth.small_model(dtype="bf16", **o)
        assert incvit.incvit_canonical_weights_bytes(incvit.make_config(m, 1)) == 2 * synth.canonical_weight_count(m)
    m, q = synth.SO400M, synth.ModelShape(**{**synth.SO400M.__dict__, "mlp_int8": True})
    f = incvit.incvit_packed_weights_bytes
    assert f(incvit.make_config(q, 1)) < 0.7 * f(incvit.make_config(m, 1))
