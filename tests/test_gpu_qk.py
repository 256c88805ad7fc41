"""Head norms with the rotation on the GPU against 64-bit arithmetic: types, head sizes, norms, pairings, partial rotation,
grouped keys, strides, alignments, padding rows, keys scattered into a cache, in place, streams and captured calls.

Tolerance, in units u = 2^-24 (fp32 half step).  A head's sum of at most 256 terms is formed as at most 16 in one lane and
6 combining steps: 24 u of the sum of squares, 12 u of its root, 4 more for the division, root, mean and products: 16 u of
each normed value; with a LayerNorm the mean's error, 24 u of mean |x|, shifts every value by that times the row's factor
and gain.  The rotation rounds two products and a sum and takes its two values with their errors: at most 20 u of
|n_a| + |n_b|.  Then one rounding to the storage type, finfo.eps / 2 of the value."""
import numpy as np
import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import ops_ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def want_and_bound(x, g, b, norm, eps, table, rows, pairing, dtype):
    """(64-bit result, bound) of [rows][heads][d] values; rows: the table rows."""
    n, r, mean = ops_ref.head_norm(f64(x), f64(g), f64(b), norm, eps)
    gain = 1.0 if g is None else np.abs(f64(g))
    base = (0.0 if b is None else np.abs(f64(b))) + np.abs(n)
    err = np.zeros_like(n) if norm is None else 16 * U * base + (24 * U * mean * r * gain if norm == "layer" else 0.0)
    y = n
    if table is not None and table.shape[1]:
        t = f64(table)[rows]
        y = ops_ref.rotate(n, t[..., 0], t[..., 1], pairing)
        p = t.shape[1]

        def both(v):  # |v_a| + |v_b| for both members of a pair
            s = np.array(v)
            a, c = (slice(0, p), slice(p, 2 * p)) if pairing == "halves" else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
            s[..., a] = s[..., c] = v[..., a] + v[..., c]
            return s

        err = both(err) + 4 * U * both(np.abs(n))
    return y, err + torch.finfo(dtype).eps / 2 * (np.abs(y) + err) + 1e-30


def check(got, want):
    y, bound = want
    d = np.abs(f64(got) - y)
    assert np.all(d <= bound), (d / bound).max()


def make(rows, hq, hk, d, dtype, seed=0, shift=0.0):
    g = torch.Generator().manual_seed(seed + 17 * rows + d)
    rnd = lambda *s: (torch.randn(*s, generator=g) * 1.5 + shift).to(DT[dtype]).cuda()  # noqa: E731
    gain = lambda m: (torch.randn(d, generator=g) * 0.1 + m).to(DT[dtype]).cuda()  # noqa: E731
    return rnd(rows, hq, d), rnd(rows, hk, d), gain(1.0), gain(1.0), gain(0.0), gain(0.0)


def make_table(rows, pairs, seed=3):
    ang = torch.rand(rows, pairs, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 2000 - 1000
    return torch.stack([ang.cos(), ang.sin()], -1).float().cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot", [(64, 64), (72, 72), (80, 60), (128, 128), (2, 2), (6, 4), (44, 44), (16, 16), (256, 256), (250, 2),
                                   (96, 48), (32, 0)])
@pytest.mark.parametrize("norm,pairing", [("rms", "halves"), ("layer", "adjacent"), (None, "halves"), ("rms", "adjacent"),
                                          ("layer", "halves")])
def test_values(dtype, d, rot, norm, pairing):
    rows, hq, hk = 37, 6, 2
    q, k, qg, kg, qb, kb = make(rows, hq, hk, d, dtype)
    if norm != "layer":
        qb = kb = None
    table = make_table(rows, rot // 2) if rot else None
    qo, ko = incvit.qk_norm_rope(q, k, table, pairing, norm, qg, kg, qb, kb)
    t = np.arange(rows)
    if norm is None:
        qg = kg = None
    check(qo, want_and_bound(q, qg, qb, norm, 1e-6, table, t, pairing, DT[dtype]))
    check(ko, want_and_bound(k, kg, kb, norm, 1e-6, table, t, pairing, DT[dtype]))


@pytest.mark.parametrize("rows,hq,hk", [(1, 16, 4), (1, 1, 0), (3, 0, 1), (257, 16, 16), (1031, 3, 1)])
def test_rows_and_heads(rows, hq, hk):
    q, k, qg, kg, _, _ = make(rows, max(hq, 1), max(hk, 1), 72, "bf16")
    q, k = (q if hq else None), (k if hk else None)
    table = make_table(7, 36)  # rows share it in turn
    qo, ko = incvit.qk_norm_rope(q, k, table, q_gamma=qg, k_gamma=kg)
    t = np.arange(rows) % 7
    assert (qo is None) == (q is None) and (ko is None) == (k is None)
    if hq:
        check(qo, want_and_bound(q, qg, None, "rms", 1e-6, table, t, "halves", torch.bfloat16))
    if hk:
        check(ko, want_and_bound(k, kg, None, "rms", 1e-6, table, t, "halves", torch.bfloat16))


def test_no_rows():
    q, k, qg, kg, _, _ = make(1, 4, 2, 64, "bf16")
    qo, ko = incvit.qk_norm_rope(q[:0], k[:0], make_table(4, 32), q_gamma=qg, k_gamma=kg)
    assert qo.shape == (0, 4, 64) and ko.shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 4, 8])
def test_views_of_a_projection_and_transposed_outputs(dtype, offset):
    """q and k inside [rows][q | k | v] at any element offset; outputs laid out [heads][rows][d]."""
    rows, h, d = 50, 5, 72
    buf = (torch.randn(offset + rows * 3 * h * d + 5, generator=torch.Generator().manual_seed(1))).to(DT[dtype]).cuda()
    x = buf[offset:offset + rows * 3 * h * d].view(rows, 3, h, d)
    q, k = x[:, 0], x[:, 1]
    keep = buf.clone()
    table = make_table(rows, 36)
    qo = torch.zeros(h, rows, d, dtype=DT[dtype], device="cuda").transpose(0, 1)
    ko = torch.zeros(h, rows, d, dtype=DT[dtype], device="cuda").transpose(0, 1)
    incvit.qk_norm_rope(q, k, table, norm="layer", q_out=qo, k_out=ko)
    check(qo, want_and_bound(q, None, None, "layer", 1e-6, table, np.arange(rows), "halves", DT[dtype]))
    check(ko, want_and_bound(k, None, None, "layer", 1e-6, table, np.arange(rows), "halves", DT[dtype]))
    assert torch.equal(buf, keep)
    # in place: the same values, the value heads and what surrounds them untouched
    incvit.qk_norm_rope(q, k, table, norm="layer", q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    y = buf[offset:offset + rows * 3 * h * d].view(rows, 3, h, d)
    assert torch.equal(y[:, 2], keep[offset:offset + rows * 3 * h * d].view(rows, 3, h, d)[:, 2])
    assert torch.equal(buf[:offset], keep[:offset]) and torch.equal(buf[-5:], keep[-5:])


@pytest.mark.parametrize("d", [64, 72, 44])
def test_padding_rows_and_keys_into_a_cache(d):
    """Rows whose table index is outside the table get nothing, rows whose cache row is outside it no key; cache rows that
    nobody names stay as they were."""
    rows, h, n = 9, 4, 32
    q, k, qg, kg, _, _ = make(rows, h, h, d, "bf16")
    table = make_table(n, d // 2)
    index = torch.tensor([5, -1, 0, 31, 32, 7, 2 ** 31 - 1, -2 ** 31, 8], dtype=torch.int32, device="cuda")
    dst = torch.tensor([3, 4, 31, -1, 6, 32, 9, 10, 0], dtype=torch.int32, device="cuda")
    qo = torch.full_like(q, 9.0)
    ko = torch.full((n, h, d), 9.0, dtype=k.dtype, device="cuda")
    incvit.qk_norm_rope(q, k, table, q_gamma=qg, k_gamma=kg, index=index, k_rows=dst, q_out=qo, k_out=ko)
    ok = [i for i in range(rows) if 0 <= index[i] < n]
    y, b = want_and_bound(q, qg, None, "rms", 1e-6, table, np.clip(f64(index).astype(int), 0, n - 1), "halves", torch.bfloat16)
    check(qo[ok], (y[ok], b[ok]))
    assert torch.all(qo[[i for i in range(rows) if i not in ok]] == 9.0)
    y, b = want_and_bound(k, kg, None, "rms", 1e-6, table, np.clip(f64(index).astype(int), 0, n - 1), "halves", torch.bfloat16)
    named = {int(dst[i]): i for i in ok if 0 <= dst[i] < n}
    assert sorted(named) == [0, 3, 31]
    for c in range(n):
        if c in named:
            check(ko[c:c + 1], (y[named[c]:named[c] + 1], b[named[c]:named[c] + 1]))
        else:
            assert torch.all(ko[c] == 9.0), c


@pytest.mark.parametrize("norm", ["rms", "layer", None])
def test_rows_that_are_not_finite_stay_alone(norm):
    q, _, qg, _, _, _ = make(8, 3, 1, 72, "bf16")
    q[2, 1, 5] = float("nan")
    q[4, 0, 70] = float("inf")
    table = make_table(8, 36)
    qo, _ = incvit.qk_norm_rope(q, None, table, norm=norm, q_gamma=qg)
    clean = q.clone()
    clean[2, 1], clean[4, 0] = 0.5, 0.5
    co, _ = incvit.qk_norm_rope(clean, None, table, norm=norm, q_gamma=qg)
    for r in range(8):
        for h in range(3):
            if (r, h) in ((2, 1), (4, 0)):
                assert not torch.isfinite(qo[r, h].float()).all()
            else:
                assert torch.equal(qo[r, h], co[r, h])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_means_zeros_and_extremes(dtype):
    """A mean eighty times the spread (no cancellation), rows of zeros, of the type's largest and of tiny values."""
    q, k, qg, kg, qb, kb = make(6, 2, 2, 64, dtype, shift=120.0)
    q[1] = 0.0
    q[2] = 1e-20
    q[3] = 1e18  # squares stay below the largest fp32 number over 64 values
    table = make_table(6, 32)
    qo, ko = incvit.qk_norm_rope(q, k, table, "adjacent", "layer", qg, kg, qb, kb)
    check(qo, want_and_bound(q, qg, qb, "layer", 1e-6, table, np.arange(6), "adjacent", DT[dtype]))
    check(ko, want_and_bound(k, kg, kb, "layer", 1e-6, table, np.arange(6), "adjacent", DT[dtype]))
    qo, _ = incvit.qk_norm_rope(q, None, table, "adjacent", "rms", qg)
    check(qo, want_and_bound(q, qg, None, "rms", 1e-6, table, np.arange(6), "adjacent", DT[dtype]))


def test_offsets_beyond_32_bits():
    """Rows of a buffer more than 2^32 bytes long: the last ones are right."""
    h, d = 2, 64
    stride = (1 << 31) // 2 + 64   # elements: three rows span over 4 GiB of bf16
    buf = torch.zeros(2 * stride + h * d, dtype=torch.bfloat16, device="cuda")
    q = buf.as_strided((3, h, d), (stride, d, 1))
    src, _, qg, _, _, _ = make(3, h, 1, d, "bf16")
    q.copy_(src)
    table = make_table(3, 32)
    incvit.qk_norm_rope(q, None, table, q_gamma=qg, q_out=q)
    check(q.contiguous(), want_and_bound(src, qg, None, "rms", 1e-6, table, np.arange(3), "halves", torch.bfloat16))


def test_another_stream_and_captured_calls():
    q, k, qg, kg, _, _ = make(23, 16, 16, 72, "bf16")
    table = make_table(256, 36)
    index = torch.arange(0, 230, 10, dtype=torch.int32, device="cuda")
    ko = torch.zeros(256, 16, 72, dtype=torch.bfloat16, device="cuda")
    run = lambda q_out, k_out: incvit.qk_norm_rope(q, k, table, q_gamma=qg, k_gamma=kg, index=index, k_rows=index,  # noqa: E731
                                                   q_out=q_out, k_out=k_out)
    want, wk = run(torch.zeros_like(q), ko.clone())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got, gk = run(torch.zeros_like(q), ko.clone())
    st.synchronize()
    assert torch.equal(got, want) and torch.equal(gk, wk)
    out, kout = torch.zeros_like(q), ko.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(out, kout)
    for seed in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)))
        kout.zero_()
        g.replay()
        torch.cuda.synchronize()
        want, wk = run(torch.zeros_like(q), ko.clone())
        assert torch.equal(out, want) and torch.equal(kout, wk)


def test_more_rows_than_one_launch_counts():
    """70 million rows of one head of two values: a launch of a thread each would pass 2^32."""
    rows = 70_000_001
    x = torch.randn(rows, 1, 2, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(torch.bfloat16)
    table = make_table(7, 1)
    got, _ = incvit.qk_norm_rope(x, None, table, norm=None)
    t = table[torch.arange(rows, device="cuda") % 7, 0].double()
    for lo in range(0, rows, 1 << 24):
        s = slice(lo, lo + (1 << 24))
        a, b, c, n = x[s, 0, 0].double(), x[s, 0, 1].double(), t[s, 0], t[s, 1]
        for i, y in ((0, a * c - b * n), (1, b * c + a * n)):
            bound = 4 * U * (a.abs() + b.abs()) + 2.0 ** -8 * y.abs() + 1e-30
            assert bool(((got[s, 0, i].double() - y).abs() <= bound).all())
