"""8-bit products on the GPU against exact integer sums: sizes around every tile, types, GELU, residual, strides, alignments,
integer weights, a LayerNorm before the rows, rows that are zero or not finite, streams and captured calls.

Tolerance, u = 2^-24: the integers and scales are those of the definition, bit for bit (each is one rounded division), and so
is the sum; its conversion, the product of the scales and the fused multiply-add round once each: 3 u of |sum s s| and 1 u of
the result.  GELU multiplies an error by at most 1.13 and is x / (1 + 2^t) with t rounded three times (3 u |t| ln 2 of
2^t / (1 + 2^t) <= 1) and the hardware's exponential and reciprocal, one ulp (2 u) each: (5 + 3 |t|) u of the result; below
2^-126 it may be flushed.  The residual adds 1 u.  Then one rounding to the output type, finfo.eps / 2 of the value."""
import numpy as np
import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import ops_ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.double().cpu().numpy()


def want_and_bound(xq, xs, wq, ws, b, gelu, res, dtype):
    z = (xq @ wq) * xs * ws
    y = z + (0.0 if b is None else f64(b))
    err = 3 * U * np.abs(z) + U * np.abs(y)
    if gelu:
        t = 2.0 * np.sqrt(2.0 / np.pi) * np.abs(y + 0.044715 * y ** 3) * 1.4427
        y, err = ops_ref.gelu(y), 1.13 * err + (5 + 3 * t) * U * np.abs(ops_ref.gelu(y)) + 2.0 ** -126
    if res is not None:
        y = y + f64(res)
        err = err + U * np.abs(y)
    return y, err + torch.finfo(dtype).eps / 2 * (np.abs(y) + err) + 1e-38


def check(got, want):
    y, bound = want
    g = f64(got)
    nan = np.isnan(y)
    assert np.array_equal(np.isnan(g), nan)
    d = np.where(nan, 0.0, np.abs(g - y))
    assert np.all(d <= np.where(nan, 1.0, bound)), np.nanmax(d / bound)


def make(rows, K, N, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + rows * 31 + K * 7 + N)
    x = torch.randn(rows, K, generator=g) * (torch.rand(rows, 1, generator=g) * 3 + 0.05)
    w = torch.randn(K, N, generator=g) * 0.03 * (torch.rand(1, N, generator=g) + 0.3)
    b, r = torch.randn(N, generator=g) * 0.1, torch.randn(rows, N, generator=g)
    return tuple(t.to(DT[dtype]).cuda() for t in (x, w, b, r))


def run(x, w, b, r, gelu, lin=None, **kw):
    lin = lin or incvit.QLinear(w, b)
    got = lin(x, gelu=gelu, residual=r, **kw)
    xq, xs = ops_ref.quantized(f64(x), 1)
    wq, ws = ops_ref.quantized(f64(w), 0)
    check(got, want_and_bound(xq, xs, wq, ws, b, gelu, r, x.dtype))
    return lin, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N", [(1, 1, 1), (1, 64, 16), (1, 1152, 4304), (2, 7, 3), (16, 65, 17), (17, 100, 50), (23, 1152, 1013),
                                      (33, 200, 31), (64, 128, 48), (100, 777, 130), (128, 64, 64), (129, 64, 64), (130, 70, 1),
                                      (257, 1000, 1013), (300, 4304, 160), (546, 130, 99), (1024, 192, 768), (2050, 65, 515),
                                      (3000, 512, 1536)])
def test_sizes(dtype, rows, K, N):
    x, w, b, r = make(rows, K, N, dtype)
    lin, _ = run(x, w, b, None, False)
    run(x, w, b, r, False, lin)
    run(x, w, b, None, True, lin)


@pytest.mark.parametrize("rows,K,N,dtype", [(8192, 256, 4096, "bf16"), (4100, 65, 4111, "f32"), (9000, 1024, 1152, "bf16")])
def test_many_tiles(rows, K, N, dtype):
    x, w, b, r = make(rows, K, N, dtype)
    run(x, w, None, r, True)


def test_longest_sum_is_exact():
    """K = 65536 of the largest integers: the sum is 65536 * 127^2 and needs every bit of int32."""
    K = 65536
    x = torch.ones(3, K, device="cuda")
    x[1] = -1.0
    w = torch.ones(K, 2, device="cuda")
    lin = incvit.QLinear(w)
    got = f64(lin(x))
    s = np.float64(np.float32(1.0) / np.float32(127.0))
    assert np.all(np.abs(np.abs(got) - K * 127.0 ** 2 * s * s) <= 4 * U * K)
    assert (got[1] < 0).all() and (got[0] > 0).all()
    # and every row count's kernel
    big = lin(torch.ones(200, K, device="cuda"))
    assert torch.equal(big[0], lin(x)[0])


@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 1, 4, 8])
def test_strides_alignments_and_guards(rows, dtype, pad):
    """x, residual and out inside wider rows that start at any element; what lies around the output stays."""
    K, N = 136, 52
    x0, w, b, r0 = make(rows, K, N, dtype)
    wide = lambda t: torch.full((rows, t.shape[1] + 2 * pad + 3), 7.0, dtype=t.dtype, device="cuda")  # noqa: E731
    xb, rb, ob = wide(x0), wide(r0), wide(r0)
    x, r, o = xb[:, pad:pad + K], rb[:, pad:pad + N], ob[:, pad:pad + N]
    x.copy_(x0)
    r.copy_(r0)
    run(x, w, b, r, False, out=o)
    assert torch.all(ob[:, :pad] == 7.0) and torch.all(ob[:, pad + N:] == 7.0)
    assert torch.equal(x, x0) and torch.equal(r, r0)
    keep = o.clone()
    incvit.QLinear(w, b)(x, residual=r, out=r)  # in place on the residual
    assert torch.equal(r, keep)
    assert torch.all(rb[:, pad + N:] == 7.0)


def test_broadcast_rows_and_residual():
    x, w, b, r = make(1, 96, 40, "bf16")
    lin = incvit.QLinear(w, b)
    one = lin(x, residual=r)
    many = lin(x.expand(300, 96), residual=r.expand(300, 40))
    assert torch.equal(many, one.expand(300, 40))


def test_no_rows():
    x, w, b, _ = make(1, 96, 40, "bf16")
    lin = incvit.QLinear(w, b)
    assert lin(x[:0]).shape == (0, 40)
    assert lin(incvit.quantize_rows(x[:0])).shape == (0, 40)


@pytest.mark.parametrize("rows", [6, 200])
def test_zeros_extremes_and_rows_that_are_not_finite(rows):
    x, w, b, _ = make(rows, 130, 70, "f32")
    x[0] = 0.0
    x[1] *= 1e30
    x[2] *= 1e-30
    x[3, 129] = float("nan")
    x[4, 0] = float("inf")
    x[5] = torch.full((130,), 1e-42)  # a scale below the normal numbers
    w[:, 3] = 0.0
    w[:, 5] *= 1e-20
    run(x, w, b, None, False)
    w[7, 9] = float("-inf")
    _, got = run(x, w, b, None, False)
    assert torch.isnan(got[:, 9]).all() and torch.isnan(got[3]).all() and torch.isnan(got[4]).all()
    assert torch.isfinite(got[0, :9]).all()


def test_ties_go_to_even():
    """127 / 254 of the row's largest value, and its odd multiples, lie halfway between two integers."""
    top = 127.0
    x = torch.tensor([[top] + [i + 0.5 for i in range(-60, 60)]], device="cuda")
    w = torch.eye(121, device="cuda")
    got = f64(incvit.QLinear(w)(x))[0]
    want = np.array([top] + [np.rint(i + 0.5) for i in range(-60, 60)])
    assert np.all(np.abs(got - want) <= 4 * U * 127)  # scales 1 and 1 / 127, integers 127 and the rounded ones


def test_weights_stored_by_channel_and_integer_weights():
    x, w, b, _ = make(40, 200, 88, "bf16")
    want = incvit.QLinear(w, b)(x)
    assert torch.equal(incvit.QLinear(w.t().contiguous().t(), b)(x), want)
    wq, ws = ops_ref.quantized(f64(w), 0)
    q8 = torch.from_numpy(wq.astype(np.int8)).cuda()
    sc = torch.from_numpy(ws[0].astype(np.float32)).cuda()
    assert torch.equal(incvit.QLinear(q8, b.float(), scales=sc)(x), want)
    assert torch.equal(incvit.QLinear(q8.t().contiguous().t(), b.float(), scales=sc)(x), want)
    q8[0] = -128  # integers that the library would not make
    xq, xs = ops_ref.quantized(f64(x), 1)
    check(incvit.QLinear(q8, scales=sc)(x), want_and_bound(xq, xs, f64(q8), f64(sc), None, False, None, torch.bfloat16))


@pytest.mark.parametrize("rows", [20, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [72, 777, 1152, 1500, 4304])
def test_rows_behind_a_layernorm(rows, dtype, K):
    """The norm is in fp32, so a quotient within its error of a border may round to either side: the bound counts one step
    for each such value.  A lane adds at most 8 * 9 terms (K <= 4608) and six steps join the lanes: 78 u of mean |x| for the
    mean, 39 u of a normed value for its root, 6 u for the division, products and the sum: below 96 u of |n| + |beta| + mean
    |x| * factor * gain in all."""
    x, w, b, _ = make(rows, K, 60, dtype)
    g = torch.Generator().manual_seed(K)
    gamma = (1 + 0.2 * torch.randn(K, generator=g)).to(DT[dtype]).cuda()
    beta = (0.2 * torch.randn(K, generator=g)).to(DT[dtype]).cuda()
    lin = incvit.QLinear(w, b)
    q = incvit.quantize_rows(x, gamma, beta, 1e-6)
    got = lin(q)
    assert torch.equal(lin(q), got)  # the rows serve several products
    n, r, mean = ops_ref.head_norm(f64(x), f64(gamma), f64(beta), "layer", 1e-6)
    xq, xs = ops_ref.quantized(n, 1)
    wq, ws = ops_ref.quantized(f64(w), 0)
    y, bound = want_and_bound(xq, xs, wq, ws, b, False, None, DT[dtype])
    err = 96 * U * (np.abs(n) + np.abs(f64(beta)) + mean * r * np.abs(f64(gamma)))
    ratio = n / xs
    near = np.abs(np.abs(ratio - np.floor(ratio)) - 0.5) <= 2 * err / xs + 8 * U * np.abs(ratio)
    assert near.mean() < 0.02  # the bound below says something
    scale_err = (err / np.abs(n).max(axis=1, keepdims=True)).max(axis=1, keepdims=True)
    bound = bound + (near.astype(float) @ np.abs(wq)) * xs * ws + (scale_err + 4 * U) * np.abs((xq @ wq) * xs * ws)
    d = np.abs(f64(got) - y)
    assert np.all(d <= bound * 1.01), (d / bound).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,N", [(1152, 176), (2048, 40), (2056, 48), (5000, 33), (6144, 24), (1001, 50), (63, 8)])
def test_a_few_tokens_in_one_launch(dtype, K, N):
    """Up to 8 rows are quantised by the product itself: the same bits as in two steps, and as 9 rows that are not."""
    x, w, b, r = make(9, K, N, dtype)
    x[4] = 0.0
    x[6, K - 1] = float("inf")
    lin = incvit.QLinear(w, b)
    nine = lin(x, residual=r)
    for rows in (1, 2, 5, 7, 8):
        got = lin(x[:rows], residual=r[:rows])
        assert torch.equal(got.nan_to_num(7.0), nine[:rows].nan_to_num(7.0))
        two = lin(incvit.quantize_rows(x[:rows]), residual=r[:rows])
        assert torch.equal(got.nan_to_num(7.0), two.nan_to_num(7.0))
    keep = x[:3].clone()
    wide = torch.full((3, K + 5), float("nan"), dtype=x.dtype, device="cuda")  # what follows a row is not read into it
    wide[:, :K] = keep
    assert torch.equal(lin(wide[:, :K]), lin(keep))


def test_quantised_rows_serve_products_of_other_widths():
    x, w, b, _ = make(50, 320, 96, "bf16")
    a, c = incvit.QLinear(w, b), incvit.QLinear(w[:, :40].contiguous())
    q = incvit.quantize_rows(x)
    assert torch.equal(a(q), a(x)) and torch.equal(c(q), c(x))


@pytest.mark.parametrize("rows", [23, 700])
def test_another_stream_and_captured_calls(rows):
    x, w, b, _ = make(rows, 320, 272, "bf16")
    lin = incvit.QLinear(w, b)
    want = lin(x, gelu=True)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = lin(x, gelu=True)
    st.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lin(x, gelu=True, out=out)
    for seed in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, lin(x, gelu=True))


def test_the_front_of_an_attention_layer():
    """The operators as they are used together: a LayerNorm and an 8-bit projection to queries, keys and values, norms and
    rotation by a grid's table with the new keys scattered into the cache, against the same in 64 bits from the integers."""
    N, D, H = 256, 576, 8
    d = D // H
    g = torch.Generator().manual_seed(9)
    x = torch.randn(23, D, generator=g).to(torch.bfloat16).cuda()
    w = (torch.randn(D, 3 * D, generator=g) * 0.04).to(torch.bfloat16).cuda()
    b = (torch.randn(3 * D, generator=g) * 0.02).to(torch.bfloat16).cuda()
    gq, gk = ((1 + 0.1 * torch.randn(d, generator=g)).to(torch.bfloat16).cuda() for _ in range(2))
    tok = torch.randperm(N, generator=g)[:23].sort().values.int().cuda()
    cache = torch.randn(N, H, d, generator=g).to(torch.bfloat16).cuda()
    before = cache.clone()
    table = incvit.rope_table(incvit.make_rope(d, (d // 4, d // 4)), grids=[(1, 16, 16)])
    qkv = incvit.QLinear(w, b)(x)
    q, k = qkv[:, :D].view(23, H, d), qkv[:, D:2 * D].view(23, H, d)
    q, _ = incvit.qk_norm_rope(q, k, table, q_gamma=gq, k_gamma=gk, index=tok, k_rows=tok, k_out=cache)
    xq, xs = ops_ref.quantized(f64(x), 1)
    wq, ws = ops_ref.quantized(f64(w), 0)
    y, _ = want_and_bound(xq, xs, wq, ws, b, False, None, torch.bfloat16)
    pos = ops_ref.grid_positions([(1, 16, 16)], 1, 2)[:, tok.cpu().numpy()]
    ang = ops_ref.rope_angles(pos, (d // 4, d // 4))
    for got, part, gain in ((q, 0, gq), (cache[tok.long()], 1, gk)):
        n, _, _ = ops_ref.head_norm(y[:, part * D:(part + 1) * D].reshape(23, H, d), f64(gain), None, "rms", 1e-6)
        want = ops_ref.rotate(n, np.cos(ang), np.sin(ang), "halves")
        # the projection rounds to bf16 (2^-8 of each value; a norm and a rotation pass it on), then the result does
        bound = 2 * 2.0 ** -8 * (np.abs(n).max(axis=-1, keepdims=True) * 1.5) + 2.0 ** -8 * np.abs(want)
        assert np.all(np.abs(f64(got) - want) <= bound)
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[tok.long()] = False
    assert torch.equal(cache[rest], before[rest])


def test_more_rows_than_one_launch_counts():
    """70 million rows of one value: each is its own scale, so the integers are +-127 (or 0) and the product is known."""
    rows = 70_000_003
    x = torch.randn(rows, 1, device="cuda", generator=torch.Generator("cuda").manual_seed(6)).to(torch.bfloat16)
    w = torch.tensor([[0.75]], device="cuda", dtype=torch.bfloat16)
    got = incvit.QLinear(w)(x)
    for lo in range(0, rows, 1 << 24):
        y = x[lo:lo + (1 << 24)].double() * 0.75
        # two scales rounded to fp32, their product and the sum's scaling: 5 u, then bf16
        assert bool(((got[lo:lo + (1 << 24)].double() - y).abs() <= (5 * U + 2.0 ** -8) * y.abs() + 1e-38).all())


@pytest.mark.parametrize("rows,K,N,dtype", [(1000, 1100, 1160, "bf16"), (1024, 260, 1280, "f32"), (1000, 4304, 1152, "bf16"),
                                            (300, 1152, 4312, "bf16"), (1024, 2500, 1084, "f32"), (641, 1024, 2040, "bf16")])
def test_tiles_of_96_columns(rows, K, N, dtype):
    """More than 256 tiles of 64 x 64 and at most 256 of 64 x 96, with column blocks and chunks that do not fill the last."""
    x, w, b, r = make(rows, K, N, dtype)
    lin, _ = run(x, w, b, None, True)
    run(x, w, b, r, False, lin)


@pytest.mark.parametrize("rows", [1, 8, 9, 300])
def test_output_over_the_input(rows):
    """The rows are read before any output is written: in place, shifted by a row's half, and beside each other in one buffer."""
    K = 640
    x, w, b, _ = make(rows, K, K, "bf16")
    lin = incvit.QLinear(w, b)
    want = lin(x)
    y = x.clone()
    lin(y, out=y)
    assert torch.equal(y, want)
    buf = torch.zeros(rows * K + K // 2, device="cuda", dtype=x.dtype)
    src = buf[:rows * K].view(rows, K)
    src.copy_(x)
    out = buf[K // 2:].view(rows, K)
    lin(src, out=out)
    assert torch.equal(out, want)
    pair = torch.cat([x, torch.zeros_like(x)], dim=1)
    lin(pair[:, :K], out=pair[:, K:])
    assert torch.equal(pair[:, K:], want) and torch.equal(pair[:, :K], x)
