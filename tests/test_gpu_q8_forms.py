"""8-bit products on every tile shape of the large-row GEMM and every form of the few-row kernel, at sizes where the last
tiles, column blocks and staged chunks are not full, and the quantised rows themselves, bit for bit.

FORMS says which kernel each size takes; tests/test_op_forms.py holds the library to it on the CPU.  The tolerance of the
products is that of test_gpu_qlinear."""
import math

import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import ops_ref_torch as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# (rows, K, N, kernel: its template arguments past the epilogue); N is a multiple of 8, and N + 1 ends off 16 bytes
FORMS = [
    (20, 100, 64, "q_gemm 1,2"), (17, 2500, 64, "q_gemm 1,4"), (23, 1152, 4304, "q_gemm 2,2"), (100, 320, 1032, "q_gemm 2,2"),
    (40, 2200, 4304, "q_gemm 2,4"), (500, 449, 1144, "q_gemm 4,2"), (300, 4304, 808, "q_gemm 4,4"),
    (770, 430, 1144, "gemm_tiled 64,64,2,2,8"), (200, 1000, 4096, "gemm_tiled 64,64,2,2,8"),
    (1000, 333, 1152, "gemm_tiled 64,96,4,4,4"), (1030, 520, 1144, "gemm_tiled 64,96,4,4,4"),
    (1024, 257, 2040, "gemm_tiled 64,128,2,2,6"), (130, 70, 9000, "gemm_tiled 64,128,2,2,6"),
    (2050, 330, 1920, "gemm_tiled 256,128,4,1,6"), (4352, 70, 1016, "gemm_tiled 256,128,4,1,6"),
    (2048, 200, 2000, "gemm_tiled 128,128,2,1,8"), (1930, 700, 2024, "gemm_tiled 128,128,2,1,8"),
    (4300, 70, 2040, "gemm_tiled 128,128,2,1,4"),
    (4090, 330, 4088, "gemm_tiled 256,256,2,1,4"), (8190, 130, 4088, "gemm_tiled 256,256,2,1,4"),
]
# the same for outputs of N + 1 columns
FORMS_ANY = [
    (20, 100, 65, "q_gemm 1,2"), (17, 2500, 65, "q_gemm 1,4"), (100, 320, 1033, "q_gemm 2,2"), (40, 2200, 4305, "q_gemm 2,4"),
    (500, 449, 1145, "q_gemm 4,2"), (300, 4304, 809, "q_gemm 4,4"), (770, 430, 1145, "gemm_tiled 64,64,2,2,8"),
    (1030, 333, 1145, "gemm_tiled 64,96,4,4,4"), (400, 700, 4305, "gemm_tiled 64,128,2,2,6"), (2500, 330, 2041, "gemm_tiled 256,128,4,1,6"),
    (2048, 200, 2001, "gemm_tiled 128,128,2,1,8"), (4090, 330, 4089, "gemm_tiled 128,128,2,1,4"), (8190, 70, 1985, "gemm_tiled 128,128,2,1,4"),
]


def make(rows, K, N, dtype):
    g = torch.Generator("cuda").manual_seed(rows * 31 + K * 7 + N)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    x = rnd(rows, K) * (rnd(rows, 1).abs() * 3 + 0.05)
    w = rnd(K, N) * 0.03 * (rnd(1, N).abs() + 0.3)
    return tuple(t.to(DT[dtype]) for t in (x, w, rnd(N) * 0.1, rnd(rows, N)))


def check(got, x, w, b, gelu, res):
    xq, xs = ref.quantized(x, 1)
    wq, ws = ref.quantized(w, 0)
    z = (xq @ wq) * xs * ws
    y = z + b.double()
    err = 3 * U * z.abs() + U * y.abs()
    if gelu:
        t = 2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3).abs() * 1.4427
        y = ref.gelu(y)
        err = 1.13 * err + (5 + 3 * t) * U * y.abs() + 2.0 ** -126
    if res is not None:
        y = y + res.double()
        err = err + U * y.abs()
    bound = err + torch.finfo(x.dtype).eps / 2 * (y.abs() + err) + 1e-38
    d = (got.double() - y).abs()
    assert bool((d <= bound).all()), float((d / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N,form", FORMS + FORMS_ANY)
def test_forms(dtype, rows, K, N, form):
    x, w, b, r = make(rows, K, N, dtype)
    lin = incvit.QLinear(w, b)
    guard = torch.full((rows + 2, N), 7.0, dtype=x.dtype, device="cuda")
    if N % 8 == 0:
        out = guard[1:-1]
    else:
        out = guard.view(-1)[N:-N].view(rows, N)  # starts off 16 bytes
    lin(x, out=out)
    check(out, x, w, b, False, None)
    assert bool((guard[0] == 7.0).all() and (guard[-1] == 7.0).all())
    check(lin(x, gelu=True), x, w, b, True, None)
    check(lin(x, residual=r), x, w, b, False, r)
    keep = r.clone()
    assert torch.equal(lin(x, residual=r, out=r), lin(x, residual=keep))  # in place


def rows_held(q):
    """(integers [rows][K], scales [rows]) of quantised rows, from the operands' order: 16 rows by 64 values are a kilobyte, in
    which 16 values of one row follow one another, then the 16 rows, then the four runs of 16 values."""
    tiles, kc = (q.rows + 15) // 16, (q.K + 63) // 64
    n = tiles * kc * 1024
    v = q.buf[:n].view(torch.int8).view(tiles, kc, 4, 16, 16).permute(0, 3, 1, 2, 4).reshape(tiles * 16, kc * 64)
    at = (n + 255) // 256 * 256
    return v[:q.rows], q.buf[at:at + 4 * q.rows].view(torch.float32)


def same_rows(x):
    """The integers and scales of x are the definition's, the padding of the last chunk zeros."""
    q, s = rows_held(incvit.quantize_rows(x))
    wq, ws = ref.quantized(x, 1)
    assert torch.equal(s.double(), ws[:, 0])
    assert torch.equal(q[:, :x.shape[1]].double(), wq)
    assert not q[:, x.shape[1]:].any()


@pytest.mark.parametrize("exponent", [0, -1, 89, 96, 97, 100, 126, -80, -83, -84, -90, -110, -120])
def test_every_pair_of_bf16_significands(exponent):
    """A row for each significand of the largest magnitude (its exponent given), which holds every significand of the exponents
    from there to ten below, either sign: all quotients of a largest bf16 value above a quarter, either side of the range that is
    quantised without a division."""
    sig = torch.arange(128, 256, device="cuda").double() / 128
    drop = 2.0 ** -torch.arange(10, device="cuda").double()
    vals = (sig[None, :] * drop[:, None]).reshape(-1)
    x = torch.cat([vals, -vals])[None, :].expand(128, -1)
    x = torch.where(x.abs() <= sig[:, None], x, torch.zeros_like(x))
    x = torch.cat([sig[:, None], x], dim=1)
    x = (x * 2.0 ** exponent).to(torch.bfloat16)
    assert torch.equal(x.double()[:, 0], sig * 2.0 ** exponent)  # bf16 holds them
    same_rows(x)


@pytest.mark.parametrize("scale", [1.0, 1e-24, 1e-27, 1e27, 1e32, 3e-37])
def test_fp32_values_around_every_border(scale):
    """For 4096 largest magnitudes the values next to (n + 1/2) * scale, n = 0 .. 126, and two steps to either side."""
    g = torch.Generator("cuda").manual_seed(4)
    top = ((torch.rand(4096, 1, device="cuda", generator=g) + 1.0) * scale).float()
    s = (top.double() / 127).float()
    mid = ((torch.arange(127, device="cuda").double() + 0.5) * s.double()).float()
    up = torch.full_like(mid, math.inf)
    steps = [mid]
    for to in (up, -up):
        v = mid
        for _ in range(2):
            v = torch.nextafter(v, to)
            steps.append(v)
    x = torch.cat([top] + steps + [-v for v in steps], dim=1)
    same_rows(torch.where(x.abs() <= top, x, top))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(1, 1), (37, 63), (300, 1024), (19, 1025), (50, 2048), (33, 2051), (21, 6144), (21, 6145), (37, 6152),
                                    (5, 7001), (18, 20000), (3, 65536)])
def test_integers_of_random_rows(dtype, rows, K):
    x, _, _, _ = make(rows, K, 1, dtype)
    same_rows(x)
    wide = torch.full((rows, K + 3), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, 1:K + 1] = x  # unaligned, with what no row may take in around it
    same_rows(wide[:, 1:K + 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,N", [(1, 6152, 40), (2, 20000, 33), (6, 7001, 56), (7, 6200, 16), (1, 48000, 24), (20, 6152, 40),
                                      (40, 9001, 33), (600, 6200, 1152)])
def test_long_rows(dtype, rows, K, N):
    """K past what a workgroup holds in registers: one launch for a few tokens, two for more."""
    x, w, b, r = make(rows, K, N, dtype)
    lin = incvit.QLinear(w, b)
    got = lin(x, residual=r)
    check(got, x, w, b, False, r)
    assert torch.equal(lin(incvit.quantize_rows(x), residual=r), got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K", [(20, 1152), (20, 6152), (5, 7001), (40, 16000)])
def test_integers_behind_a_layernorm(dtype, rows, K):
    """The norm is in fp32: below 96 u of |n| + |beta| + mean |x| * factor * gain, as test_gpu_qlinear counts it (a lane adds at
    most 8 * 8 terms here, K <= 16384, and nine steps join them).  The scale is off by at most the largest value's error and its
    own rounding, an integer by one and only where the quotient is that near a border."""
    x, _, _, _ = make(rows, K, 1, dtype)
    g = torch.Generator("cuda").manual_seed(K)
    gamma = (1 + 0.2 * torch.randn(K, device="cuda", generator=g)).to(DT[dtype])
    beta = (0.2 * torch.randn(K, device="cuda", generator=g)).to(DT[dtype])
    q, s = rows_held(incvit.quantize_rows(x, gamma, beta, 1e-6))
    n, f, mean = ref.head_norm(x, gamma, beta, "layer", 1e-6)
    err = 96 * U * (n.abs() + beta.double().abs() + mean * f * gamma.double().abs())
    wq, ws = ref.quantized(n, 1)
    top = n.abs().amax(dim=1, keepdim=True)
    rel = (err.amax(dim=1, keepdim=True) / top) + 2 * U
    assert bool(((s.double()[:, None] - ws).abs() <= rel * ws).all())
    ratio = (n / ws).abs()
    near = (ratio - ratio.floor() - 0.5).abs() <= err / ws + (rel + 2 * U) * ratio
    assert float(near.double().mean()) < 0.02  # the check below says something
    d = (q[:, :K].double() - wq).abs()
    assert bool((d <= near.double()).all())
    assert not q[:, K:].any()
