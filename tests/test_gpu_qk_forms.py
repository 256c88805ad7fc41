"""Head norms with the rotation at row counts where two heads of a row share a group of lanes, in every instance of it.

CASES says which kernel each size takes; tests/test_op_forms.py holds the library to it on the CPU.  The tolerance is that of
test_gpu_qk."""
import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import ops_ref_torch as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

# (type, rows, q heads, k heads, head dim, rotated dims, kernel: type, values of a run, lanes, runs, heads)
CASES = [
    ("bf16", 2051, 16, 16, 64, 64, "bf16,8,4,1,2"), ("bf16", 16390, 2, 2, 64, 64, "bf16,8,4,1,2"), ("bf16", 2055, 12, 4, 128, 128, "bf16,8,8,1,2"),
    ("bf16", 4100, 6, 2, 96, 48, "bf16,8,8,1,2"), ("bf16", 1030, 14, 2, 256, 256, "bf16,8,16,1,2"), ("bf16", 2060, 24, 8, 24, 16, "bf16,4,4,1,2"),
    ("bf16", 1029, 24, 8, 56, 56, "bf16,4,8,1,2"), ("bf16", 1024, 16, 16, 72, 72, "bf16,4,16,1,2"), ("bf16", 1025, 12, 4, 72, 40, "bf16,4,16,1,2"),
    ("bf16", 4100, 12, 4, 12, 12, "bf16,2,4,1,2"), ("bf16", 2049, 12, 4, 28, 20, "bf16,2,8,1,2"), ("bf16", 1031, 14, 2, 44, 44, "bf16,2,16,1,2"),
    ("f32", 2051, 16, 16, 32, 32, "float,4,4,1,2"), ("f32", 2051, 12, 4, 64, 64, "float,4,8,1,2"), ("f32", 1024, 16, 16, 72, 72, "float,4,16,1,2"),
    ("f32", 1031, 14, 2, 128, 64, "float,4,16,1,2"), ("f32", 4101, 12, 4, 12, 12, "float,2,4,1,2"), ("f32", 2051, 12, 4, 28, 28, "float,2,8,1,2"),
    ("f32", 1025, 12, 4, 60, 20, "float,2,16,1,2"),
]


def make(dtype, rows, hq, hk, d, rot):
    g = torch.Generator("cuda").manual_seed(rows + d)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    t = [(rnd(rows, h, d) * 1.5).to(DT[dtype]) for h in (hq, hk)] + [(rnd(d) * 0.1 + m).to(DT[dtype]) for m in (1.0, 1.0, 0.0, 0.0)]
    ang = torch.rand(rows, rot // 2, device="cuda", generator=g, dtype=torch.float64) * 2000 - 1000
    return (*t, torch.stack([ang.cos(), ang.sin()], -1).float())


def check(got, x, g, b, norm, table, pairing):
    n, r, mean = ref.head_norm(x, g, b, norm, 1e-6)
    gain = 1.0 if g is None else g.double().abs()
    base = n.abs() + (0.0 if b is None else b.double().abs())
    err = torch.zeros_like(n) if norm is None else 16 * U * base + (24 * U * mean * r * gain if norm == "layer" else 0.0)
    y = ref.rotate(n, table, pairing)
    a, c = ref.pair_slices(table.shape[1], pairing)

    def both(v):  # |v_a| + |v_b| for both members of a pair
        s = v.clone()
        s[..., a] = s[..., c] = v[..., a] + v[..., c]
        return s

    err = both(err) + 4 * U * both(n.abs())
    bound = err + torch.finfo(x.dtype).eps / 2 * (y.abs() + err) + 1e-30
    d = (got.double() - y).abs()
    assert bool((d <= bound).all()), float((d / bound).max())


@pytest.mark.parametrize("norm,pairing", [("rms", "halves"), ("layer", "adjacent"), (None, "adjacent"), ("layer", "halves")])
@pytest.mark.parametrize("dtype,rows,hq,hk,d,rot,form", CASES)
def test_two_heads_to_a_group(norm, pairing, dtype, rows, hq, hk, d, rot, form):
    q, k, qg, kg, qb, kb, table = make(dtype, rows, hq, hk, d, rot)
    if norm != "layer":
        qb = kb = None
    qo, ko = incvit.qk_norm_rope(q, k, table, pairing, norm, qg, kg, qb, kb)
    if norm is None:
        qg = kg = None
    check(qo, q, qg, qb, norm, table, pairing)
    check(ko, k, kg, kb, norm, table, pairing)


@pytest.mark.parametrize("dtype,d", [("bf16", 72), ("bf16", 64), ("f32", 64)])
def test_padding_a_cache_and_views(dtype, d):
    """q and k inside a projection's output, padding rows, keys into a cache; then in place.  The values are those of single
    heads, which take another instance, to the last bit or two: the bound above."""
    rows, h, n = 2100, 16, 2500
    q, k, qg, kg, _, _, table = make(dtype, rows, h, h, d, d)
    big = torch.cat([table, table[:400]])  # 2500 table rows
    x = torch.cat([q.reshape(rows, -1), k.reshape(rows, -1), q.reshape(rows, -1)], dim=1).contiguous()
    qv, kv = x[:, :h * d].unflatten(1, (h, d)), x[:, h * d:2 * h * d].unflatten(1, (h, d))
    g = torch.Generator("cuda").manual_seed(1)
    index = torch.randint(0, n, (rows,), device="cuda", generator=g, dtype=torch.int32)
    dst = torch.randperm(n, device="cuda", generator=g)[:rows].int()
    index[5::11], dst[7::13] = -1, n
    qo, ko = torch.full_like(q, 9.0), torch.full((n, h, d), 9.0, dtype=q.dtype, device="cuda")
    keep = x.clone()
    incvit.qk_norm_rope(qv, kv, big, q_gamma=qg, k_gamma=kg, index=index, k_rows=dst, q_out=qo, k_out=ko)
    assert torch.equal(x, keep)
    live = index >= 0
    check(qo[live], q[live], qg, None, "rms", big[index[live].long()], "halves")
    assert bool((qo[~live] == 9.0).all())
    put = live & (dst < n)
    check(ko[dst[put].long()], k[put], kg, None, "rms", big[index[put].long()], "halves")
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[dst[put].long()] = False
    assert bool((ko[rest] == 9.0).all())
    a, b = incvit.qk_norm_rope(qv, kv, table, q_gamma=qg, k_gamma=kg)
    incvit.qk_norm_rope(qv, kv, table, q_gamma=qg, k_gamma=kg, q_out=qv, k_out=kv)
    assert torch.equal(qv, a) and torch.equal(kv, b) and torch.equal(x[:, 2 * h * d:], keep[:, 2 * h * d:])
    one, _ = incvit.qk_norm_rope(q[:64], None, table[:64], q_gamma=qg)  # one head to a group
    assert torch.equal(one, a[:64])
