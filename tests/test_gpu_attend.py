"""Attention over the cache in 8 bits and over given keys and values on the GPU, against 64-bit arithmetic: types, head sizes,
groups, lengths, masks, ragged batches, splits over workgroups, strides, what masked places hold, streams and captured calls.
The bound is derived in kv_ref.attention."""
import math

import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import kv_ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def randn(*shape, dtype="bf16", seed=0):
    g = torch.Generator().manual_seed(seed + 7 * shape[0] + shape[-1])
    return torch.randn(*shape, generator=g).to(DT[dtype]).cuda()


def starts(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


def starts_of(lens):
    return torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


class Cached:
    """Sequences in a pool of shuffled blocks, and the values that the cache holds for them in 64 bits."""

    def __init__(self, lens, hk, d, dtype="bf16", block=16, k=None, v=None, spare=2):
        n = sum(lens)
        need = [-(-m // block) for m in lens]
        order = torch.randperm(sum(need) + spare, generator=torch.Generator().manual_seed(n)).tolist()
        self.table = torch.full((len(lens), max(need + [1])), -1, dtype=torch.int32)
        slots, at = [], 0
        for i, m in enumerate(lens):
            self.table[i, :need[i]] = torch.tensor(order[at:at + need[i]], dtype=torch.int32)
            slots += [order[at + t // block] * block + t % block for t in range(m)]
            at += need[i]
        self.lens, self.table = torch.tensor(lens, dtype=torch.int32, device="cuda"), self.table.cuda()
        k = randn(n, hk, d, dtype=dtype, seed=1) if k is None else k
        v = randn(n, hk, d, dtype=dtype, seed=2) if v is None else v
        self.cache = incvit.KVCache(len(order), hk, d, block=block)
        self.cache.write(k, v, torch.tensor(slots, dtype=torch.int32, device="cuda"), begin=True)
        self.k, self.v = [], []
        for x, out in ((k, self.k), (v, self.v)):
            held = kv_ref.Held(len(order), hk, d, block)
            held.write(x, slots, True)
            y, at = held.exact()[slots].cuda(), 0
            for m in lens:
                out.append(y[at:at + m])
                at += m

    def attend(self, q, **kw):
        return self.cache.attend(q, self.table, self.lens, **kw)


class Plain:
    def __init__(self, lens, hk, d, dtype="bf16", block=None, k=None, v=None):
        n = sum(lens)
        self.ka = randn(n, hk, d, dtype=dtype, seed=1) if k is None else k
        self.va = randn(n, hk, d, dtype=dtype, seed=2) if v is None else v
        self.start = starts(lens)
        self.k, self.v = self.ka.split(lens), self.va.split(lens)

    def attend(self, q, q_start=None, **kw):
        if q_start is None:
            n = len(self.k)
            q_start = torch.arange(n + 1, dtype=torch.int32, device="cuda") * (q.shape[0] // n)
        return incvit.attend(q, self.ka, self.va, q_start=q_start, k_start=self.start, **kw)


KINDS = {"cached": Cached, "plain": Plain}
both = pytest.mark.parametrize("kind", ["cached", "plain"])
types = pytest.mark.parametrize("dtype", ["bf16", "f32"])


def compare(got, x, q, new, scale=None, **mask):
    at = 0
    for k, v, n in zip(x.k, x.v, new):
        see = kv_ref.visible(n, k.shape[0], device="cuda", **mask)
        want, bound = kv_ref.attention(q[at:at + n], k, v, see, scale)
        kv_ref.check(got[at:at + n], want, bound)
        at += n


def run(kind, lens, new, hq, hk, d, dtype="bf16", block=16, scale=None, **mask):
    x = KINDS[kind](lens, hk, d, dtype, block)
    q = randn(sum(new), hq, d, dtype=dtype, seed=3)
    same = len(set(new)) == 1
    got = x.attend(q, q_start=None if same else starts(new), scale=scale, **mask)
    assert got.dtype == q.dtype and got.shape == q.shape
    compare(got, x, q, new, scale, **mask)
    return x, q, got


@both
@types
@pytest.mark.parametrize("d", [8, 32, 40, 64, 72, 80, 96, 120, 128, 136, 192, 200, 256])
@pytest.mark.parametrize("nq", [1, 5, 9, 70])  # one, two and four row tiles to a workgroup, and several workgroups
def test_head_sizes(kind, dtype, d, nq):
    run(kind, [99, 99], [nq, nq], 4, 1, d, dtype)


@both
@types
@pytest.mark.parametrize("d", [8, 40, 64, 80, 96, 128, 136, 192, 256])
@pytest.mark.parametrize("nq", [1, 30, 150])
def test_keys_shared_by_workgroups(kind, dtype, d, nq):
    run(kind, [3000, 3000], [nq, nq], 8, 2, d, dtype)


@pytest.mark.parametrize("d", [8, 32, 40, 64, 72, 80, 96, 120, 128, 136, 192, 200, 256])
@pytest.mark.parametrize("mask", [dict(causal=False), dict(window=150, sinks=3)])
def test_thousands_of_rows(d, mask):
    """So many that a wave has two row tiles."""
    run("plain", [300, 99, 8192], [70, 200, 8192], 4, 1, d, **mask)


@pytest.mark.parametrize("mask", [dict(), dict(causal=False), dict(window=40, sinks=1), dict(causal=False, window=9, sinks=40)])
def test_thousands_of_rows_key_by_key(mask):
    n = 250
    v = torch.zeros(n, 1, 256)
    v[torch.arange(n), :, torch.arange(n)] = 1.0
    x = Plain([n], 1, 256, v=v.to(DT["bf16"]).cuda())
    q = randn(16400, 2, 256, seed=3) / 4
    compare(x.attend(q, **mask), x, q, [16400], **mask)


@both
@types
@pytest.mark.parametrize("hq,hk", [(1, 1), (3, 3), (6, 2), (7, 1), (24, 8), (40, 2)])
def test_groups(kind, dtype, hq, hk):
    run(kind, [150], [3], hq, hk, 64, dtype)
    run(kind, [150], [41], hq, hk, 64, dtype, window=33, sinks=3)


@both
@pytest.mark.parametrize("nk", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 511, 513, 1025, 4099])
def test_lengths(kind, nk):
    run(kind, [nk], [1], 4, 2, 64)
    run(kind, [nk], [min(nk, 21)], 2, 2, 64, "f32")


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_sizes(block, dtype):
    run("cached", [1, 300, 127, 129, 64], [1, 7, 127, 2, 1], 4, 2, 80, dtype, block=block, window=100, sinks=5)


MASKS = [dict(), dict(causal=False), dict(window=1), dict(window=7), dict(window=40, sinks=1), dict(window=32, sinks=33),
         dict(window=50, sinks=200), dict(causal=False, window=1), dict(causal=False, window=20), dict(causal=False, window=9, sinks=40),
         dict(sinks=5), dict(window=2 ** 30, sinks=2 ** 30), dict(causal=False, window=2 ** 30)]


@both
@types
@pytest.mark.parametrize("mask", MASKS)
def test_masks_key_by_key(kind, dtype, mask):
    """Values that are one in a dim of their own: each output is the weight of a few keys, alone at its dim, so that no key
    is missing and none is there that should not be."""
    for lens, new in (([130, 64, 7], [130, 64, 7]), ([250, 33, 90], [1, 17, 9])):
        n = sum(lens)
        v = torch.zeros(n, 2, 256)
        place = torch.cat([torch.arange(m) for m in lens])
        v[torch.arange(n), :, place] = 1.0
        v = v.to(DT[dtype]).cuda()
        x = KINDS[kind](lens, 2, 256, dtype, v=v)
        q = randn(sum(new), 4, 256, dtype=dtype, seed=3) / 4
        compare(x.attend(q, q_start=starts(new), **mask), x, q, new, **mask)


@both
@types
@pytest.mark.parametrize("mask", [dict(), dict(causal=False), dict(window=700, sinks=4), dict(causal=False, window=900, sinks=70)])
def test_long_and_ragged(kind, dtype, mask):
    run(kind, [3000, 1, 777, 5000, 31], [1, 1, 1, 1, 1], 8, 2, 64, dtype, **mask)
    run(kind, [3000, 1, 777, 1500, 31], [3, 1, 300, 33, 31], 4, 2, 64, dtype, **mask)


@both
def test_many_sequences(kind):
    """More starts than a wave looks at together, and sequences without queries among them."""
    lens = [1 + (37 * i) % 90 for i in range(200)]
    new = [0 if i % 5 == 3 else 1 + i % min(m, 7) for i, m in enumerate(lens)]
    run(kind, lens, new, 4, 2, 32)


@pytest.mark.parametrize("n", [63, 64, 65, 4096, 4097, 6000])
def test_thousands_of_sequences(n):
    """Starts that a wave searches in one, two and three steps: each sequence's only key gives its value back."""
    new = [0 if i % 7 == 3 else 1 + i % 3 for i in range(n)]
    v = torch.arange(n, device="cuda").float()[:, None, None].expand(n, 1, 32).contiguous()
    q = torch.zeros(sum(new), 1, 32, device="cuda")
    got = incvit.attend(q, v, v, q_start=starts_of(new), k_start=starts_of([1] * n), causal=False)
    want = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(new, device="cuda")).float()
    assert torch.equal(got, want[:, None, None].expand_as(got))


@both
@types
def test_rows_that_see_nothing_are_zeros(kind, dtype):
    lens, new = [3, 0, 40], [10, 4, 2]  # more queries than keys: the first positions are negative
    for mask in (dict(), dict(causal=False, window=2), dict(causal=False)):
        x = KINDS[kind](lens, 1, 64, dtype)
        q = randn(16, 2, 64, dtype=dtype)
        got = x.attend(q, q_start=starts(new), **mask)
        compare(got, x, q, new, **mask)
        assert (got[10:14] == 0).all()
        if mask.get("causal", True):
            assert (got[:7] == 0).all() and (got[7:10] != 0).any()


@both
def test_rows_behind_the_last_sequence(kind):
    lens, new = [30, 20], [3, 5]
    x = KINDS[kind](lens, 2, 64)
    q = randn(200, 4, 64)
    out = torch.full_like(q, 7.0)
    assert x.attend(q, q_start=starts(new), out=out) is out
    compare(out, x, q, new)
    assert (out[8:] == 7).all()
    fresh = torch.empty_like(q).fill_(math.nan)  # what a new output finds in its memory
    del fresh
    got = x.attend(q, q_start=starts(new))
    assert torch.equal(got[:8], out[:8]) and (got[8:] == 0).all()


@both
@types
def test_what_masked_places_hold_does_not_count(kind, dtype):
    """Infinities, NaN and the type's largest values in keys and values that some rows of a tile do not see."""
    d, n = 64, 100
    k, v = randn(n, 1, d, dtype=dtype, seed=1), randn(n, 1, d, dtype=dtype, seed=2)
    q = randn(n, 2, d, dtype=dtype, seed=3)
    start = 64 if kind == "cached" else 70  # (a block of the cache is not finite as a whole)
    plain = KINDS[kind]([n], 1, d, dtype, k=k, v=v).attend(q)
    k2, v2 = k.clone(), v.clone()
    k2[start:, :, ::3] = math.inf
    k2[start + 1, 0, 5] = math.nan
    v2[start:, :, ::2] = math.nan
    v2[start + 2, 0, 1] = -math.inf
    v2[start + 5] = torch.finfo(v.dtype).max
    got = KINDS[kind]([n], 1, d, dtype, k=k2, v=v2).attend(q)
    assert torch.equal(got[:start], plain[:start])
    # whoever sees a NaN has one
    assert got[start:, :, ::2].isnan().all()
    # values alone: infinities reach the rows that see them and no other
    v3 = v.clone()
    v3[start + 3, 0, 7] = math.inf
    got = KINDS[kind]([n], 1, d, dtype, k=k, v=v3).attend(q)
    first = start if kind == "cached" else start + 3
    assert torch.equal(got[:first], plain[:first])
    assert not got[first:, :, 7].isfinite().any()
    if kind == "plain":
        assert (got[first:, :, 7] == math.inf).all()
        keep = [i for i in range(d) if i != 7]
        assert torch.equal(got[first:][..., keep], plain[first:][..., keep])


@both
@types
def test_queries_that_are_not_finite_stay_alone(kind, dtype):
    x = KINDS[kind]([90], 1, 64, dtype)
    q = randn(90, 2, 64, dtype=dtype)
    want = x.attend(q)
    q2 = q.clone()
    q2[40, 1, 3] = math.nan
    q2[50, 0, 9] = math.inf
    got = x.attend(q2)
    assert got[40, 1].isnan().all() and got[50, 0].isnan().all()
    keep = torch.ones(90, 2, dtype=torch.bool, device="cuda")
    keep[40, 1] = keep[50, 0] = False
    assert torch.equal(got[keep], want[keep])


@both
def test_scores_of_minus_infinity_alone(kind):
    """Keys are seen, but every score is -inf: 0 / 0, not the zeros of a row that sees nothing."""
    k = torch.full((40, 1, 64), 2.0 ** 127).bfloat16().cuda()
    x = KINDS[kind]([40], 1, 64, k=k)
    q = torch.full((1, 1, 64), -2.0 ** 120).bfloat16().cuda()
    assert x.attend(q).isnan().all()


@both
@types
def test_large_scores(kind, dtype):
    run(kind, [200], [30], 2, 1, 64, dtype, scale=30.0)
    run(kind, [2000], [1], 2, 1, 64, dtype, scale=1e-6)


@pytest.mark.parametrize("nq", [1, 5, 100])
@types
def test_scales_far_from_one(dtype, nq):
    """Blocks of keys and values of very different sizes, zeros among them: each weight keeps its place in the sum."""
    n, d = 200, 64
    k, v = randn(n, 1, d, dtype=dtype, seed=1), randn(n, 1, d, dtype=dtype, seed=2)
    sizes = torch.tensor([1.0, 1e-30, 1e30, 0.0, 1e-38, 3e-3], device="cuda")[torch.arange(n, device="cuda") // 16 % 6, None, None]
    k2 = (k.float() * sizes.clamp(max=3.0)).to(k.dtype)
    for x in (Cached([n], 1, d, dtype, k=k, v=(v.float() * sizes).to(v.dtype)), Cached([n], 1, d, dtype, k=k2, v=v)):
        q = randn(nq, 2, d, dtype=dtype, seed=3)
        compare(x.attend(q, causal=False), x, q, [nq], causal=False)
    # values without the huge ones: the others are not lost behind them
    sizes = sizes.clamp(max=1.0)
    x = Cached([n], 1, d, dtype, k=k, v=(v.float() * sizes).to(v.dtype))
    q = randn(nq, 2, d, dtype=dtype, seed=3)
    compare(x.attend(q, window=9), x, q, [nq], window=9)


@both
@types
def test_strides(kind, dtype):
    lens = [70, 40]
    n, hq, hk, d = sum(lens), 6, 2, 72
    x = randn(n, hq + 2 * hk, d, dtype=dtype)
    q, k, v = x.split([hq, hk, hk], dim=1)
    c = KINDS[kind](lens, hk, d, dtype, k=k, v=v)
    want = c.attend(q, q_start=starts(lens), causal=False)
    compare(want, c, q, lens, causal=False)
    heads_first = torch.full((hq, n, d + 8), 7.0, dtype=DT[dtype], device="cuda")
    c.attend(q.contiguous(), q_start=starts(lens), causal=False, out=heads_first[..., 8:].transpose(0, 1))
    assert torch.equal(heads_first[..., 8:].transpose(0, 1), want) and (heads_first[..., :8] == 7).all()


@both
@types
@pytest.mark.parametrize("new", [[1, 1], [40, 90]])
def test_the_output_may_be_the_queries(kind, dtype, new):
    x = KINDS[kind]([3000, 200], 2, 64, dtype)
    q = randn(sum(new), 4, 64, dtype=dtype)
    want = x.attend(q, q_start=starts(new))
    same = x.attend(q, q_start=starts(new), out=q)
    assert same is q and torch.equal(q, want)


@both
def test_keys_that_all_sequences_share(kind):
    """The same blocks in every row of the table; rows without a stride."""
    x = Cached([333], 2, 64)
    q = randn(4, 4, 64)
    if kind == "cached":
        got = x.cache.attend(q, x.table.expand(4, -1), x.lens.expand(4).contiguous())
        want, bound = kv_ref.attention(q, x.k[0], x.v[0], torch.ones(4, 333, dtype=torch.bool, device="cuda"))
    else:
        k = randn(1, 2, 64, seed=1).expand(100, -1, -1)
        q = randn(300, 4, 64)
        got = incvit.attend(q, k, k, causal=False)
        want, bound = kv_ref.attention(q, k, k, torch.ones(300, 100, dtype=torch.bool, device="cuda"))
    kv_ref.check(got, want, bound)


def test_a_cache_past_4_gib():
    """Blocks whose bytes, and whose scales' numbers, lie past 32 bits."""
    blocks, hk, d = 400000, 4, 128
    c = incvit.KVCache(blocks, hk, d)
    assert c.buf.numel() > 2 ** 32 + 2 ** 30
    k, v, n = randn(100, hk, d, seed=1), randn(100, hk, d, seed=2), 100
    table = torch.tensor([[blocks - 1, 3, blocks - 7, 262144, blocks - 2, 262143, 0]], dtype=torch.int32, device="cuda")
    slots = (table[0].long()[torch.arange(n, device="cuda") // 16] * 16 + torch.arange(n, device="cuda") % 16).int()
    c.write(k, v, slots, begin=True)
    small = Cached([n], hk, d, k=k, v=v)
    got = c.read(slots, dtype=torch.float32)
    for y, want in zip(got, (small.k[0], small.v[0])):
        assert torch.equal(y.double(), want.float().double())
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    for nq in (1, 30, 70):
        q = randn(nq, 8, d)
        assert torch.equal(c.attend(q, table, lens), small.attend(q))


def test_blocks_outside_the_pool_are_not_seen():
    lens, d = [100, 100], 64
    x = Cached(lens, 1, d)
    q = randn(2, 2, d)
    bad = x.table.clone()
    bad[0, 2], bad[0, 5] = -1, 10 ** 6
    see = kv_ref.visible(1, 100, device="cuda").clone()
    see[:, 32:48] = see[:, 80:96] = False
    got = x.cache.attend(q, bad, x.lens)
    want, bound = kv_ref.attention(q[:1], x.k[0], x.v[0], see)
    kv_ref.check(got[:1], want, bound)
    assert torch.equal(got[1:], x.attend(q)[1:])
    assert (x.cache.attend(q, torch.full_like(bad, -5), x.lens) == 0).all()
    # a table narrower than the lengths: what it names
    got = x.cache.attend(q, x.table[:, :3], x.lens, causal=False)
    want, bound = kv_ref.attention(q[:1], x.k[0][:48], x.v[0][:48], torch.ones(1, 48, dtype=torch.bool, device="cuda"))
    kv_ref.check(got[:1], want, bound)
    # columns of a wider table
    wide = torch.full((2, 20), 3, dtype=torch.int32, device="cuda")
    wide[:, 4:11] = x.table
    assert torch.equal(x.cache.attend(q, wide[:, 4:11], x.lens), x.attend(q))


@both
def test_the_hint_of_the_longest_does_not_change_what_is_seen(kind):
    for hint in (1, 100, 2500, 10 ** 6):
        run_hint(kind, hint)


def run_hint(kind, hint):
    lens, new = [2500, 1200], [1, 1]
    x = KINDS[kind](lens, 2, 64)
    q = randn(2, 4, 64, seed=3)
    compare(x.attend(q, max_len=hint), x, q, new)


@both
def test_malformed_starts_stay_inside(kind):
    """Starts that go back or beyond the rows: whatever is computed, nothing outside the output is written."""
    x = KINDS[kind]([40, 40, 40], 1, 64)
    q = randn(300, 1, 64)
    big = torch.full((900, 1, 64), 7.0, device="cuda").bfloat16()
    for s in ([0, 1000, 2000, 3000], [300, 200, 100, 0], [-50, -20, 4, 300], [0, 4, 2, 300], [0, 250, 0, 300], [2 ** 31 - 1] * 4):
        x.attend(q, q_start=torch.tensor(s, dtype=torch.int32, device="cuda"), out=big[300:600])
        assert (big[:300] == 7).all() and (big[600:] == 7).all()


@both
@types
def test_other_streams_and_captured_calls(kind, dtype):
    """A captured call with a split over workgroups, replayed with other lengths and values between the program's own work."""
    lens = [1500, 900]
    x = KINDS[kind](lens, 2, 64, dtype)
    q = randn(2, 4, 64, dtype=dtype)
    want = x.attend(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = x.attend(q)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    out = torch.empty_like(q)
    starts_q = torch.arange(3, dtype=torch.int32, device="cuda")
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    out2 = torch.empty_like(q)
    with torch.cuda.graph(g):
        x.attend(q, q_start=starts_q, out=out)
    with torch.cuda.graph(g2, pool=g.pool()):  # two graphs whose workspaces share memory
        x.attend(q, q_start=starts_q, causal=False, window=300, out=out2)
    for i in range(4):
        q.copy_(randn(2, 4, 64, dtype=dtype, seed=50 + i))
        if kind == "cached":
            x.lens.copy_(torch.tensor([1500 - 301 * i, 900 - 200 * i], dtype=torch.int32))
        g.replay()
        g2.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, x.attend(q, q_start=starts_q)), i
        assert torch.equal(out2, x.attend(q, q_start=starts_q, causal=False, window=300)), i


@both
def test_the_same_call_gives_the_same_bits(kind):
    x = KINDS[kind]([5000, 300, 2000], 2, 128)
    q = randn(3, 8, 128)
    want = x.attend(q)
    for _ in range(5):
        assert torch.equal(x.attend(q), want)


def test_no_rows_and_no_sequences():
    x = Cached([20], 1, 64)
    assert x.cache.attend(randn(1, 2, 64)[:0], x.table, x.lens).shape == (0, 2, 64)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = x.cache.attend(randn(4, 2, 64), x.table[:0], x.lens[:0], q_start=none)
    assert (got == 0).all()
    k = randn(5, 1, 64)
    assert (incvit.attend(randn(4, 2, 64), k[:0], k[:0]) == 0).all()
    assert (incvit.attend(randn(4, 2, 64), k, k, q_start=none, k_start=none) == 0).all()
