"""The cache of keys and values in 8 bits on the GPU: what is written and read back, bit for bit.  Scales, integers and values are
roundings that the definition names, so the plain statement gives the same bits and nothing is tolerated."""
import math

import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import kv_ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows_of(n, heads, d, dtype, seed=0, size=1.0):
    g = torch.Generator().manual_seed(1000 * seed + 31 * n + d)
    x = torch.randn(n, heads, d, generator=g) * (torch.rand(n, 1, 1, generator=g) + 0.2) * size
    return x.to(DT[dtype])


class Pair:
    """The library's cache and the plain one, written alike."""

    def __init__(self, blocks, heads, d, block):
        self.cache = incvit.KVCache(blocks, heads, d, block=block)
        self.k, self.v = kv_ref.Held(blocks, heads, d, block), kv_ref.Held(blocks, heads, d, block)
        self.slots = blocks * block

    def write(self, k, v, slots, begin=False):
        self.cache.write(k.cuda(), v.cuda(), torch.tensor(slots, dtype=torch.int32, device="cuda"), begin=begin)
        self.k.write(k, slots, begin)
        self.v.write(v, slots, begin)

    def check(self, dtype="f32"):
        at = torch.arange(self.slots, dtype=torch.int32, device="cuda")
        for got, want in zip(self.cache.read(at, dtype=DT[dtype]), (self.k, self.v)):
            assert torch.equal(got.cpu().double().nan_to_num(nan=12345.0), want.values(DT[dtype]).double().nan_to_num(nan=12345.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 32, 40, 64, 72, 80, 96, 104, 128, 136, 192, 200, 256])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_prompts(dtype, d, block):
    p = Pair(5, 2, d, block)
    n = 2 * block + block // 2 + 3
    table = [3, 0, 4]
    slots = [table[t // block] * block + t % block for t in range(n)]
    p.write(rows_of(n, 2, d, dtype), rows_of(n, 2, d, dtype, 1), slots, True)
    p.check()
    p.check("bf16")
    # token by token on, in ever larger ones and smaller ones, then a sequence that takes a used block
    for i in range(4):
        t = n + i
        p.write(rows_of(1, 2, d, dtype, 2 + i, 2.0 ** (i - 1)), rows_of(1, 2, d, dtype, 9 + i, 0.5), [table[t // block] * block + t % block], True)
    p.check()
    p.write(rows_of(3, 2, d, dtype, 20), rows_of(3, 2, d, dtype, 21), [0, 1, 2], True)
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 64])
def test_refreshed_rows_leave_the_others(dtype, block):
    p = Pair(256 // block, 3, 72, block)
    p.write(rows_of(256, 3, 72, dtype), rows_of(256, 3, 72, dtype, 1), list(range(256)))
    for seed, step in enumerate((11, 7, 1)):  # few to a block, several, all of them: nothing is kept then
        at = list(range(seed, 256, step))
        p.write(rows_of(len(at), 3, 72, dtype, 5 + seed, 0.6 + 0.5 * seed), rows_of(len(at), 3, 72, dtype, 8 + seed, 1.5 - seed / 2), at)
        p.check()


def test_padding_and_repeated_slots():
    p = Pair(4, 2, 64, 16)
    p.write(rows_of(40, 2, 64, "bf16"), rows_of(40, 2, 64, "bf16", 1), list(range(40)))
    # of the rows of one slot the last stays, also behind the 64 that a wave looks at together
    slots = [-1, 17, 18, 17, -7, 33, 63, 64, 2 ** 31 - 1, 5] + [6] * 70 + [7, 6]
    n = len(slots)
    p.write(rows_of(n, 2, 64, "bf16", 3), rows_of(n, 2, 64, "bf16", 4), slots)
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_zeros_infinities_and_tiny_values(dtype):
    p = Pair(8, 1, 32, 16)
    k, v = rows_of(128, 1, 32, dtype), rows_of(128, 1, 32, dtype, 1)
    k[0:16] = 0
    k[20, 0, 3] = math.inf
    v[37, 0, 31] = math.nan
    v[50, 0, 0] = -math.inf
    k[64:80] *= 1e-38
    v[64:80] = 1e-44
    k[80:96] = torch.finfo(k.dtype).max
    k[96:112] *= 1e30
    k[97] *= 1e-60
    slots = list(range(128))
    p.write(k, v, slots, True)
    p.check()
    # one token of a block that is not finite does not mend it; the block begun anew is sound
    p.write(rows_of(2, 1, 32, dtype, 5), rows_of(2, 1, 32, dtype, 6), [20, 37])
    p.check()
    p.write(rows_of(16, 1, 32, dtype, 7), rows_of(16, 1, 32, dtype, 8), list(range(16, 32)))
    p.write(rows_of(1, 1, 32, dtype, 7), rows_of(1, 1, 32, dtype, 8), [32], True)
    p.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    """Views of a projection's output in, views of a wider tensor out; what lies between stays."""
    n, h, d = 50, 4, 40
    x = rows_of(n, 3 * h, d, dtype).cuda()
    c, want = incvit.KVCache(4, h, d), [kv_ref.Held(4, h, d) for _ in range(2)]
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    c.write(x[:, h:2 * h], x[:, 2 * h:], slots)
    for w, y in zip(want, (x[:, h:2 * h], x[:, 2 * h:])):
        w.write(y, range(n))
    heads_first = torch.full((2, h, n, d), 7.0, dtype=DT[dtype], device="cuda")
    c.read(slots, k_out=heads_first[0].transpose(0, 1), v_out=heads_first[1].transpose(0, 1))
    wide = torch.full((n + 1, 2 * h + 1, d + 8), 7.0, dtype=DT[dtype], device="cuda")
    c.read(slots, k_out=wide[1:, 1:h + 1, 8:], v_out=wide[1:, h + 1:, 8:])
    for i in range(2):
        v = want[i].values(DT[dtype])[:n].cuda()
        assert torch.equal(heads_first[i].transpose(0, 1), v)
        assert torch.equal(wide[1:, 1 + i * h:1 + (i + 1) * h, 8:], v)
    assert (wide[0] == 7).all() and (wide[:, 0] == 7).all() and (wide[..., :8] == 7).all()


def test_reads_of_padding_leave_the_rows():
    c = incvit.KVCache(2, 1, 64)
    x = rows_of(32, 1, 64, "f32").cuda()
    c.write(x, 2 * x, torch.arange(32, dtype=torch.int32, device="cuda"))
    at = torch.tensor([-1, 3, 32, 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    k, v = torch.full((2, 6, 1, 64), 5.0, device="cuda").unbind(0)
    c.read(at, k_out=k, v_out=v)
    assert (k[[0, 2, 4, 5]] == 5).all() and torch.equal(k[1], k[3]) and torch.equal(v[1], 2 * k[1])
    k, v = c.read(at, dtype=torch.float32)
    assert (k[[0, 2, 4, 5]] == 0).all() and (v[[0, 2, 4, 5]] == 0).all() and (k[1] != 0).any()
    k, v = c.read(at[:0])
    assert k.shape == (0, 1, 64)
    c.write(x[:0], x[:0], at[:0])


def test_many_rows_and_heads():
    """As many rows as a prompt has, in a pool whose blocks are dealt out in any order."""
    n, h, d = 5000, 12, 80
    g = torch.Generator().manual_seed(3)
    order = torch.randperm(400, generator=g)[:-(-n // 16)]
    slots = (order[torch.arange(n) // 16] * 16 + torch.arange(n) % 16).int()
    x = torch.randn(2, n, h, d, generator=g).bfloat16()
    p = Pair(400, h, d, 16)
    p.write(x[0], x[1], slots.tolist(), True)
    p.check("bf16")


def test_other_streams_and_captured_calls():
    c = incvit.KVCache(8, 2, 64)
    x = rows_of(1, 2, 64, "bf16").cuda()
    k, v, slot = x.clone(), x.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    at = torch.arange(128, dtype=torch.int32, device="cuda")
    ko, vo = torch.zeros(2, 128, 2, 64, dtype=torch.bfloat16, device="cuda").unbind(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.write(k, v, slot)
        c.read(at, k_out=ko, v_out=vo)
    torch.cuda.current_stream().wait_stream(side)
    want = [kv_ref.Held(8, 2, 64) for _ in range(2)]
    for w in want:
        w.write(x, [0])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.write(k, v, slot)
        c.read(at, k_out=ko, v_out=vo)
    for i in range(1, 40):
        y = rows_of(1, 2, 64, "bf16", i, 1 + i / 10)
        k.copy_(y)
        v.copy_(-2 * y)
        slot.fill_(i)
        g.replay()
        (k @ k.transpose(1, 2)).sum()  # the program's own work between the replays
        torch.cuda.synchronize()
        want[0].write(y, [i])
        want[1].write(-2 * y, [i])
        assert torch.equal(ko.cpu(), want[0].values(torch.bfloat16)) and torch.equal(vo.cpu(), want[1].values(torch.bfloat16)), i
