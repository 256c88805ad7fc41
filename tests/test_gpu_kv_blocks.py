"""Rows written into the cache in 8 bits as workgroups take them: padding between the rows of a block.  Bit for bit, as in
test_gpu_kv."""
import random

import pytest
import torch

from tests.test_gpu_kv import Pair, rows_of

pytestmark = pytest.mark.gpu
blocks_of = pytest.mark.parametrize("block", [16, 32, 64, 128])


def write(p, slots, heads, d, dtype="bf16", seed=0, size=1.0, begin=False):
    n = len(slots)
    p.write(rows_of(n, heads, d, dtype, seed, size), rows_of(n, heads, d, dtype, seed + 1, size), slots, begin)


@blocks_of
@pytest.mark.parametrize("heads", [1, 8, 32])  # 512, 4096 and 16384 items: a workgroup's rows are 1 and 4
def test_frames_whose_other_tokens_are_padding(block, heads):
    """A call of one size for every frame: a row for each token, and no slot for those that stay."""
    p = Pair(256 // block, heads, 40, block)
    write(p, list(range(256)), heads, 40, begin=True)
    pick = random.Random(block + heads)
    for i, share in enumerate((0.7, 0.3, 0.05, 0.01, 0.0)):
        slots = [t if pick.random() < share else pick.choice([-1, -9, 256, 2 ** 31 - 1, -2 ** 31]) for t in range(256)]
        write(p, slots, heads, 40, seed=10 + i, size=0.5 + 0.4 * i)
        p.check()


@blocks_of
@pytest.mark.parametrize("heads", [1, 2, 6])  # 1 (4 for the longest), 4 and 16 or 32 rows of a workgroup
@pytest.mark.parametrize("gap", [62, 63, 64, 65, 511, 512, 513, 577, 1200])
def test_long_padding_between_the_rows_of_a_block(block, heads, gap):
    p = Pair(4, heads, 32, block)
    write(p, list(range(4 * block)), heads, 32, begin=True)
    # two rows of a block, one and two of the next, with padding before, between and behind; then a block's second half
    valid = [5, 3, block + 1, 2 * block + 7, 2 * block + 7, 3 * block + 15]
    slots = [-1] * (gap // 2)
    for s in valid:
        slots += [s] + [-1] * gap
    n = 3600 if heads == 1 else 5000
    slots += [-1] * max(0, n - len(slots))
    write(p, slots, heads, 32, seed=3, size=2.0)
    p.check()
    write(p, [-1] * n + [block], heads, 32, seed=5, size=3.0)  # behind padding alone
    write(p, [-1] * n, heads, 32, seed=7, size=3.0)
    p.check()


@blocks_of
@pytest.mark.parametrize("dtype,heads,n", [("bf16", 4, 1500), ("f32", 3, 6000)])  # 12000 and 36000 items: 4 and 16 or 32 rows
def test_workgroups_that_take_several_blocks(block, dtype, heads, n):
    """Prompts through shuffled blocks, from the middle of one to the middle of one, then rows here and there: groups of a block
    with new rows and without, under a scale that stays and one that grows."""
    need = -(-n // block) + 2
    order = torch.randperm(need, generator=torch.Generator().manual_seed(n)).tolist()
    p = Pair(need, heads, 40, block)
    slots = [order[t // block] * block + t % block for t in range(block // 2 + 3, block // 2 + 3 + n)]
    write(p, slots, heads, 40, dtype, begin=True)
    p.check()
    pick = random.Random(block)
    for seed, (share, size) in enumerate(((0.9, 0.3), (0.9, 2.0))):
        write(p, [s for s in slots if pick.random() < share], heads, 40, dtype, 10 + 2 * seed, size)
        p.check()
    write(p, [-1 if (s // 16) % 3 else s for s in slots], heads, 40, dtype, 20, 3.0)  # two groups of three without new rows
    p.check(dtype)


@blocks_of
@pytest.mark.parametrize("heads,n", [(12, 400), (24, 700)])  # 9600 and 33600 items
def test_a_token_of_each_of_many_sequences(block, heads, n):
    """Every row begins a block's run: a workgroup takes as many blocks as it has rows."""
    p = Pair(n, heads, 8, block)
    for i in range(3):
        write(p, [b * block + (7 * b + i) % block for b in range(n)], heads, 8, "bf16", 2 * i, 1.0 + i, begin=i == 1)
    p.check()
