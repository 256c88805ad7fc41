"""Rotary tables on the GPU against 64-bit angles: positions given and packed grids, one to three axes, both ladders and
layouts, far and negative positions, windows, more grids than one launch takes, another stream, a captured call.

Tolerance: the reduced angle |x| <= pi/4 is rounded to fp32 (2^-25), each polynomial's last two operations round once more
(2 * 2^-24 of at most 1) and its truncation is below 2e-9: 4 * 2^-24 in all; the angle itself is formed from a rounded
frequency in 64 bits: three roundings of it, 2^-51 of the angle."""
import numpy as np
import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import ops_ref

pytestmark = pytest.mark.gpu


def check(got, ang):
    got = got.cpu().numpy().astype(np.float64)
    bound = 4 * 2.0 ** -24 + 2.0 ** -51 * np.abs(ang)
    assert got.shape == ang.shape + (2,)
    assert np.all(np.abs(got[..., 0] - np.cos(ang)) <= bound)
    assert np.all(np.abs(got[..., 1] - np.sin(ang)) <= bound)


@pytest.mark.parametrize("pairs,ladder,layout,theta,scale", [
    ((36,), "axis", "blocks", 10000.0, None),
    ((18, 18), "axis", "blocks", 100.0, None),
    ((16, 24, 24), "head", "blocks", 1e6, None),
    ((14, 13, 13), "head", "cycle", 10000.0, (0.5, 1.0, -2.0)),
    ((1, 5, 2), "axis", "cycle", 1.0, None),
    ((1,), "axis", "blocks", 10000.0, None),
    ((128,), "head", "blocks", 1e12, None),
])
@pytest.mark.parametrize("tokens,reach", [(1, 5), (257, 4096), (1000, 2 ** 31 - 1)])
def test_positions(pairs, ladder, layout, theta, scale, tokens, reach):
    rng = np.random.default_rng(tokens + len(pairs))
    pos = rng.integers(-reach, reach + 1, size=(len(pairs), tokens)).astype(np.int32)
    rope = incvit.make_rope(2 * sum(pairs), pairs, theta, ladder, layout, scale)
    got = incvit.rope_table(rope, positions=torch.from_numpy(pos).cuda())
    check(got, ops_ref.rope_angles(pos, pairs, theta, ladder, layout, scale))


def test_positions_of_a_view_and_none():
    pos = torch.arange(60, dtype=torch.int32, device="cuda").reshape(3, 20)
    rope = incvit.make_rope(64, (10, 11, 11))
    got = incvit.rope_table(rope, positions=pos[:, 3:16])
    check(got, ops_ref.rope_angles(pos[:, 3:16].cpu().numpy(), (10, 11, 11)))
    assert incvit.rope_table(rope, positions=pos[:, :0]).shape == (0, 32, 2)
    assert incvit.rope_table(rope, grids=[]).shape == (0, 32, 2)


@pytest.mark.parametrize("axes", [1, 2, 3])
@pytest.mark.parametrize("merge,grids", [
    (1, [(1, 16, 16)]),
    (1, [(1, 1, 1), (3, 5, 7, 100, 2, 9), (2, 1, 13, -4)]),
    (2, [(2, 4, 6, 7), (1, 2, 2), (1, 10, 2, 0, 3)]),
    (3, [(2, 9, 6, 1, 2, 3)]),
    (1, [(1 + i % 2, 1 + i % 3, 1 + i % 4, i, 2 * i, 3 * i) for i in range(71)]),
])
def test_grids(axes, merge, grids):
    pairs = {1: (20,), 2: (9, 11), 3: (4, 8, 8)}[axes]
    rope = incvit.make_rope(40, pairs, ladder="head")
    got = incvit.rope_table(rope, grids=grids, merge=merge)
    check(got, ops_ref.rope_angles(ops_ref.grid_positions(grids, merge, axes), pairs, ladder="head"))


def test_grid_equals_its_positions_bit_for_bit():
    grids = [(4, 6, 8, 9, 1, 2), (1, 14, 10)]
    rope = incvit.make_rope(128, (16, 24, 24), 1e6, "head")
    pos = torch.from_numpy(ops_ref.grid_positions(grids, 2, 3).astype(np.int32)).cuda()
    assert torch.equal(incvit.rope_table(rope, grids=grids, merge=2), incvit.rope_table(rope, positions=pos))


def test_only_the_tables_own_bytes_are_written():
    rope = incvit.make_rope(72, (18, 18))
    buf = torch.full((16 + 35 * 36 * 2 + 16,), 7.0, device="cuda")
    incvit.rope_table(rope, grids=[(1, 5, 7)], out=buf[16:-16].view(35, 36, 2))
    assert torch.all(buf[:16] == 7.0) and torch.all(buf[-16:] == 7.0)
    check(buf[16:-16].view(35, 36, 2), ops_ref.rope_angles(ops_ref.grid_positions([(1, 5, 7)], 1, 2), (18, 18)))


def test_another_stream_and_a_captured_call():
    rope = incvit.make_rope(64, (16, 16))
    pos = torch.randint(-500, 500, (2, 333), dtype=torch.int32, device="cuda")
    want = incvit.rope_table(rope, positions=pos)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = incvit.rope_table(rope, positions=pos)
    st.synchronize()
    assert torch.equal(got, want)
    out = torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        incvit.rope_table(rope, positions=pos, out=out)
    for seed in range(3):
        pos.copy_(torch.randint(-500, 500, pos.shape, generator=torch.Generator().manual_seed(seed)))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, incvit.rope_table(rope, positions=pos))
