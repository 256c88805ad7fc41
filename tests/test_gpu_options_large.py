"""Encoders with every option at the row counts of 448x448 frames and batches of streams: the 8-bit down projection of the
large-row GEMM on each of its tiles (its residual in operand order, its rows' map and its write to the cache), and the norms
and rotation with two heads to a group.

* Queries' and keys' norms and rotation: the keys and values of every layer, from the library's own inputs of it, against the
  oracle within the bars of gpu_util.
* The 8-bit MLP: one call of all streams, on the large-row tiles, against a call for each stream, whose down projections take
  the few-row kernel: bit for bit, since integer sums are exact and everything else has one order (tuned to one form here).
  The few-row kernel is compared with the oracle in test_gpu_options.  (A bar against the oracle would say little here: H
  differs by roundings of bf16, 2^-8 of a value, and where the row's largest does, every integer is rounded anew: a step of
  max|x| / 127, which changes a product by 1% of its rms, and the worst of a million outputs by five times that.)

CASES says which kernels each takes; tests/test_op_forms.py holds the library to it on the CPU."""
import numpy as np
import pytest
import torch

from oracle import vit
from paper_2607_12287_amd import incvit, synth
from tests.gpu_util import TOL, Pair, rel_err

pytestmark = pytest.mark.gpu


def shape(dim, heads, mlp, side=96, dtype="bf16", **kw):
    kw = {**dict(rope="halves", qk_norm="layer", mlp_int8=True), **kw}
    return synth.ModelShape(side, side, 3, 6, dim, 2, heads, mlp, dtype, **kw)


# (name, model, streams, streams that the oracle follows, 8-bit down projection, norms and rotation); 256 tokens to a stream
# of 96 x 96
CASES = [
    ("one_448_frame", synth.ModelShape(448, 448, 3, 14, 1152, 2, 16, 4304, "bf16", rope="halves", qk_norm="rms", mlp_int8=True), 1, [0],
     "64,96,4,4,4", "bf16,4,16,2"),
    ("down_64x64", shape(1152, 16, 450), 3, [0, 2], "64,64,2,2,8", "bf16,4,16,2"),
    ("down_64x96", shape(1152, 16, 1210), 4, [1, 3], "64,96,4,4,4", "bf16,4,16,2"),
    ("down_64x128", shape(1024, 16, 4096), 8, [0, 7], "64,128,2,2,6", "bf16,8,4,2"),
    ("down_128x128", shape(1024, 8, 203), 10, [3, 9], "128,128,2,1,8", "bf16,8,8,2"),
    ("down_256x128", shape(1024, 16, 300, rope="adjacent", qk_norm="rms"), 17, [0, 16], "256,128,4,1,6", "bf16,8,4,2"),
    ("down_128x128_rounds", shape(1024, 16, 130), 33, [0, 32], "128,128,2,1,4", "bf16,8,4,2"),
    ("down_256x256", shape(2048, 16, 100), 32, [0, 31], "256,256,2,1,4", "bf16,8,8,2"),
    ("heads_of_24", shape(384, 16, 203), 9, [0, 8], None, "bf16,4,4,2"),
    ("heads_of_56", shape(448, 8, 203), 9, [8], None, "bf16,4,8,2"),
    ("f32_down_64x64", shape(1152, 16, 450, dtype="f32"), 3, [0], "64,64,2,2,8", "float,4,16,2"),
    ("f32_down_64x96", shape(1152, 16, 700, dtype="f32", qk_norm="rms"), 4, [0, 3], "64,96,4,4,4", "float,4,16,2"),
    ("f32_down_64x128", shape(1024, 32, 300, dtype="f32"), 8, [7], "64,128,2,2,6", "float,4,4,2"),
    ("f32_down_256x128", shape(1024, 16, 300, dtype="f32"), 17, [0, 16], "256,128,4,1,6", "float,4,8,2"),
]


def frames(m, views):
    return [np.stack([synth.random_patches(m, 60 + t, 1)[0] + np.float32(0.01 * v) for v in range(views)]) for t in range(2)]


@pytest.mark.parametrize("name,m,views,sample,down,qk", CASES, ids=[c[0] for c in CASES])
def test_keys_and_values_of_every_layer(name, m, views, sample, down, qk):
    """A full encode, then a step of all tokens but three of a stream: rows that fill no tile, whose tokens have gaps."""
    p = Pair(m, synth.make_weights(m, 51), views, oracle_views=sample, guard=512)
    x = frames(m, views)

    def check(rows_of, label):
        for v in sample:
            g, U = p.enc.export(p.caches[v]), rows_of(v)
            assert np.array_equal(g["X"][0][U], p.ora[v].X[0][U]), (label, v)
            for l in range(m.depth):
                K, V = g["K"][l].copy(), g["V"][l].copy()
                vit.attn_branch(p.model, l, g["X"][l][U], U, K, V)
                for what, a, b in (("K", g["K"][l][U], K[U]), ("V", g["V"][l][U], V[U])):
                    e = rel_err(a, b)
                    assert e <= TOL[m.dtype], (label, v, l, what, e)
        p.check_guards(label)

    p.full_encode(x[0])
    check(lambda v: np.arange(m.n_tokens), "full")
    idx, count, refreshed, res = p.step(x[1], float("inf"), [m.n_tokens - 3] * views)
    p.check_step(idx, count, refreshed, res, free_y=False)
    check(lambda v: res[v].idx, "step")
    p.enc.close()


@pytest.mark.parametrize("name,m,views,sample,down,qk", [c for c in CASES if c[2] > 1], ids=[c[0] for c in CASES if c[2] > 1])
def test_one_call_of_all_streams_has_the_bits_of_a_call_for_each(name, m, views, sample, down, qk):
    enc = incvit.Encoder(m, synth.flatten_weights(m, synth.make_weights(m, 51)), max_streams=views)
    assert incvit.incvit_set_tuning(enc.h, cols=(1, 1, 1, 1), attn_qtiles=1, attn_waves=4, row_groups=1, fc2_mode=1, tiled=1) == 0
    x = [torch.from_numpy(f).cuda() for f in frames(m, views)]
    buf_a, a = enc.new_caches(views)
    buf_b, b = enc.new_caches(views)
    caps = [m.n_tokens - 3] * views
    for t in range(2):
        if t == 0:
            enc.full_encode(x[t], a)
        else:
            enc.step(x[t], a, float("inf"), caps)
        for v in range(views):
            one = x[t][v:v + 1].contiguous()
            if t == 0:
                enc.full_encode(one, b[v:v + 1])
            else:
                enc.step(one, b[v:v + 1], float("inf"), caps[:1])
        torch.cuda.synchronize()
        for v in range(views):
            p, q = enc.export(a[v]), enc.export(b[v])
            for k in p:
                assert np.array_equal(p[k], q[k]), (t, v, k)
    del buf_a, buf_b
    enc.close()
