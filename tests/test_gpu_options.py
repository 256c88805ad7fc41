"""Encoders with rotated queries and keys, head norms and an 8-bit MLP on the GPU against the oracle: full encodes and steps
layer by layer, with every other mode of the encoder, and what the options must leave as it is."""
import numpy as np
import pytest
import torch

from oracle import vit
from paper_2607_12287_amd import incvit, synth
from tests.gpu_util import Pair, rel_err

pytestmark = pytest.mark.gpu

ALL = dict(rope="halves", qk_norm="layer", mlp_int8=True)


def run_steps(m, seed, views=2, frames=3, tau=0.98, caps=None, row_groups=0, **kw):
    w = synth.make_weights(m, seed)
    p = Pair(m, w, views, guard=512, **kw)
    if row_groups:
        assert incvit.incvit_set_tuning(p.enc.h, row_groups=row_groups) == 0
    streams = [synth.RefillRectStream(m, seed + 1, v, m.img_h // 2, m.img_w // 3) for v in range(views)]
    its = [s.frames(frames) for s in streams]
    worst, rows = 0.0, 0
    for t in range(frames):
        batch = np.stack([synth.patchify(next(i), m.patch) for i in its])
        if t == 0:
            p.full_encode(batch)
            worst = max(worst, p.check_layers(label="full"))
        else:
            idx, count, refreshed, res = p.step(batch, tau, caps or [m.n_tokens] * views)
            p.check_step(idx, count, refreshed, res, free_y=False)
            worst = max(worst, p.check_layers(lambda v: res[v].idx, label=f"step {t}"))
            rows += int(count.sum())
        p.check_guards()
    assert rows > 0 or tau < 0
    return worst


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("options", [dict(rope="halves"), dict(rope="adjacent", rope_theta=100.0), dict(qk_norm="rms"),
                                     dict(qk_norm="layer"), dict(rope="halves", qk_norm="rms"), dict(mlp_int8=True), ALL])
def test_each_option(dtype, options):
    run_steps(synth.small_model(dim=96, depth=2, heads=3, mlp=100, img=48, patch=8, dtype=dtype, **options), 31)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,heads", [(64, 8), (72 * 4, 4), (80 * 2, 2), (96 * 2, 2), (128, 1), (32, 2)])
def test_head_sizes(dtype, dim, heads):
    m = synth.ModelShape(30, 42, 3, 6, dim, 2, heads, 52, dtype, rope="adjacent", qk_norm="layer")
    run_steps(m, 32)


@pytest.mark.parametrize("kw", [dict(score="key"), dict(mlp="all"), dict(tau=float("inf"), caps=[7, 0]), dict(tau=-2.0),
                                dict(row_groups=8), dict(mlp="all", tau=-2.0)])
def test_with_the_other_modes(kw):
    run_steps(synth.small_model(dim=96, depth=2, heads=3, mlp=130, img=48, patch=6, dtype="bf16", **ALL), 33, **kw)


@pytest.mark.parametrize("mlp", ["reuse", "all"])
def test_large_calls(mlp):
    """Rows enough for the large-row products: 4 streams of 168 tokens, an odd MLP width."""
    m = synth.ModelShape(84, 98, 3, 7, 288, 2, 4, 603, "bf16", rope="halves", qk_norm="rms", mlp_int8=True)
    run_steps(m, 34, views=4, frames=2, mlp=mlp)


def test_headline_widths():
    m = synth.ModelShape(224, 224, 3, 14, 1152, 2, 16, 4304, "bf16", **ALL)
    run_steps(m, 35, views=1, frames=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_full_refresh_equals_a_full_encode_bit_for_bit(dtype):
    m = synth.small_model(dim=96, depth=2, heads=3, mlp=100, img=96, patch=6, dtype=dtype, **ALL)
    enc = incvit.Encoder(m, synth.flatten_weights(m, synth.make_weights(m, 36)))
    a, b = (torch.from_numpy(synth.random_patches(m, s)).cuda() for s in (1, 2))
    buf_one, one = enc.new_caches(1)  # the buffers live as long as their caches
    buf_two, two = enc.new_caches(1)
    enc.full_encode(a, one)
    enc.step(b, one, float("inf"), [m.n_tokens])
    enc.full_encode(b, two)
    x, y = enc.export(one[0]), enc.export(two[0])
    for k in ("K", "V", "Y"):
        assert np.array_equal(x[k], y[k]), k
    del buf_one, buf_two
    enc.close()


def test_captured_step_and_noalloc_and_schedule():
    m = synth.small_model(dim=96, depth=2, heads=3, mlp=100, img=48, patch=8, dtype="bf16", **ALL)
    enc = incvit.Encoder(m, synth.flatten_weights(m, synth.make_weights(m, 37)))
    frames = [torch.from_numpy(synth.random_patches(m, s)).cuda() for s in range(4)]
    bufs = [enc.new_caches(1) for _ in range(2)]
    out = [(torch.zeros(1, m.n_tokens, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
            torch.zeros(1, m.n_tokens, m.dim, dtype=torch.bfloat16, device="cuda")) for _ in range(2)]
    for _, c in bufs:
        enc.full_encode(frames[0], c)
    x = frames[0].clone()
    g = enc.step_graph(x, bufs[0][1], float("inf"), [9], out[0])
    for f in frames[1:]:
        x.copy_(f)
        enc.launch(g)
        enc.step(f, bufs[1][1], float("inf"), [9], out=out[1])
        torch.cuda.synchronize()
        for u, v in zip(*out):
            assert torch.equal(u, v)
    enc.drop_graph(g)
    torch.cuda.synchronize()
    idx, count, ref = out[0]
    assert incvit.incvit_step_noalloc(enc.h, 1, frames[0].data_ptr(), bufs[0][1], float("inf"), [9], idx.data_ptr(),
                                      count.data_ptr(), ref.data_ptr(), enc.stream_ptr()) == 0
    enc.step(frames[0], bufs[1][1], float("inf"), [9], out=out[1])
    torch.cuda.synchronize()
    assert torch.equal(ref[0, :9], out[1][2][0, :9])
    enc.encode_frame(frames[2], bufs[1][1], 4, 2, 0.98, [9], out=out[1])
    model = vit.Model(m, synth.make_weights(m, 37))
    assert rel_err(out[1][2][0].float().cpu().numpy(), vit.full_encode(model, frames[2][0].cpu().numpy()).Y) <= 5e-2
    enc.close()


def test_profile_names_the_kernels():
    m = synth.small_model(dim=96, depth=3, heads=3, mlp=100, img=48, patch=8, dtype="bf16", **ALL)
    enc = incvit.Encoder(m, synth.flatten_weights(m, synth.make_weights(m, 38)))
    _, c = enc.new_caches(1)
    incvit.incvit_profile_enable(enc.h, True)
    enc.full_encode(torch.from_numpy(synth.random_patches(m, 1)).cuda(), c)
    got = incvit.incvit_profile_read(enc.h)
    assert got["qk_norm"][1] == 3 and got["quant"][1] == 6 and got["fc1"][1] == 3 and got["fc2"][1] == 3
    enc.close()


def test_caches_of_other_options_are_not_read():
    base = dict(dim=96, depth=1, heads=3, mlp=100, img=48, patch=8, dtype="bf16")
    shapes = [synth.small_model(**base)] + [synth.small_model(**base, **o) for o in
              (dict(rope="halves"), dict(rope="halves", rope_theta=100.0), dict(rope="adjacent"), dict(qk_norm="rms"), dict(mlp_int8=True))]
    encs = [incvit.Encoder(m, synth.flatten_weights(m, synth.make_weights(m, 39))) for m in shapes]
    x = torch.from_numpy(synth.random_patches(shapes[0], 1)).cuda()
    for i, e in enumerate(encs):
        _, c = e.new_caches(1)
        e.full_encode(x, c)
        for j, other in enumerate(encs):
            assert (other.status(c[0]) == incvit.INCVIT_OK) == (i == j)
    for e in encs:
        e.close()


def test_more_rows_than_expected():
    """A step told to expect 256 rows refreshes 800: the MLP's workgroups take several of the tiles chosen for 256 (64 x 96)."""
    m = synth.ModelShape(120, 120, 3, 6, 640, 1, 8, 4352, "bf16", mlp_int8=True)
    run_steps(m, 41, views=2, frames=2, tau=2.0, row_groups=8)
