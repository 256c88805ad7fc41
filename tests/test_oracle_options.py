"""The oracle's rotation, head norms and 8-bit MLP against statements of their own, and what they must leave as it is."""
import numpy as np
import pytest

from oracle import vit
from paper_2607_12287_amd import synth
from tests import ops_ref

OPTIONS = [dict(rope="halves"), dict(rope="adjacent", rope_theta=100.0), dict(qk_norm="rms"), dict(qk_norm="layer", rope="halves"),
           dict(mlp_int8=True), dict(rope="adjacent", qk_norm="rms", mlp_int8=True)]


@pytest.mark.parametrize("norm", [None, "rms", "layer"])
@pytest.mark.parametrize("rope", [None, "halves", "adjacent"])
def test_head_norm_rotate(norm, rope):
    rng = np.random.default_rng(3)
    heads, dh, gw, tok = 3, 24, 5, np.array([0, 4, 7, 19])
    x = rng.standard_normal((4, heads * dh)) + 2.0
    g, b = rng.standard_normal(dh), rng.standard_normal(dh)
    got = vit.head_norm_rotate(x, heads, norm, g, b, 1e-6, rope, 50.0, tok, gw)
    n, _, _ = ops_ref.head_norm(x.reshape(4, heads, dh), g, b if norm == "layer" else None, norm, 1e-6)
    if rope:
        ang = ops_ref.rope_angles(np.stack([tok // gw, tok % gw]), (dh // 4, dh // 4), 50.0)
        n = ops_ref.rotate(n, np.cos(ang), np.sin(ang), rope)
    assert np.allclose(got, n.reshape(4, -1), rtol=1e-13, atol=1e-13)


def test_scores_depend_on_offsets_alone():
    """Rotated queries and keys at (y, x) and (y', x') meet as they do anywhere else with the same offset."""
    rng = np.random.default_rng(4)
    q, k = rng.standard_normal((1, 32)), rng.standard_normal((1, 32))
    turn = lambda v, t: vit.head_norm_rotate(v, 1, None, None, None, 0.0, "halves", 100.0, np.array([t]), 10)  # noqa: E731
    one = turn(q, 23) @ turn(k, 45).T
    two = turn(q, 34) @ turn(k, 56).T   # both one row and one column further
    assert abs((one - two).item()) < 1e-12 and abs((one - q @ k.T).item()) > 1e-3


def test_linear_int8():
    rng = np.random.default_rng(5)
    x, w, b = rng.standard_normal((7, 90)), rng.standard_normal((90, 11)), rng.standard_normal(11)
    x[2] = 0.0
    xq, xs = ops_ref.quantized(x, 1)
    wq, ws = ops_ref.quantized(w, 0)
    assert np.allclose(vit.linear_int8(x, w, b), (xq * xs) @ (wq * ws) + b, rtol=1e-13, atol=1e-13)
    exact = x @ w + b
    assert np.abs(vit.linear_int8(x, w, b) - exact).max() < 0.02 * np.abs(exact).max()


def test_no_option_changes_nothing():
    m = synth.small_model(dtype="bf16")
    assert [n for n, _ in synth.param_shapes(m)] == [n for n, _ in synth.param_shapes(synth.small_model(dtype="bf16", mlp_int8=True,
                                                                                                       rope="halves"))]
    w = synth.make_weights(m, 1)
    p = synth.random_patches(m, 2)[0]
    plain = vit.full_encode(vit.Model(m, w), p).Y
    for o in OPTIONS:
        mo = synth.small_model(dtype="bf16", **o)
        y = vit.full_encode(vit.Model(mo, {**synth.make_weights(mo, 1), **w}), p).Y
        assert not np.array_equal(y, plain), o


@pytest.mark.parametrize("options", OPTIONS)
@pytest.mark.parametrize("mlp", ["reuse", "all"])
def test_invariants_hold(options, mlp):
    """Refreshing every token equals a full encode bit for bit; the same frame again selects nothing; only refreshed rows'
    keys change."""
    m = synth.small_model(dtype="bf16", **options)
    model = vit.Model(m, synth.make_weights(m, 6), mlp=mlp)
    a, b = synth.random_patches(m, 7)[0], synth.random_patches(m, 8)[0]
    cache = vit.full_encode(model, a)
    before = cache.copy()
    assert vit.step(model, a, cache, 0.98, m.n_tokens).count == 0
    assert np.array_equal(cache.K, before.K) and np.array_equal(cache.Y, before.Y)
    res = vit.step(model, b, cache, float("inf"), 5)
    rest = np.setdiff1d(np.arange(m.n_tokens), res.idx)
    assert np.array_equal(cache.K[:, rest], before.K[:, rest]) and not np.array_equal(cache.K, before.K)
    vit.step(model, b, cache, float("inf"), m.n_tokens)
    full = vit.full_encode(model, b)
    assert np.array_equal(cache.Y, full.Y) and np.array_equal(cache.K, full.K)
