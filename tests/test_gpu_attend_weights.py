"""What attention of few rows in bf16 does with its weights: over the cache they are two bf16 numbers, over given keys they are
rounded to one and summed as rounded.  Held to bounds without a rounding of the weights, which that of other forms would not keep."""
import math

import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import kv_ref
from tests.test_gpu_attend import Cached, Plain, randn

pytestmark = pytest.mark.gpu
D = 64


def inside(got, want, bound):
    """Whether bf16 results are roundings of values within the bound (a rounding keeps the order; from 64 bits it goes by way of
    fp32, which may move it by u)."""
    b = bound + 2 * kv_ref.U * (want.abs() + bound)
    return (got >= (want - b).bfloat16()) & (got <= (want + b).bfloat16())


def exactly(q, k, v, see):
    """The 64-bit result, the bound of fp32 arithmetic, and the sum of weights times magnitudes."""
    want, bound = kv_ref.attention(q.float(), k, v, see)
    return want, bound, kv_ref.attention(q.float(), k, v.abs(), see)[0]


@pytest.mark.parametrize("window", [0, 1])
def test_a_row_of_one_key_over_given_keys_is_its_value(window):
    for nk in (1,) if not window else (1, 37, 200):
        x = Plain([nk], 2, D)
        q = randn(1, 4, D, seed=3)
        assert torch.equal(x.attend(q, window=window)[0], x.va[nk - 1].repeat_interleave(2, 0))


def test_a_row_of_one_key_over_the_cache_is_its_value_rounded_once():
    """The scale times the weight goes in as two numbers of 8 bits each: within 2^-15."""
    apart = 0
    for nk in (1, 18, 200):
        x = Cached([nk], 2, D)
        q = randn(1, 4, D, seed=3)
        got = x.attend(q, window=1)[0]
        want = x.v[0][nk - 1].repeat_interleave(2, 0)
        assert inside(got, want, want.abs() * 2.0 ** -15).all()
        s = want.abs().amax(-1, keepdim=True) / 127  # near the scale, if not its bits
        apart += (~inside((want * (s.bfloat16().double() / s)).bfloat16(), want, want.abs() * 2.0 ** -15)).sum().item()
    assert apart > 0  # one number of 8 bits would be seen


@pytest.mark.parametrize("nk", [5, 60, 700])
@pytest.mark.parametrize("nq", [1, 4])
def test_few_rows_over_the_cache(nk, nq):
    x = Cached([nk], 2, D)
    q = randn(nq, 4, D, seed=3)
    see = kv_ref.visible(nq, nk, device="cuda")
    want, bound, size = exactly(q, x.k[0], x.v[0], see)
    assert inside(x.attend(q), want, bound + size * 2.0 ** -15).all()


def test_a_key_that_carries_a_row_over_given_keys():
    """The maximum follows the scores by steps of 2^8 only: the second key's weight lies between 1 and 2^8 and is rounded; with
    weights w_i = p_i (1 + e_i), |e_i| <= 2^-8, and a sum of the same, the result is off by at most sum p_i |e_i| |v_i - o|."""
    nk, far = 200, 150  # tiles of 32 keys: the first and the fifth, which one wave takes
    k, v = torch.zeros(nk, 1, D), torch.zeros(nk, 1, D)
    k[far, 0, 0] = 1.0
    v[far] = torch.randn(1, D, generator=torch.Generator().manual_seed(5))
    k[1:far] = k[far + 1:] = 0
    k[:, 0, 1] = -64.0
    k[0, 0, 1] = k[far, 0, 1] = 0.0
    x = Plain([nk], 1, D, k=k.bfloat16().cuda(), v=v.bfloat16().cuda())
    apart = 0
    for step in range(40):
        q = torch.zeros(1, 1, D)
        q[..., 0], q[..., 1] = 8.0 * (3.0 + step / 20), 64.0  # scores 0, 3 to 5, and -512 for the others
        q = q.bfloat16().cuda()
        see = kv_ref.visible(1, nk, device="cuda")
        want, bound, _ = exactly(q, x.k[0], x.v[0], see)
        w = torch.exp(q[0, 0, 0].double() / 8)
        p = w / (1 + w)
        off = 2.0 ** -8 / (1 - 2.0 ** -8) * (p * (x.v[0][far].double() - want[0]).abs() + (1 - p) * want[0].abs())
        assert inside(x.attend(q)[0], want[0], bound[0] + off).all()
        apart += (~inside((want[0] * (w.bfloat16().double() / w)).bfloat16(), want[0], bound[0] + off)).sum().item()
    assert apart > 0  # a sum of the weights as they were would be seen
