"""Attention over given keys and values where a form of the kernels is at its limits: the smallest heads with values that are not
finite.  The bound is derived in kv_ref.attention."""
import math

import pytest
import torch

from paper_2607_12287_amd import incvit
from tests import kv_ref
from tests.test_gpu_attend import DT, randn, types

pytestmark = pytest.mark.gpu


@types
@pytest.mark.parametrize("d", [8, 16, 24, 40, 72, 256])
@pytest.mark.parametrize("rows", [5, 100])  # waves with keys, and with rows
def test_values_that_are_not_finite_in_the_last_head(d, dtype, rows):
    """The last key's, of the last head: the tensors end there."""
    n = 100
    q, k, v = (randn(m, h, d, dtype=dtype, seed=s) for m, h, s in ((rows, 4, 3), (n, 2, 1), (n, 2, 2)))
    want = incvit.attend(q, k, v)
    see = kv_ref.visible(rows, n, device="cuda")
    kv_ref.check(want, *kv_ref.attention(q, k, v, see))
    v2 = v.clone()
    v2[n - 1, 1, ::3] = -math.inf
    v2[n - 2, 1, d - 1] = math.nan
    got = incvit.attend(q, k, v2)
    assert torch.equal(got[:-2], want[:-2]) and torch.equal(got[:, :2], want[:, :2])  # who does not see them
    assert (got[-1, 2:, 0:d - 1:3] == -math.inf).all() and got[-2:, 2:, d - 1].isnan().all()
    keep = [i for i in range(d - 1) if i % 3]
    assert torch.equal(got[..., keep], want[..., keep]) and torch.equal(got[-2, :, :d - 1], want[-2, :, :d - 1])
