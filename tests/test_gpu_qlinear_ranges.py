"""8-bit products of sizes past 32 bits are refused, not taken for their low half."""
import pytest
import torch

from paper_2607_12287_amd import incvit

pytestmark = pytest.mark.gpu
LONG = 2 ** 32 + 64


def test_weights_past_32_bits():
    one = torch.ones(1, 1, device="cuda")
    for shape in ((LONG, 1), (64, LONG), (65537, 1)):
        with pytest.raises(incvit.IncvitError, match="UNSUPPORTED"):
            incvit.QLinear(one.expand(*shape))


def test_rows_past_32_bits():
    x = torch.zeros(1, LONG, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(incvit.IncvitError, match="UNSUPPORTED"):
        incvit.quantize_rows(x)
    with pytest.raises(incvit.IncvitError, match="UNSUPPORTED"):
        incvit.quantize_rows(x[:, :65537])
