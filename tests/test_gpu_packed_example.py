"""The example's packed cache: its steps agree with attention over the numbers that its rows stand for."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("bits", [4, 8])
def test_serving_from_a_packed_cache(bits):
    import attention_within_a_limit as example
    out, held, full, packed, plain = example.serve_packed(bits, lengths=(300, 1, 64), slots=310)
    assert out.shape == held.shape == full.shape and torch.isfinite(out.float()).all()
    assert packed * 256 == plain * {4: 80, 8: 144}[bits]
    # two ways of rounding: a probability by 2^-8 of itself, and the result, on either side
    assert (out.float() - held.float()).abs().max() <= 4 * 2.0 ** -8 * max(1.0, float(held.float().abs().max()))
