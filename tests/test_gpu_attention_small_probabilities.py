"""binary16 probabilities far below their row's largest: what many of them come to together is in the output.

One key is ahead of all others, which have 2^-25.5 of its probability each, w in sum.  Its values are 0 and theirs are 1, so the
output is w / (1 + w).  Probabilities are rounded in units of at most 2^-31 of the largest, to within 2^-32 or 2^-6.5 of each;
all equal, they may all be off to one side.  Sums in 32 bits of n / 16 and n / 32 additions are off by up to 2^-24 of
themselves with each; the result is rounded once (it is in the type's normal range)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


# rows and query heads of one key head: keys in parts; four, two and one wave to a row's keys; tiles of 32 keys
@pytest.mark.parametrize("rows,heads", [(1, 2), (9000, 1), (1100, 16), (33_000, 1), (132_000, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_many_small_ones(lap, rows, heads, d):
    n, scale = 400_000, 25.5 * math.log(2)
    q, k, v = (torch.zeros(1, h, m, d, dtype=torch.float16, device="cuda") for h, m in ((heads, rows), (1, n), (1, n)))
    q[..., 3], k[:, :, 5, 3], v[:] = 1, 1, 1
    v[:, :, 5] = 0
    got = lap.attention(q, k, v, scale=scale)
    w = (n - 1) * 2.0 ** -25.5
    want, lse = w / (1 + w), scale + math.log1p(w)
    assert float((got["out"].double() - want).abs().max()) <= want * (2.0 ** -6.5 + (n / 16 + n / 32) * 2.0 ** -24 + 2.0 ** -11)
    assert float((got["lse"].double() - lse).abs().max()) <= n / 32 * 2.0 ** -24 + 1e-5 * lse
