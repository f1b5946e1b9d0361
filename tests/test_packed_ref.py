"""The packed rows' definition, on the CPU: what a row stands for is near what went in."""
import math

import pytest
import torch

import packed_ref as ref


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [8, 40, 128])
def test_error_is_half_a_step(kind, bits, d):
    gen = torch.Generator().manual_seed(d)
    x = (torch.randn(6, d, generator=gen) * torch.tensor([1.0, 1e-3, 100.0, 1.0, 0.0, 30.0])[:, None]).to(kind)
    x[3] += 7
    rows = ref.pack(x, bits)
    assert rows.shape == (6, ref.row_bytes(d, bits)) and rows.shape[1] % 16 == 0
    y = ref.unpack(rows, kind, d, bits)
    for i in range(6):
        assert torch.equal(y[i], ref.unpack_row(rows[i], kind, d, bits))
        for s in range(0, d, 32):
            g = x[i, s:s + 32].double()
            # step is rounded up by at most one part in 2^7 (2^10 in binary16), or, where it is tiny, by the least number there is
            step = (g.max() - g.min()) / (2 ** bits - 1) * (1 + torch.finfo(kind).eps) + 2.0 ** -24
            assert ((y[i, s:s + 32].double() - g).abs() <= step / 2 + g.abs().max() * torch.finfo(kind).eps).all()


def test_groups_that_are_not_numbers():
    x = torch.ones(3, 64).bfloat16()
    x[0, 40], x[1, 3] = math.nan, math.inf
    x[2, 0], x[2, 1] = -3e38, 3e38
    y = ref.unpack(ref.pack(x, 4), torch.bfloat16, 64, 4)
    assert y[0, :32].eq(1).all() and y[0, 32:].isnan().all()
    assert y[1, :32].isnan().all() and y[1, 32:].eq(1).all()
    assert y[2, :32].isnan().all() and y[2, 32:].eq(1).all()


def test_the_largest_numbers_stay_numbers():
    for kind in (torch.bfloat16, torch.float16):
        top = torch.finfo(kind).max
        x = torch.full((1, 32), top, dtype=kind)
        x[0, 0] = top * 0.37 if kind is torch.float16 else top - 2.0 ** 120 + 0.0
        x[0, 1] = x[0, 0]
        for bits in (4, 8):
            y = ref.unpack(ref.pack(x, bits), kind, 32, bits)
            if kind is torch.float16:
                assert y.isfinite().all()
            else:
                assert y.isnan().all()      # a range over 2^100
