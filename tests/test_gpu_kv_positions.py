"""Evictions by positions up to the end of their range, in every form of the kernel."""
import pytest
import torch

import attention_ref as ref
from test_gpu_kv_cache import bits

pytestmark = pytest.mark.gpu

LAST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


def check(lap, kind, d, w, pos, lens, keep, recent, slots):
    b, h, n = w.shape
    gen = torch.Generator().manual_seed(n + keep)
    k, v = (torch.randn(b, n, h, d, generator=gen).to(kind).cuda().transpose(1, 2) for _ in range(2))
    got = lap.cache_evict(k, v, w.cuda(), keep, recent, slots=slots, positions=None if pos is None else pos.cuda(),
                          lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for i in range(b):
        m = n if lens is None else lens[i]
        assert int(got["lens"][i]) == min(keep, m)
        for j in range(h):
            at = torch.tensor(ref.evict(w[i, j], None if pos is None else pos[i, j], m, keep, recent), dtype=torch.long)
            c = len(at)
            want = at.int() if pos is None else pos[i, j, at]
            assert got["positions"][i, j].tolist() == want.tolist() + [-1] * (slots - c), (i, j)
            assert torch.equal(bits(got["weights"][i, j, :c].cpu()), bits(w[i, j, at])) and not got["weights"][i, j, c:].any()
            for x, y in ((k, got["k"]), (v, got["v"])):
                assert torch.equal(bits(y[i, j, :c]), bits(x[i, j, at.cuda()])) and not y[i, j, c:].any()


@pytest.mark.parametrize("recent", [0, 1, 3])
@pytest.mark.parametrize("last", [LAST, LAST - 1, 9])
@pytest.mark.parametrize("n", [100, 5000, 17_000])
def test_positions_up_to_the_largest(lap, n, last, recent):
    gen = torch.Generator().manual_seed(recent)
    w = torch.rand(1, 2, n, generator=gen)
    pos = (last - (n - 1) + torch.arange(n)).clamp(min=-1).int().expand(1, 2, n).contiguous()
    check(lap, torch.bfloat16, 64, w, pos, None, 20, recent, 20)
