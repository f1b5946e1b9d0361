"""Evictions in every form of the kernel (up to 4096, up to 16384 and more slots), rows shared by several workgroups, with ties,
weights that are not numbers, positions in any order, holes, and lengths from 0 on."""
import pytest
import torch

from test_gpu_kv_cache import weights_of
from test_gpu_kv_positions import check

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


def positions(gen, places, b, h, n):
    if places is None:
        return None
    pos = torch.stack([torch.stack([torch.randperm(4 * n, generator=gen)[:n] for _ in range(h)]) for _ in range(b)]).int()
    if places == "holes":
        pos[torch.rand(b, h, n, generator=gen) < 0.4] = -1
        pos[0, 0] = -1
    return pos


@pytest.mark.parametrize("n", [4096, 4097, 10_000, 16_384, 16_385, 30_011])
@pytest.mark.parametrize("weights,places", [("ties", None), ("odd", "mixed"), ("odd", "holes"), ("even", "holes"), ("plain", None)])
def test_every_form(lap, n, weights, places):
    gen = torch.Generator().manual_seed(n)
    lens = [n, n // 2 + 1, 1, 0, 65]
    w, pos = weights_of(gen, weights, 5, 2, n), positions(gen, places, 5, 2, n)
    kind, d = (BF, 8) if n % 2 else (HF, 128)
    for keep, recent, slots in ((1, 0, 1), (700, 70, 700), (n // 2, n // 2, n // 2 + 300), (n, 0, n)):
        check(lap, kind, d, w, pos, lens, keep, recent, slots)


@pytest.mark.parametrize("n", [5000, 16_385])
def test_many_rows(lap, n):
    """As many rows as leave each one workgroup, and none to spare."""
    gen = torch.Generator().manual_seed(n)
    w = weights_of(gen, "ties", 50, 6, n)
    check(lap, BF, 16, w, None, None, 300, 20, 300)
