"""Numbers of keys and slots that are none are refused, and not taken for the next one below."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_counts():
    import paper_1903_06631_amd as lap
    lap.load_library()
    k, w = torch.ones(1, 2, 16, 64, dtype=torch.bfloat16, device="cuda"), torch.rand(1, 2, 16, device="cuda")
    for bad in (0.5, 2.5, float("nan"), float("inf"), -1):
        with pytest.raises(ValueError):
            lap.attention(k, k, k, causal=True, window=bad)
        for args, kw in (((bad, 0), {}), ((4, bad), {}), ((4, 0), dict(slots=bad))):
            with pytest.raises(ValueError):
                lap.cache_evict(k, k, w, *args, **kw)
    for good in (4, 4.0, True + 3):
        assert lap.cache_evict(k, k, w, good, 0, slots=good)["k"].shape[2] == 4
