"""The example at sizes where the backward pass takes its rows in parts, and the forward pass its keys."""
import pytest
import torch

from test_gpu_attention_example import example  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,heads,tokens,size", [(1, 4, 2048, 64), (1, 1, 4096, 128), (2, 3, 65, 8)])
def test_training_in_a_pool(example, batch, heads, tokens, size):  # noqa: F811
    import paper_1903_06631_amd as lap
    shape, numbers = (batch, heads, tokens, size), batch * heads * tokens * 4
    need = [lap.attention_workspace_bytes(call, shape, shape, torch.bfloat16, causal=True) for call in (lap.AT_FORWARD, lap.AT_GRAD)]
    assert (need[0] > 0) == (tokens > 1000) and (need[1] > 2 * numbers + 256) == (tokens > 1000)
    grads, alone, plans = example.train(layers=2, batch=batch, heads=heads, tokens=tokens, size=size)
    assert all(torch.equal(a[n], b[n]) for a, b in zip(grads, alone) for n in a)
    assert plans["peak"] <= plans["footprint"]
