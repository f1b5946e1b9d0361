"""The example runs the operators together: a training pass inside a planned pool gives the bits that it gives outside, and
a cache's choice follows the weights."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("attention_within_a_limit", os.path.join(ROOT, "examples", "attention_within_a_limit.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_training_in_a_pool(example):
    grads, alone, plans = example.train(layers=3, batch=1, heads=4, tokens=300, size=64)
    assert all(torch.equal(a[n], b[n]) for a, b in zip(grads, alone) for n in a)
    assert plans["peak"] <= plans["footprint"] < plans["peak_kept"]


def test_serving_from_few_slots(example):
    out, full, cache, tokens = example.serve(prompt=400, slots=64, recent=16, new=20)
    pos = cache["positions"]
    assert ((pos >= 420 - 16).sum(-1) == 16).all()                        # the newest are there
    assert all(len(set(row.tolist())) == 64 for row in pos.reshape(-1, 64))      # and no token twice
    assert tokens == 420
    # with a slot for every token the cache holds all of them, and the output is that of full attention
    out, full, cache, tokens = example.serve(prompt=100, slots=120, recent=16, new=20)
    assert (cache["positions"].sort(-1).values == torch.arange(120, device="cuda")).all()
    assert torch.allclose(out.float(), full.float(), rtol=2 ** -6, atol=2 ** -8)
