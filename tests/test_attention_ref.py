"""The 64-bit reference of the attention tests against a second method and against differences, on the CPU."""
import math

import pytest
import torch

import attention_ref as ref


def _inputs(seed, b, h, kv, nq, nk, d):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g).to(torch.float16) for s in ((b, h, nq, d), (b, kv, nk, d), (b, kv, nk, d), (b, h, nq, d))]


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 0), (True, 3)])
def test_gradients_are_those_of_autograd_and_of_differences(causal, window):
    q, k, v, g = _inputs(1, 2, 4, 2, 7, 9, 8)
    case = ref.Case(q, k, v, causal=causal, window=window, q_lens=[7, 5], k_lens=[9, 4])

    def loss(q, k, v):
        kg, vg = k.repeat_interleave(2, 1), v.repeat_interleave(2, 1)
        s = (q @ kg.transpose(-1, -2)) / math.sqrt(8)
        s = s.masked_fill(~case.see, -1e300)
        p = torch.softmax(s, -1) * case.see
        return (p @ vg * g.double()).sum()

    ts = [x.clone().requires_grad_() for x in (case.q, case.k, case.v)]
    loss(*ts).backward()
    got = case.grads(g, case.out)
    for name, t in zip(("dq", "dk", "dv"), ts):
        assert torch.allclose(got[name][0], t.grad, rtol=1e-9, atol=1e-9), name
        step = torch.randn(t.shape, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
        h = 1e-5
        args = lambda s: [x + s * step if x is t else x for x in (ts[0], ts[1], ts[2])]
        with torch.no_grad():
            diff = (loss(*[a.detach() for a in args(h)]) - loss(*[a.detach() for a in args(-h)])) / (2 * h)
        assert abs(float(diff - (t.grad * step).sum())) < 1e-6 * (1 + float(diff.abs()))


def test_rows_that_see_nothing():
    q, k, v, g = _inputs(3, 1, 2, 1, 5, 3, 8)
    case = ref.Case(q, k, v, causal=True)      # five rows at the end of three keys: the first two see none
    assert torch.equal(case.lse[0, :, :2], torch.full((2, 2), -math.inf, dtype=torch.float64))
    assert not case.out[0, :, :2].any() and not case.grads(g, case.out)["dq"][0][0, :, :2].any()


def test_choice_of_slots_by_hand():
    w = [3.0, 1.0, float("nan"), 1.0, 0.5, 9.0, 2.0]
    assert ref.evict(w, None, 7, 7, 1) == list(range(7))
    assert ref.evict(w, None, 7, 4, 1) == [0, 1, 5, 6]          # the newest, 9, 3 and the lower of the two 1s
    assert ref.evict(w, None, 7, 2, 2) == [5, 6]
    assert ref.evict(w, None, 3, 2, 0) == [0, 1]                # not a number is least
    assert ref.evict(w, [4, 5, -1, 6, 7, 8, -1], 7, 3, 1) == [0, 1, 5]
    assert ref.insert(w, range(7), 7, 2) == 2
    assert ref.insert(w[:2] + w[3:], range(6), 6, 2) == 3       # 0.5
    assert ref.insert(w[:2] + w[3:], range(6), 6, 4) == 2       # slots 3 .. are among the newest, and 1 and 2 are equal
    assert ref.insert([1.0, 1.0, 4.0], [0, 1, 2], 3, 1) == 1    # of equal ones the higher
    assert ref.insert(w, [4, 5, 9, -1, 7, -1, 6], 10, 2) == 3
