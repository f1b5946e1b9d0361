"""Results carry no gradient, which is said where one would be expected; the function around the two calls gives the gradients."""
import warnings

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_warning_where_a_gradient_is_expected():
    import paper_1903_06631_amd as lap
    lap.load_library()
    q = torch.randn(1, 2, 9, 64, device="cuda").half()
    for i in range(3):
        args = [q.clone().requires_grad_(i == j) for j in range(3)]
        with pytest.warns(UserWarning, match="attention_grad"):
            got = lap.attention(*args)
        assert not got["out"].requires_grad
        with pytest.warns(UserWarning, match="no gradient"):
            lap.attention_step(args[0][:, :, 0], *args[1:])
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            with torch.no_grad():
                lap.attention(*args)
                lap.attention_step(args[0][:, :, 0], *args[1:])
            lap.attention(q, q, q)


def test_a_function_around_both():
    import paper_1903_06631_amd as lap

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            f = lap.attention(q, k, v, causal=True, sync=False)
            ctx.save_for_backward(q, k, v, f["out"], f["lse"])
            return f["out"]

        @staticmethod
        def backward(ctx, dout):
            return tuple(lap.attention_grad(dout.contiguous(), *ctx.saved_tensors, causal=True, sync=False).values())

    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, g = (torch.randn(2, 4, 70, 64, generator=gen, device="cuda").bfloat16() for _ in range(4))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        xs = [x.clone().requires_grad_() for x in (q, k, v)]
        (Attention.apply(*xs).float() * g.float()).sum().backward()
    f = lap.attention(q, k, v, causal=True)
    want = lap.attention_grad(g, q, k, v, f["out"], f["lse"], causal=True)
    assert all(torch.equal(x.grad, want[n]) for x, n in zip(xs, ("dq", "dk", "dv")))
