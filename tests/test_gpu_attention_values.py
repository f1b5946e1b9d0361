"""Values that are not finite, or lie at the ends of their type, where the definition still says what a result is."""
import math

import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


def normal(gen, h, n, d, kind):
    return torch.randn(1, h, n, d, generator=gen).to(kind).cuda()


# head size; query heads and key heads; the rest of the shapes as few as reach the sharings of the waves
@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("d,heads,kv", [(72, 2, 1), (8, 2, 2), (40, 150, 75), (120, 300, 300), (64, 2, 1), (128, 2, 1)])
def test_a_key_hidden_by_minus_infinity(lap, kind, d, heads, kv):
    """The last element of the head as a mask: 1 in every query, minus infinity in the keys that are not to be seen.  Their
    scores are minus infinity, their probabilities 0, and so are their weights and the gradients of their values; all else is
    what it is without those keys."""
    gen = torch.Generator().manual_seed(d)
    n = 130
    q, k, v, g = normal(gen, heads, n, d, kind), normal(gen, kv, n, d, kind), normal(gen, kv, n, d, kind), normal(gen, heads, n, d, kind)
    hide = torch.zeros(n, dtype=torch.bool)
    hide[[3, 64, 100, n - 1]] = True
    q[..., d - 1], k[..., d - 1] = 1, 0
    want = ref.Case(q, k[:, :, ~hide], v[:, :, ~hide])
    k[:, :, hide.cuda(), d - 1] = -math.inf
    got = lap.attention(q, k, v)
    assert float(((got["lse"].cpu().double() - want.lse).abs() - want.lse_bound).max()) <= 0
    assert float(((got["out"].cpu().double() - want.out).abs() - want.out_bound).max()) <= 0
    grads = lap.attention_grad(g, q, k, v, got["out"], got["lse"])
    dv, bound = want.grads(g, got["out"])["dv"]
    assert float(((grads["dv"][:, :, ~hide.cuda()].cpu().double() - dv).abs() - bound).max()) <= 0 and not grads["dv"][:, :, hide.cuda()].any()
    w, bound = want.weights()
    got_w = lap.attention_weights(q, k, got["lse"])["weights"].cpu().double()
    assert float(((got_w[:, :, ~hide] - w).abs() - bound).max()) <= 0 and not got_w[:, :, hide].any()


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("kv,slots,lens", [(1, 40, [33]), (8, 1000, [1000 - 7]), (2, 5000, [4097]), (96, 1500, [1025, 3, 64])])
def test_an_infinite_value_in_the_last_slot_of_a_step(lap, kind, kv, slots, lens):
    """Its sign is the output's: the rest of its tile, past the length, has no part in it."""
    gen = torch.Generator().manual_seed(slots)
    b, d = len(lens), 64
    q = torch.randn(b, 2 * kv, d, generator=gen).to(kind).cuda()
    k, v = (torch.randn(b, kv, slots, d, generator=gen).to(kind).cuda() for _ in range(2))
    clean = lap.attention_step(q, k, v, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))["out"]
    for i, n in enumerate(lens):
        v[i, :, n - 1, 5], v[i, :, n - 1, 6] = math.inf, -math.inf
    out = lap.attention_step(q, k, v, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))["out"]
    assert (out[..., 5] == math.inf).all() and (out[..., 6] == -math.inf).all()
    rest = [e for e in range(d) if e not in (5, 6)]
    assert torch.equal(out[..., rest], clean[..., rest])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,heads", [(200, 2), (600, 40)])
def test_weights_of_a_row_that_is_not_a_number(lap, n, heads, causal):
    """Every key that such a row sees has a weight that is not a number, and no key that only others see."""
    gen = torch.Generator().manual_seed(n)
    q, k, v = normal(gen, heads, n, 64, BF), normal(gen, heads // 2, n, 64, BF), normal(gen, heads // 2, n, 64, BF)
    k[:, :, 150] = math.nan
    got = lap.attention(q, k, v, causal=causal)
    w = lap.attention_weights(q, k, got["lse"], causal=causal)["weights"]
    assert torch.isnan(w).all()      # the last rows see key 150 and all before them; without a mask all do
    k[:, :, 150] = 1
    q[:, ::2, 100] = math.nan        # one row: keys up to 100 under a causal mask
    got = lap.attention(q, k, v, causal=causal)
    w = lap.attention_weights(q, k, got["lse"], causal=causal)["weights"]
    assert torch.isnan(w[..., :101]).all() and (not causal or torch.isfinite(w[..., 101:]).all())


@pytest.mark.parametrize("product,scale,hidden", [(-2.0 ** 93, 2.0 ** 10, False), (-2.0 ** 93, 2.0 ** -10, False), (-2.0 ** 101, 2.0 ** 10, True),
                                                  (-2.0 ** 101, 2.0 ** -10, True)])
def test_one_rule_for_what_counts_as_hidden(lap, product, scale, hidden):
    """A product q.k below -1e30 (2^99.7), whatever the scale, in a prompt, in its weights and in a step."""
    for n in (1, 700, 3000):
        q, k, v = torch.zeros(1, 1, 1, 64, dtype=BF, device="cuda"), torch.zeros(1, 1, n, 64, dtype=BF, device="cuda"), torch.ones(1, 1, n, 64, dtype=BF, device="cuda")
        q[..., 0], k[..., 0] = 2.0 ** 40, product / 2.0 ** 40
        # n equal scores: the logarithm of n is far below what 32 bits hold beside them
        want = -math.inf if hidden else product * scale
        weight = 0.0 if hidden else 1.0
        a, b = lap.attention(q, k, v, scale=scale), lap.attention_step(q[:, :, 0], k, v, torch.zeros(1, 1, n, device="cuda"), scale=scale)
        assert float(a["lse"][0, 0, 0]) == want
        assert float(b["lse"][0, 0]) == (want if hidden else pytest.approx(want, rel=1e-6))      # (held to base 2 there)
        assert (a["out"] == weight).all() and (b["out"] == weight).all()
        w = lap.attention_weights(q, k, a["lse"], scale=scale)["weights"]
        if n == 1:
            assert float(w[0, 0, 0]) == weight and float(b["weights"][0, 0, 0]) == weight
        elif hidden:
            assert not w.any() and not b["weights"].any()
