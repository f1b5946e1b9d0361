"""binary16 over its range: gradients of any size that the type holds, and probabilities far below a row's largest, come out
as accurately as results in 32 bits that are rounded once to the type, but for one relative rounding of each probability and
each ds.  The bounds are those of attention_ref.py without its allowance for values below the type's normal range (`tiny`);
in its place stand the kernels' own: ds = p z, z = g.v - delta, is rounded in multiples of a power of two that puts the largest
z of its row above 2^11, so that half the type's smallest unit, 2^-25, is at most 2^-36 of that largest one (2^-35 with its own
error), and probabilities as multiples of 2^-12, so 2^-37.  A result below the normal range is off by another 2^-25."""
import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu

HF = torch.float16
HALF_UNIT = 2.0 ** -25


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


def over(got, want, bound):
    """How far the worst element is beyond its bound."""
    got = got.detach().cpu().double()
    assert torch.isfinite(want).all() and float(want.abs().max()) < 65504
    assert torch.isfinite(got).all(), "not finite"
    return float(((got - want).abs() - bound).max())


def grads_within(lap, q, k, v, g, **mask):
    want = ref.Case(q, k, v, **mask)
    want.tiny = 0.0
    got = lap.attention(*[x.cuda() for x in (q, k, v)], **mask)
    grads = lap.attention_grad(*[x.cuda() for x in (g, q, k, v)], got["out"], got["lse"], **mask)
    exact = want.grads(g, got["out"])
    dp = g.double() @ want.vg.transpose(-1, -2)
    z = (dp - (g.double() * got["out"].cpu().double()).sum(-1, keepdim=True)).abs() * want.see
    see, t = want.see.double().expand(want.p.shape), lambda x: x.transpose(-1, -2)
    unit = 2.0 ** -35
    floor = dict(dq=want.scale * unit * z.amax(-1, keepdim=True) * (see @ want.kg.abs()),
                 # a key's largest is that over all query heads that share it
                 dk=want.scale * unit * want.shared(z.amax(-2)).unsqueeze(-1) * want.shared(t(see) @ want.q.abs()),
                 dv=2.0 ** -37 * want.shared(t(see) @ g.double().abs()))
    for name, (value, bound) in exact.items():
        assert over(grads[name], value, bound + floor[name] + HALF_UNIT) <= 0, name


# head size, query heads, key heads, tokens: every sharing of the waves, and rows in parts
SIZES = [(128, 2, 2, 333), (64, 8, 1, 1100), (72, 300, 150, 150), (128, 130, 130, 130), (128, 700, 700, 130)]


@pytest.mark.parametrize("d,heads,kv,n", SIZES)
@pytest.mark.parametrize("kind", ["2^-18", "2^-10", "2^0", "2^12", "rows", "values"])
def test_gradients_of_every_size(lap, d, heads, kv, n, kind):
    gen = torch.Generator().manual_seed(d + n)
    normal = lambda h, times=1.0: torch.randn(1, h, n, d, generator=gen) * times
    q, k, v, g = normal(heads, 1.5), normal(kv), normal(kv), normal(heads)
    if kind == "rows":          # rows next to each other 2^26 apart
        g = g * 2.0 ** torch.randint(-16, 11, (1, heads, n, 1), generator=gen)
    elif kind == "values":      # large values, small keys: ds beyond the type's largest, its sums within
        q, k, v, g = q / 8, k / 8, v * 32, g * 2.0 ** 10
    else:
        g = g * 2.0 ** int(kind[2:])
        if kind == "2^12" and heads > 2 * kv:
            g = g / 4
    grads_within(lap, *[x.to(HF) for x in (q, k, v, g)], causal=True)


def test_gradients_of_many_even_keys(lap):
    """Probabilities of 1/150000, below the type's normal range, in every sum."""
    n, d, rows = 150_000, 64, 33
    gen = torch.Generator().manual_seed(1)
    q = torch.zeros(1, 1, rows, d, dtype=HF)
    k, v = (torch.randn(1, 1, n, d, generator=gen).to(HF) for _ in range(2))
    g = torch.rand(1, 1, rows, d, generator=gen).add(0.5).mul(256).to(HF)
    grads_within(lap, q, k, v, g)
