"""Eviction and insertion: the same slots as the order's definition gives, and rows copied bit by bit."""
import math

import pytest
import torch

import attention_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


def bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def weights_of(gen, kind, *shape):
    if kind == "ties":
        return torch.randint(0, 3, shape, generator=gen).float()
    if kind == "even":
        return torch.zeros(shape)
    w = torch.rand(shape, generator=gen).pow(-0.7)
    if kind == "odd":      # what a sum may come to
        w[..., ::7] = math.nan
        w[..., 1::11] = -0.0
        w[..., 2::11] = 0.0
        w[..., 3::13] = math.inf
        w[..., 4::13] = -math.inf
        w[..., 5::17] = -w[..., 5::17]
    return w


# slots, keep, recent, slots of the new cache, lengths, weights, positions
EVICT = [
    (1, 1, 1, 1, None, "plain", None),
    (64, 16, 4, 16, None, "plain", None),
    (100, 100, 10, 128, [100, 0, 1], "plain", None),
    (1000, 300, 1, 300, [1000, 299, 300], "ties", None),
    (1500, 200, 200, 201, [1500, 150, -4], "plain", None),
    (777, 31, 0, 31, [777, 400, 32], "even", None),
    (2049, 512, 64, 600, None, "odd", None),
    (3000, 700, 50, 700, [3000, 2000, 5], "odd", "mixed"),
    (500, 100, 20, 100, None, "ties", "holes"),
    (40_000, 1000, 100, 1000, None, "plain", None),
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: "-".join(map(str, c)) if isinstance(c, tuple) else None)
def test_evict(lap, case):
    n, keep, recent, slots, lens, kind, places = case
    gen = torch.Generator().manual_seed(n)
    b, h, d = (2 if lens is None else len(lens)), 2, 72
    k, v = (torch.randn(b, n, h, d, generator=gen).to(torch.bfloat16).cuda().transpose(1, 2) for _ in range(2))
    w = weights_of(gen, kind, b, h, n)
    pos = None
    if places:
        pos = torch.stack([torch.stack([torch.randperm(4 * n, generator=gen)[:n] for _ in range(h)]) for _ in range(b)]).int()
        if places == "holes":
            pos[torch.rand(b, h, n, generator=gen) < 0.5] = -1
            pos[0, 0] = -1
    got = lap.cache_evict(k, v, w.cuda(), keep, recent, slots=slots, positions=None if pos is None else pos.cuda(),
                          lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"))
    for i in range(b):
        m = n if lens is None else max(0, lens[i])
        assert int(got["lens"][i]) == min(keep, m)
        for j in range(h):
            stay = ref.evict(w[i, j], None if pos is None else pos[i, j], m, keep, recent)
            c = len(stay)
            at = torch.tensor(stay, dtype=torch.long)
            want = at.int() if pos is None else pos[i, j, at]
            assert got["positions"][i, j].tolist() == want.tolist() + [-1] * (slots - c), (i, j)
            assert torch.equal(bits(got["weights"][i, j, :c].cpu()), bits(w[i, j, at])) and not got["weights"][i, j, c:].any()
            for x, y in ((k, got["k"]), (v, got["v"])):
                assert torch.equal(bits(y[i, j, :c]), bits(x[i, j, at.cuda()])) and not y[i, j, c:].any()


def test_an_evicted_cache_can_be_evicted_again(lap):
    gen = torch.Generator().manual_seed(2)
    k, v = (torch.randn(1, 2, 400, 64, generator=gen).half().cuda() for _ in range(2))
    w = torch.rand(1, 2, 400, generator=gen).cuda()
    once = lap.cache_evict(k, v, w, 100, 8)
    a = lap.cache_evict(once["k"], once["v"], once["weights"], 30, 8, lens=once["lens"], positions=once["positions"])
    b = lap.cache_evict(k, v, w, 30, 8)
    assert all(torch.equal(a[x], b[x]) for x in a)


def test_evict_from_nothing(lap):
    k = torch.empty(2, 3, 0, 64, dtype=torch.bfloat16, device="cuda")
    got = lap.cache_evict(k, k, torch.empty(2, 3, 0, device="cuda"), 5, 2)
    assert (got["positions"] == -1).all() and not got["lens"].any() and not got["k"].any() and not got["weights"].any()


@pytest.mark.parametrize("n,recent,kind", [(1, 1, "plain"), (5, 2, "ties"), (300, 0, "odd"), (1000, 17, "ties"), (4099, 1000, "odd")])
def test_insert_many_tokens(lap, n, recent, kind):
    """Into caches that fill up and then drop a slot for each token; one sequence sits out now and then."""
    gen = torch.Generator().manual_seed(n)
    b, h, d = 3, 2, 64
    kc, vc = (torch.zeros(b, n, h, d, dtype=torch.float16, device="cuda").transpose(1, 2) for _ in range(2))
    start = max(0, n - 2)
    w = weights_of(gen, kind, b, h, n)
    pos = torch.full((b, h, n), -1, dtype=torch.int32)
    pos[:, :, :start] = torch.arange(start, dtype=torch.int32)
    wc, pc = w.clone().cuda(), pos.clone().cuda()
    keys, values = kc.cpu().clone(), vc.cpu().clone()
    for step in range(8):
        kn, vn = (torch.randn(b, 1, h, d, generator=gen).half().transpose(1, 2)[:, :, 0] for _ in range(2))
        at = torch.tensor([start + step, start + step, -1 if step % 3 == 1 else start + step], dtype=torch.int32)
        got = lap.cache_insert(kn.cuda(), vn.cuda(), kc, vc, wc, pc, at.cuda(), recent)["slots"].cpu()
        for i in range(b):
            for j in range(h):
                if at[i] < 0:
                    assert int(got[i, j]) == -1
                    continue
                s = ref.insert(w[i, j], pos[i, j], int(at[i]), recent)
                assert int(got[i, j]) == s, (step, i, j)
                w[i, j, s], pos[i, j, s], keys[i, j, s], values[i, j, s] = 0.0, at[i], kn[i, j], vn[i, j]
    assert torch.equal(pc.cpu(), pos) and torch.equal(bits(wc.cpu()), bits(w))
    assert torch.equal(bits(kc.cpu()), bits(keys)) and torch.equal(bits(vc.cpu()), bits(values))
