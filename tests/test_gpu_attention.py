"""Attention, its gradient, the weights of the keys and the single-token form against 64 bits: every element within a bound
that follows from the roundings (attention_ref.py).  Padding is filled with not-a-number throughout."""
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


def rows(gen, b, h, n, d, kind, lens=None, layout="bhnd", times=1.0):
    """Normal values on the GPU, [b, h, n, d]; what is beyond the lengths is not a number."""
    x = torch.randn(b, h, n, d, generator=gen) * times
    if lens is not None:
        for i, m in enumerate(lens):
            x[i, :, max(0, m):] = math.nan
    x = x.to(kind)
    if layout == "bnhd":
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
    if layout == "gaps":      # rows, heads and sequences apart, starting off the allocation's start
        big = torch.full((b, h + 1, n + 3, d + 24), math.nan, dtype=kind)
        big[:, :h, 1:n + 1, 8:d + 8] = x
        return big.cuda()[:, :h, 1:n + 1, 8:d + 8]
    return x.cuda()


def lens_tensor(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


def within(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    err = (got - want).abs()[~inf]
    assert not torch.isnan(err).any(), f"{what}: not a number"
    over = err - bound.expand(want.shape)[~inf]
    assert err.numel() == 0 or float(over.max()) <= 0, f"{what}: off by {float(err.max())}, over its bound by {float(over.max())}"


# kind, head size, query heads, key heads, queries, keys, causal, window, query lengths, key lengths, layout
CASES = [
    (BF, 128, 2, 2, 1, 1, False, 0, None, None, "bhnd"),
    (HF, 64, 2, 1, 1, 300, True, 0, None, None, "bhnd"),
    (BF, 64, 1, 1, 33, 31, False, 0, None, None, "bhnd"),
    (HF, 128, 4, 2, 128, 64, True, 0, None, None, "bnhd"),            # the first 64 rows see no key
    (BF, 128, 4, 4, 129, 129, True, 0, None, None, "bnhd"),
    (BF, 80, 6, 2, 200, 333, True, 0, None, None, "gaps"),
    (HF, 8, 3, 3, 65, 97, False, 0, None, None, "gaps"),
    (BF, 120, 2, 1, 70, 70, True, 17, None, None, "bhnd"),
    (HF, 64, 2, 2, 260, 515, True, 64, None, None, "bhnd"),           # whole tiles before the window
    (BF, 128, 2, 1, 150, 190, True, 1, None, None, "bhnd"),
    (HF, 128, 8, 2, 97, 161, True, 0, [97, 0, 1, 50], [161, 7, 1, 33], "bhnd"),      # empty and single rows, more rows than keys
    (BF, 64, 2, 2, 130, 257, False, 0, [130, 129, 64, 3], [257, 0, 65, 1], "gaps"),    # no key at all
    (BF, 128, 16, 1, 40, 300, True, 33, [40, -3, 400, 17], [300, 64, 128, 5], "bhnd"),  # lengths out of range count as none and all
    (HF, 96, 2, 2, 0, 50, False, 0, None, None, "bhnd"),
    (BF, 64, 2, 2, 50, 0, True, 0, None, None, "bhnd"),
    (HF, 128, 5, 5, 513, 640, True, 0, None, None, "bhnd"),
    # few rows on many keys: the keys in parts, some of them with nothing for a row
    (BF, 128, 4, 2, 70, 2200, True, 0, [70, 0, 33], [2200, 100, 1], "bhnd"),
    (HF, 64, 2, 1, 33, 3001, False, 0, [33, 1], [3001, 0], "gaps"),
    (BF, 104, 2, 2, 65, 2100, True, 300, None, None, "bnhd"),
    # as many blocks of rows or keys as take another sharing of the waves, and fewer key heads than those by far
    (BF, 128, 66, 33, 130, 140, True, 0, [130, 0, 77, 64], [140, 140, 5, 129], "bhnd"),
    (HF, 64, 140, 70, 150, 170, True, 40, [150, 128, 1, 97], [170, 128, 64, 33], "bnhd"),
    (BF, 72, 132, 132, 129, 70, True, 0, [129, 128, 65, 2], [70, 64, 33, 70], "bhnd"),
    (HF, 128, 86, 43, 130, 137, True, 0, [130, 129, 33, 64], [137, 130, 137, 65], "bhnd"),
    # many rows on few keys: the rows in parts, for the weights and for the keys' gradients
    (BF, 64, 8, 1, 1100, 1300, True, 0, None, None, "bhnd"),
    (HF, 120, 8, 2, 900, 333, False, 0, [900, 17], [333, 0], "gaps"),
    (BF, 128, 12, 2, 400, 400, True, 50, [400, 100, 1], [400, 50, 7], "bhnd"),
]


def make(case, seed=0):
    kind, d, h, kv, nq, nk, causal, window, q_lens, k_lens, layout = case
    gen = torch.Generator().manual_seed(seed + 1000 * d + nq)
    b = 2 if q_lens is None else len(q_lens)
    q = rows(gen, b, h, nq, d, kind, q_lens, layout, 1.5)
    k, v = rows(gen, b, kv, nk, d, kind, k_lens, layout), rows(gen, b, kv, nk, d, kind, k_lens, layout)
    g = rows(gen, b, h, nq, d, kind, q_lens, layout)
    mask = dict(causal=causal, window=window)
    want = ref.Case(q, k, v, q_lens=q_lens, k_lens=k_lens, **mask)
    mask.update(q_lens=lens_tensor(q_lens), k_lens=lens_tensor(k_lens))
    return q, k, v, g, mask, want


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c[:8]) if isinstance(c, tuple) else None)
def test_forward_backward_and_weights(lap, case):
    q, k, v, g, mask, want = make(case)
    got = lap.attention(q, k, v, **mask)
    within(got["lse"], want.lse, want.lse_bound, "lse")
    within(got["out"], want.out, want.out_bound, "out")
    grads = lap.attention_grad(g, q, k, v, got["out"], got["lse"], **mask)
    for name, (value, bound) in want.grads(g, got["out"]).items():
        within(grads[name], value, bound, name)
    w = lap.attention_weights(q, k, got["lse"], **mask)["weights"]
    value, bound = want.weights()
    within(w, value, bound, "weights")
    before = torch.rand(w.shape, generator=torch.Generator().manual_seed(5)).cuda()
    more = lap.attention_weights(q, k, got["lse"], before=before, weights=before, **mask)["weights"]      # in place
    assert torch.equal(more, torch.rand(w.shape, generator=torch.Generator().manual_seed(5)).cuda() + w)
    # equal calls, equal bits
    again = lap.attention_grad(g, q, k, v, got["out"], got["lse"], **mask)
    assert all(torch.equal(grads[n], again[n]) for n in grads)


def test_gradient_against_differences(lap):
    case = (HF, 64, 4, 2, 45, 60, True, 0, None, None, "bhnd")
    q, k, v, g, mask, want = make(case)
    got = lap.attention(q, k, v, **mask)
    grads = lap.attention_grad(g, q, k, v, got["out"], got["lse"], **mask)
    bounds = want.grads(g, got["out"])
    gen = torch.Generator().manual_seed(9)
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2)):
        xs = [q, k, v]
        step = torch.randn(xs[at].shape, generator=gen, dtype=torch.float64)
        loss = []
        for sign in (1, -1):
            c = ref.Case(q, k, v, causal=True)
            full = [c.q, c.k, c.v]
            full[at] = full[at] + sign * 1e-4 * step
            s = (c.scale * full[0] @ full[1].repeat_interleave(2, 1).transpose(-1, -2)).masked_fill(~c.see, -math.inf)
            loss.append(float((torch.softmax(s, -1) @ full[2].repeat_interleave(2, 1) * g.cpu().double()).sum()))
        diff = (loss[0] - loss[1]) / 2e-4
        along = float((grads[name].cpu().double() * step).sum())
        # delta is taken from the rounded output: off by u |g||o| for each row, p-weighted
        slack = float((bounds[name][1] * step.abs()).sum()) + 2 * want.u * float(step.abs().sum())
        assert abs(diff - along) <= slack, (name, diff, along, slack)


def test_scale_and_large_scores(lap):
    gen = torch.Generator().manual_seed(4)
    q, k, v = (rows(gen, 1, 2, 90, 64, BF) for _ in range(3))
    for scale in (1e-6, 0.3, 30.0):      # nearly even, ordinary, one key takes all
        want = ref.Case(q, k, v, scale=scale, causal=True)
        got = lap.attention(q, k, v, scale=scale, causal=True)
        within(got["lse"], want.lse, want.lse_bound, f"lse at {scale}")
        within(got["out"], want.out, want.out_bound, f"out at {scale}")


@pytest.mark.parametrize("kind,d,heads,kv,n,window", [(BF, 128, 2, 2, 200, 0), (HF, 64, 4, 2, 333, 50), (BF, 72, 300, 150, 150, 0), (HF, 128, 700, 700, 130, 33)])
def test_what_is_not_finite_reaches_only_rows_that_see_it(lap, kind, d, heads, kv, n, window):
    """Keys, values, queries and gradients with infinities and not-a-numbers in places that a causal mask hides from part of
    the rows: those are within the bounds of the same call without them, wherever the places fall in a tile."""
    gen = torch.Generator().manual_seed(6)
    q, g = rows(gen, 1, heads, n, d, kind), rows(gen, 1, heads, n, d, kind)
    k, v = rows(gen, 1, kv, n, d, kind), rows(gen, 1, kv, n, d, kind)
    mask = dict(causal=True, window=window)
    want = ref.Case(q, k, v, **mask)
    see = want.see[0, 0]
    clean = lap.attention(q, k, v, **mask)
    bad_keys = [n // 2 + 3, n - 1]
    k2, v2 = k.clone(), v.clone()
    k2[:, :, bad_keys[0]], v2[:, :, bad_keys[0], 5:9], v2[:, :, bad_keys[1]] = math.inf, math.nan, -math.inf
    got = lap.attention(q, k2, v2, **mask)
    fine = ~see[:, bad_keys].any(1)
    assert fine.any() and not fine.all()
    within(got["lse"][:, :, fine], want.lse[:, :, fine], want.lse_bound[:, :, fine], "lse")
    within(got["out"][:, :, fine], want.out[:, :, fine], want.out_bound[:, :, fine], "out")
    assert not torch.isfinite(got["out"][:, :, ~fine.cuda()]).all(-1).any()      # and the others show it
    exact = want.grads(g, clean["out"])
    grads = lap.attention_grad(g, q, k2, v2, clean["out"], clean["lse"], **mask)
    within(grads["dq"][:, :, fine], exact["dq"][0][:, :, fine], exact["dq"][1][:, :, fine], "dq")
    # rows that only part of the keys is seen from
    bad_rows = [0, n // 2 - 2]
    q2, g2 = q.clone(), g.clone()
    q2[:, :, bad_rows[0]], g2[:, :, bad_rows[1], 1] = math.nan, math.inf
    grads = lap.attention_grad(g2, q2, k, v, clean["out"], clean["lse"], **mask)
    fine = ~see[bad_rows].any(0)
    assert fine.any() and not fine.all()
    for name in ("dk", "dv"):
        within(grads[name][:, :, fine], exact[name][0][:, :, fine], exact[name][1][:, :, fine], name)
    w = lap.attention_weights(q2, k, clean["lse"], **mask)["weights"]
    value, bound = want.weights()
    fine = ~see[0]
    within(w[:, :, fine], value[:, :, fine], bound[:, :, fine], "weights")


def test_broadcast_keys_and_their_gradient(lap):
    gen = torch.Generator().manual_seed(8)
    q, g = rows(gen, 3, 4, 70, 64, BF), rows(gen, 3, 4, 70, 64, BF)
    k1, v1 = rows(gen, 1, 1, 90, 64, BF), rows(gen, 1, 1, 90, 64, BF)
    k, v = k1.expand(3, 2, 90, 64), v1.expand(3, 2, 90, 64)
    a = lap.attention(q, k, v)
    b = lap.attention(q, k.contiguous(), v.contiguous())
    assert torch.equal(a["out"], b["out"])
    ga = lap.attention_grad(g, q, k, v, a["out"], a["lse"])
    gb = lap.attention_grad(g, q, k.contiguous(), v.contiguous(), a["out"], a["lse"])
    assert ga["dk"].shape == (3, 2, 90, 64) and all(torch.equal(ga[n], gb[n]) for n in ga)      # one for each copy


# kind, head size, query heads, key heads, slots, lengths, holes
STEPS = [
    (BF, 128, 2, 2, 1, None, False),
    (HF, 64, 8, 2, 31, [31, 0, 1], False),
    (BF, 128, 7, 1, 1000, [1000, 999, 33], False),
    (HF, 72, 3, 3, 515, None, True),
    (BF, 64, 40, 1, 300, [300, 0, 129], True),          # more heads than a matrix operand has columns
    (HF, 128, 16, 8, 5000, [5000, 4097, 2], False),
    (BF, 128, 256, 1, 200, None, False),
    (HF, 128, 32, 1, 1000, [1000, 31, 0, 545], True),
    (BF, 64, 4, 2, 1024, [1024, 1023], False),
    (HF, 64, 2, 2, 1025, [1025, 1024], True),
    (BF, 64, 8, 8, 1500, [1500 - 90 * i for i in range(16)], False),
    (HF, 72, 24, 24, 2100, [2100, 2047, 1, 0, 2100, 33, 999, 5], False),
]


@pytest.mark.parametrize("case", STEPS, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c) if isinstance(c, tuple) else None)
def test_step(lap, case):
    kind, d, h, kv, n, lens, holes = case
    gen = torch.Generator().manual_seed(n + h)
    b = 2 if lens is None else len(lens)
    q = rows(gen, b, h, 1, d, kind, times=1.5)
    k, v = rows(gen, b, kv, n, d, kind, lens, "gaps"), rows(gen, b, kv, n, d, kind, lens, "bnhd")
    pos = torch.randint(0, 1 << 30, (b, kv, n), generator=gen, dtype=torch.int32)
    if holes:
        pos[torch.rand(b, kv, n, generator=gen) < 0.3] = -1
        pos[0] = -1                                       # a cache with nothing in it
        empty = (pos < 0).cuda()
        k[empty], v[empty] = math.nan, math.nan           # an empty slot may hold anything
    want = ref.Case(q, torch.where(torch.isnan(k), 0, k), torch.where(torch.isnan(v), 0, v), k_lens=lens)
    if holes:      # hide the empty slots: the same definition with another visible set
        see = want.see & (pos >= 0).repeat_interleave(h // kv, 1)[:, :, None, :]
        s = (want.scale * want.q @ want.kg.transpose(-1, -2)).masked_fill(~see, -math.inf)
        want.lse = torch.logsumexp(s, -1)
        want.p = torch.exp(s - want.lse[..., None].masked_fill(want.lse[..., None] == -math.inf, 0))
        want.out = want.p @ want.vg
    before = torch.rand(b, kv, n, generator=gen)
    got = lap.attention_step(q[:, :, 0], k, v, before.cuda(), lens=lens_tensor(lens), positions=pos.cuda() if holes else None)
    within(got["lse"], want.lse[..., 0], want.lse_bound[..., 0], "lse")
    within(got["out"], want.out[:, :, 0], want.out_bound[:, :, 0], "out")
    value, bound = want.weights()
    within(got["weights"], value + before, bound + 2.0 ** -23 * (value + before), "weights")
    plain = lap.attention_step(q[:, :, 0], k, v, lens=lens_tensor(lens), positions=pos.cuda() if holes else None)
    assert plain["weights"] is None and torch.equal(plain["out"], got["out"]) and torch.equal(plain["lse"], got["lse"])


def test_step_without_slots(lap):
    q, empty = torch.ones(2, 4, 64, dtype=BF, device="cuda"), torch.empty(2, 2, 0, 64, dtype=BF, device="cuda")
    got = lap.attention_step(q, empty, empty, torch.empty(2, 2, 0, device="cuda"))
    assert not got["out"].any() and (got["lse"] == -math.inf).all() and got["weights"].numel() == 0


def test_step_agrees_with_the_last_row_of_a_prompt(lap):
    gen = torch.Generator().manual_seed(3)
    q, k, v = rows(gen, 2, 8, 300, 128, BF), rows(gen, 2, 2, 300, 128, BF), rows(gen, 2, 2, 300, 128, BF)
    want = ref.Case(q, k, v, causal=True)
    got = lap.attention_step(q[:, :, -1], k, v)
    within(got["out"], want.out[:, :, -1], want.out_bound[:, :, -1], "out")


def test_offsets_beyond_32_bits(lap):
    """Sequences, heads and rows that lie more than 2^32 elements apart."""
    gen = torch.Generator().manual_seed(12)
    d, n = 64, 130
    space = torch.empty(9 << 30, dtype=BF, device="cuda")      # 18 GiB, of which little is touched
    for strides in ((5 << 30, 1 << 20, d, 1), (1 << 20, 5 << 30, d, 1), (1 << 31, d, (1 << 24) - 8, 1)):
        k, v = (space.as_strided((2, 2, n, d), strides, at << 20) for at in (0, 512))
        small = [rows(gen, 2, 2, n, d, BF) for _ in range(2)]
        k.copy_(small[0])
        v.copy_(small[1])
        q, g = rows(gen, 2, 2, n, d, BF), rows(gen, 2, 2, n, d, BF)
        a, b = lap.attention(q, k, v, causal=True), lap.attention(q, *small, causal=True)
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"]), strides
        ga = lap.attention_grad(g, q, k, v, a["out"], a["lse"], causal=True)
        gb = lap.attention_grad(g, q, *small, a["out"], a["lse"], causal=True)
        assert all(torch.equal(ga[x], gb[x]) for x in ga), strides
        zeros = torch.zeros(2, 2, n, device="cuda")
        sa, sb = lap.attention_step(q[:, :, 0], k, v, zeros), lap.attention_step(q[:, :, 0], *small, zeros)
        assert torch.equal(sa["out"], sb["out"]) and torch.equal(sa["weights"], sb["weights"]), strides
        wa, wb = lap.attention_weights(q, k, a["lse"], causal=True), lap.attention_weights(q, small[0], a["lse"], causal=True)
        assert torch.equal(wa["weights"], wb["weights"]), strides


def test_another_stream_and_a_graph(lap):
    """A training step and a decoding step in a graph, replayed with other work in between; each replay against the eager
    result."""
    case = (BF, 128, 4, 2, 300, 300, True, 0, None, None, "bnhd")
    q, k, v, g, mask, _ = make(case)
    before = torch.rand(2, 2, 300, device="cuda")

    def step():
        f = lap.attention(q, k, v, **mask, sync=False)
        b = lap.attention_grad(g, q, k, v, f["out"], f["lse"], **mask, sync=False)
        w = lap.attention_weights(q, k, f["lse"], before=before, **mask, sync=False)
        t = lap.attention_step(q[:, :, 5].contiguous(), k, v, before, sync=False)
        e = lap.cache_evict(k, v, before, 100, 10, sync=False)
        return {**f, **b, **w, **{"t" + n: x for n, x in t.items()}, **{"e" + n: x for n, x in e.items()}}

    want = {n: x.clone() for n, x in step().items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = step()
    assert all(torch.equal(other[n], want[n]) for n in want)
    for _ in range(4):
        for x in held.values():
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[n], want[n]) for n in want)
        again = step()
        torch.cuda.synchronize()
        assert all(torch.equal(again[n], want[n]) for n in want)
