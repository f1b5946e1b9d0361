"""Attention of new tokens over a packed cache against 64 bits on the numbers that its rows stand for: every element within a
bound that follows from the roundings (attention_ref.py).  Slots past the lengths hold bytes that stand for no numbers."""
import math
import warnings

import pytest
import torch

import attention_ref as ref
import packed_ref
from test_gpu_attention import BF, HF, lens_tensor, rows, within
from test_gpu_cache_pack import empty_cache, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


def make(lap, gen, b, h, n, d, kind, bits, lens=None, layout="bhnr", numbers=None):
    """A cache of normal rows, all ones in its other slots (lo and step are not numbers), and what it stands for (of the first
    `numbers` sequences)."""
    row = packed_ref.row_bytes(d, bits)
    out = dict(k=empty_cache(b, h, n, row, layout), v=empty_cache(b, h, n, row, layout))
    for x in out.values():
        x.fill_(255)
    made = torch.Generator(device="cuda").manual_seed(n + d)
    k, v = (torch.randn(b, h, n, d, generator=made, device="cuda").to(kind) for _ in range(2))
    lap.cache_pack(k, v, lens=lens_tensor(lens), out=out)
    return out["k"], out["v"], packed_ref.unpack(out["k"][:numbers], kind, d, bits), packed_ref.unpack(out["v"][:numbers], kind, d, bits)


def check(got, want, weights, shape):
    """A Case's row results, [b, h, tokens, ...], against a call's."""
    within(got["lse"].view(shape[:3]), want.lse, want.lse_bound, "lse")
    within(got["out"].view(shape), want.out, want.out_bound, "out")
    if weights is not None:
        value, bound = want.weights()
        # the sum with what was there before is rounded once
        within(got["weights"], weights.cpu().double() + value, bound + 1e-6 * (1 + weights.cpu().double().abs()), "weights")


# type, bits, head size, query heads, key heads, slots, tokens, lengths, tokens in use, weights, layout
CASES = [
    (BF, 4, 128, 1, 1, 1, 1, None, None, True, "bhnr"),
    (HF, 4, 128, 4, 2, 33, 1, None, None, True, "bnhr"),
    (BF, 8, 128, 8, 2, 500, 1, [500, 0, 31], None, True, "bhnr"),
    (HF, 8, 64, 6, 3, 257, 1, [257, 1, 999], None, True, "gaps"),          # lengths out of range count as none and all
    (BF, 4, 64, 16, 1, 1000, 1, [-7, 1000, 64], None, True, "bhnr"),
    (HF, 4, 64, 32, 1, 300, 1, None, None, True, "bhnr"),                  # two blocks of 16 rows
    (BF, 8, 80, 21, 1, 129, 1, None, None, False, "gaps"),
    (HF, 4, 96, 70, 1, 200, 1, [200, 3], None, True, "bhnr"),              # more than a workgroup's rows
    (BF, 4, 8, 4, 2, 65, 1, None, None, True, "bhnr"),
    (HF, 8, 24, 4, 4, 97, 1, None, None, True, "bhnr"),
    (BF, 4, 40, 2, 1, 64, 1, None, None, True, "gaps"),
    (HF, 4, 120, 256, 1, 77, 1, None, None, True, "bhnr"),
    (BF, 8, 104, 3, 3, 31, 1, None, None, False, "bhnr"),
    # long: in chunks, joined
    (BF, 4, 128, 8, 2, 4999, 1, [4999, 2100, 0], None, True, "bhnr"),
    (HF, 8, 128, 2, 2, 3001, 1, None, None, True, "bnhr"),
    (HF, 4, 64, 24, 1, 5000, 1, [5000, 17], None, True, "gaps"),
    (BF, 8, 64, 1, 1, 2500, 1, None, None, False, "bhnr"),
    (HF, 8, 72, 40, 1, 2600, 1, [2600, 2599], None, True, "bhnr"),
    # several tokens
    (BF, 4, 128, 8, 2, 300, 3, None, None, True, "bhnr"),
    (HF, 4, 64, 4, 1, 290, 5, [290, 3, 0, 288], None, True, "bhnr"),       # fewer slots than tokens
    (BF, 8, 128, 2, 2, 70, 8, [70, 64, 1, 33], [8, 1, 3, 0], True, "gaps"),
    (HF, 8, 80, 32, 4, 1500, 2, [1500, 1499], [2, 1], True, "bhnr"),
    (BF, 4, 64, 7, 1, 4100, 6, [4100, 4097, 4], [6, 5, 6], True, "bhnr"),
    (HF, 4, 128, 1, 1, 40, 64, None, None, False, "bhnr"),                 # more tokens than slots
    (BF, 8, 128, 16, 1, 2305, 16, [2305, 2304], [16, 9], True, "bhnr"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_step(lap, case):
    kind, bits, d, h, kv, n, tokens, lens, q_lens, with_weights, layout = case
    b = 2 if lens is None else len(lens)
    gen = torch.Generator().manual_seed(n + d + tokens)
    k, v, kn, vn = make(lap, gen, b, kv, n, d, kind, bits, lens, layout)
    q = rows(gen, b, h, tokens, d, kind, q_lens, "gaps" if layout == "gaps" else "bnhd", 1.5)
    w = torch.rand(b, kv, n, generator=gen).cuda() if with_weights else None
    want = ref.Case(q, kn, vn, causal=True, q_lens=q_lens, k_lens=lens)
    got = lap.attention_step_packed(q if tokens > 1 else q[:, :, 0], k, v, w, lens=lens_tensor(lens), q_lens=lens_tensor(q_lens))
    assert got["lse"].shape == ((b, h, tokens) if tokens > 1 else (b, h)) and (got["weights"] is None) == (w is None)
    check(got, want, w, (b, h, tokens, d))
    again = lap.attention_step_packed(q if tokens > 1 else q[:, :, 0], k, v, w, lens=lens_tensor(lens), q_lens=lens_tensor(q_lens))
    assert all(x is None or torch.equal(x.nan_to_num(), again[name].nan_to_num()) for name, x in got.items())


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [56, 128])
@pytest.mark.parametrize("group", [4, 32])
@pytest.mark.parametrize("b,kv,n", [(3, 2, 180), (3, 2, 1020), (64, 2, 1600), (2, 1, 4200), (65, 4, 4100)])
def test_forms(lap, b, kv, n, group, d, bits, kind):
    """Every form that the sharing rule chooses, at both widths and both numbers of rows: one workgroup for a cache, its scores in LDS or
    not, and chunks, of few caches and of many."""
    h = kv * group
    gen = torch.Generator().manual_seed(d + group)
    lens = [n - 37 * (i % 7) for i in range(b)]
    k, v, kn, vn = make(lap, gen, b, kv, n, d, kind, bits, lens, numbers=1)
    q = rows(gen, b, h, 1, d, kind, times=1.5)
    w = torch.rand(b, kv, n, device="cuda")
    got = lap.attention_step_packed(q[:, :, 0], k, v, w, lens=lens_tensor(lens))
    # 64 bits on the CPU take their time: one sequence
    want = ref.Case(q[:1], kn, vn, causal=True, k_lens=lens[:1])
    check({name: x[:1] for name, x in got.items()}, want, w[:1], (1, h, 1, d))
    # the others: the same numbers through the call on rows of 16 bits, which is within the same bounds of the truth
    full = lap.cache_unpack(k, v, kind, d, lens=lens_tensor(lens))
    plain = lap.attention_step(q[:, :, 0], full["k"], full["v"], w, lens=lens_tensor(lens))
    assert torch.allclose(got["lse"], plain["lse"], rtol=1e-5, atol=1e-4)
    assert torch.allclose(got["weights"], plain["weights"], rtol=1e-4, atol=1e-4)
    assert torch.allclose(got["out"].float(), plain["out"].float(), rtol=2 ** -6, atol=2 ** -6)


@pytest.mark.parametrize("b,lens", [
    (3, "none"), (3, "equal"), (3, "empty"), (5, "one long"), (65, "mixed"), (130, "mixed"), (130, "one long"), (64, "short"), (200, "empty")])
@pytest.mark.parametrize("heads,kv,tokens,d,bits,kind", [(8, 2, 1, 64, 4, BF), (2, 1, 3, 128, 8, HF), (40, 1, 1, 48, 4, HF)])
def test_chunks_of_sequences(lap, heads, kv, tokens, d, bits, kind, b, lens):
    """Caches in chunks, shared out on the GPU by the lengths: more sequences than a wave has lanes, none with slots, all of the slots in
    one; against the call on rows of 16 bits, and 64 bits for the longest one.  Equal calls give equal bits."""
    n = 1700
    gen = torch.Generator().manual_seed(b)
    of = {"none": None, "equal": [n] * b, "empty": [0] * b, "short": [1 + i % 40 for i in range(b)],
          "one long": [n if i == b // 2 else 0 for i in range(b)],
          "mixed": [[0, -5, 31, n + 100, 700, 1, n - 1, 33][i % 8] for i in range(b)]}[lens]
    k, v, _, _ = make(lap, gen, b, kv, n, d, kind, bits, of, numbers=0)
    q = rows(gen, b, heads, tokens, d, kind, times=1.5)
    w = torch.rand(b, kv, n, device="cuda")
    q1 = q if tokens > 1 else q[:, :, 0]
    got = lap.attention_step_packed(q1, k, v, w, lens=lens_tensor(of))
    again = lap.attention_step_packed(q1, k, v, w, lens=lens_tensor(of))
    assert all(torch.equal(got[x], again[x]) for x in got)
    full = lap.cache_unpack(k, v, kind, d, lens=lens_tensor(of))
    plain = lap.attention(q, full["k"], full["v"], causal=True, k_lens=lens_tensor(of))
    added = lap.attention_weights(q, full["k"], plain["lse"], before=w, causal=True, k_lens=lens_tensor(of))["weights"]
    lse, out = got["lse"].view(plain["lse"].shape), got["out"].view(q.shape)
    assert torch.equal(lse.isneginf(), plain["lse"].isneginf())
    assert torch.allclose(lse, plain["lse"], rtol=1e-5, atol=1e-4)
    assert torch.allclose(out.float(), plain["out"].float(), rtol=2 ** -6, atol=2 ** -6)
    assert torch.allclose(got["weights"], added, rtol=1e-4, atol=1e-4)
    i = 0 if of is None else max(range(b), key=lambda j: min(of[j], n))
    want = ref.Case(q[i:i + 1], full["k"][i:i + 1], full["v"][i:i + 1], causal=True, k_lens=None if of is None else [of[i]])
    check({name: x[i:i + 1] for name, x in got.items()}, want, w[i:i + 1], (1, heads, tokens, d))


def test_lengths_that_grow_between_replays(lap):
    """A captured step reads its lengths when it is replayed."""
    gen = torch.Generator().manual_seed(7)
    b, n = 6, 3000
    k, v, _, _ = make(lap, gen, b, 2, n, 128, BF, 4, numbers=0)
    q, w, lens = rows(gen, b, 8, 1, 128, BF)[:, :, 0].contiguous(), torch.zeros(b, 2, n, device="cuda"), i32([1] * b)
    out = dict(out=torch.empty_like(q), lse=torch.empty(b, 8, device="cuda"), weights=torch.empty_like(w))
    ws = torch.empty(lap.attention_workspace_bytes(lap.AT_STEP_PACKED, q.shape, (b, 2, n, 128), BF), dtype=torch.uint8, device="cuda")
    lap.attention_step_packed(q, k, v, w, lens=lens, out=out, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lap.attention_step_packed(q, k, v, w, lens=lens, out=out, ws=ws, sync=False)
    for turn in ([1, 2, 3, 4, 5, 6], [0, 3000, 0, 17, 2999, 1000], [3000] * 6, [0] * 6, [5, 0, 0, 0, 0, 2500]):
        lens.copy_(i32(turn))
        graph.replay()
        torch.cuda.synchronize()
        eager = lap.attention_step_packed(q, k, v, w, lens=lens)
        assert all(torch.equal(out[x], eager[x]) for x in out), turn


@pytest.mark.parametrize("kind,bits,d,group,n", [(BF, 4, 64, 4, 700), (HF, 8, 128, 1, 90), (HF, 4, 128, 32, 2047), (BF, 8, 96, 9, 5001)])
def test_positions(lap, kind, bits, d, group, n):
    """Empty slots by their positions, all of a head's among them; what they hold is not a number."""
    b, kv = 2, 2
    gen = torch.Generator().manual_seed(n)
    k, v, kn, vn = make(lap, gen, b, kv, n, d, kind, bits)
    pos = torch.stack([torch.stack([torch.randperm(n, generator=gen) for _ in range(kv)]) for _ in range(b)]).int()
    pos[torch.rand(b, kv, n, generator=gen) < 0.4] = -1
    pos[1, 0] = -1
    pos[0, 1, 32:64] = -3
    for x in (k, v):
        x[(pos < 0).cuda()] = 255
    lens = [n, n - 11]
    q = rows(gen, b, kv * group, 1, d, kind, times=1.5)
    w = torch.rand(b, kv, n, generator=gen).cuda()
    got = lap.attention_step_packed(q[:, :, 0], k, v, w, lens=lens_tensor(lens), positions=pos.cuda())
    for i in range(b):
        for j in range(kv):
            at = (pos[i, j, :lens[i]] >= 0).nonzero().flatten()
            heads = slice(j * group, (j + 1) * group)
            want = ref.Case(q[i:i + 1, heads], kn[i:i + 1, j:j + 1, at], vn[i:i + 1, j:j + 1, at], causal=True)
            added = torch.zeros(n, dtype=torch.float64)
            part = {name: x[i:i + 1, heads] for name, x in got.items() if name != "weights"}
            check(part, want, None, (1, group, 1, d))
            value, bound = want.weights()
            added[at] = value[0, 0]
            off = torch.zeros(n, dtype=torch.float64)
            off[at] = bound[0, 0]
            was = w[i, j].cpu().double()
            within(got["weights"][i, j], was + added, off + 1e-6 * (1 + was), "weights")
    assert (got["out"][1, :group] == 0).all() and torch.isneginf(got["lse"][1, :group]).all()


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("d,bits", [(64, 4), (128, 8), (80, 4)])
def test_what_is_not_a_number_reaches_the_rows_that_see_it(lap, d, bits, kind):
    """A group of a value: its 32 elements of the rows that see the slot.  Of a key: those rows."""
    gen = torch.Generator().manual_seed(d)
    n, tokens, h, kv = 200, 5, 4, 2
    k0, v0 = (torch.randn(1, kv, n, d, generator=gen).to(kind) for _ in range(2))
    q = rows(gen, 1, h, tokens, d, kind)
    good = lap.cache_pack(k0.cuda(), v0.cuda(), bits)
    fine = lap.attention_step_packed(q, good["k"], good["v"])
    for slot in (n - 2, n - 5, n - 4, 60):
        bad = v0.clone()
        bad[0, 1, slot, 33] = math.inf
        c = lap.cache_pack(k0.cuda(), bad.cuda(), bits)
        got = lap.attention_step_packed(q, c["k"], c["v"])
        sees = torch.arange(tokens) + n - tokens >= slot
        out = got["out"].cpu()
        assert torch.equal(out[:, :2], fine["out"][:, :2].cpu()) and torch.equal(got["lse"], fine["lse"])
        group = torch.arange(d) // 32 == 1
        for t in range(tokens):
            row = out[0, 2:, t]
            assert torch.equal(row.isnan(), (group & sees[t]).expand(2, d)), (slot, t)
            assert torch.equal(row[:, ~group], fine["out"][0, 2:, t].cpu()[:, ~group])
            if not sees[t]:
                assert torch.allclose(row.float(), fine["out"][0, 2:, t].cpu().float(), rtol=2 ** -6, atol=2 ** -6)
        bad = k0.clone()
        bad[0, 0, slot, 2] = math.nan
        c = lap.cache_pack(bad.cuda(), v0.cuda(), bits)
        got = lap.attention_step_packed(q, c["k"], c["v"], torch.zeros(1, kv, n, device="cuda"))
        assert torch.equal(got["out"][:, 2:], fine["out"][:, 2:]) and not got["weights"][:, 1].isnan().any()
        for t in range(tokens):
            assert got["out"][0, :2, t].isnan().all() == bool(sees[t]) and got["lse"][0, :2, t].isnan().all() == bool(sees[t])
            if not sees[t]:
                assert torch.equal(got["out"][0, :2, t], fine["out"][0, :2, t])
    # rows that are not in use see nothing
    bad = v0.clone()
    bad[0, :, 3] = math.nan
    c = lap.cache_pack(k0.cuda(), bad.cuda(), bits)
    got = lap.attention_step_packed(q, c["k"], c["v"], torch.zeros(1, kv, n, device="cuda"), q_lens=i32([2]))
    assert got["out"][0, :, :2].isnan().all() and (got["out"][0, :, 2:] == 0).all() and torch.isneginf(got["lse"][0, :, 2:]).all()
    assert not got["weights"].isnan().any()


@pytest.mark.parametrize("kind", [BF, HF])
def test_large_scores_and_scales(lap, kind):
    """One slot takes all; a scale of its own; scores below what counts as hidden."""
    gen = torch.Generator().manual_seed(3)
    k, v, kn, vn = make(lap, gen, 2, 2, 400, 64, kind, 4)
    for scale, times in ((3.0, 4.0), (1e-4, 1.0), (0.125, 30.0)):
        q = rows(gen, 2, 4, 3, 64, kind, times=times)
        want = ref.Case(q, kn, vn, causal=True, scale=scale)
        check(lap.attention_step_packed(q, k, v, scale=scale), want, None, (2, 4, 3, 64))
    if kind is BF:
        x = torch.full((1, 1, 40, 64), -1e28).bfloat16().cuda()
        x[:, :, 7] = 1.0
        c = lap.cache_pack(x, x.abs().clamp(max=3), 8)
        got = lap.attention_step_packed(torch.full((1, 1, 64), 100.0).bfloat16().cuda(), c["k"], c["v"])
        assert (got["out"] == 1).all()
        got = lap.attention_step_packed(torch.full((1, 1, 64), 100.0).bfloat16().cuda(), c["k"], c["v"], lens=i32([7]))
        assert (got["out"] == 0).all() and torch.isneginf(got["lse"]).all()


def test_without_slots(lap):
    c = torch.zeros(2, 2, 0, 80, dtype=torch.uint8, device="cuda")
    q = torch.ones(2, 4, 128, device="cuda").half()
    got = lap.attention_step_packed(q, c, c, torch.zeros(2, 2, 0, device="cuda"))
    assert (got["out"] == 0).all() and torch.isneginf(got["lse"]).all() and got["weights"].shape == (2, 2, 0)


def test_offsets_beyond_32_bits(lap):
    n, far, d = 300, 1 << 24, 128
    gen = torch.Generator().manual_seed(1)
    k, v = (torch.randn(2, 1, n, d, generator=gen).bfloat16().cuda() for _ in range(2))
    near = lap.cache_pack(k, v, 4)
    raw = torch.empty(((n - 1) * far + 4096,), dtype=torch.uint8, device="cuda")
    cache = {name: torch.as_strided(raw, (2, 1, n, 80), (512, 512, far, 1), at) for name, at in (("k", 0), ("v", 2048))}
    lap.cache_pack(k, v, out=cache)
    q = rows(gen, 2, 4, 3, d, BF)
    for lens in (None, i32([299, 45])):
        a, b = lap.attention_step_packed(q, cache["k"], cache["v"], lens=lens), lap.attention_step_packed(q, near["k"], near["v"], lens=lens)
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("n,tokens", [(900, 1), (6000, 1), (6000, 3)])
def test_streams_graphs_and_workspaces(lap, n, tokens):
    """Two calls at once with workspaces of their own, in place of the weights before, and captured: replays with eager work
    between them, every one equal to the eager call."""
    gen = torch.Generator().manual_seed(n)
    c = [make(lap, gen, 2, 2, n, 128, BF, 4)[:2] for _ in range(2)]
    q = [rows(gen, 2, 8, tokens, 128, BF, times=1.5) for _ in range(2)]
    w = [torch.rand(2, 2, n, generator=gen).cuda() for _ in range(2)]
    want = [lap.attention_step_packed(q[i], *c[i], w[i]) for i in range(2)]
    need = lap.attention_workspace_bytes(lap.AT_STEP_PACKED, q[0].shape, (2, 2, n, 128), BF)
    ws = [torch.empty(need + 256, dtype=torch.uint8, device="cuda") for _ in range(2)]
    out = [dict(out=torch.empty_like(q[i]), lse=torch.empty(2, 8, tokens, device="cuda"), weights=w[i].clone()) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            lap.attention_step_packed(q[i], *c[i], out[i]["weights"], out=out[i], ws=ws[i], sync=False)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(out[i][x], want[i][x]) for x in ("out", "lse", "weights")), i
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in range(2):      # one after the other in one workspace
            lap.attention_step_packed(q[i], *c[i], w[i], out=out[i], ws=ws[0], sync=False)
    for turn in range(4):
        for x in q:
            x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for i in range(2):
            eager = lap.attention_step_packed(q[i], *c[i], w[i])
            assert all(torch.equal(out[i][x], eager[x]) for x in ("out", "lse", "weights")), (turn, i)


def test_refusals(lap):
    x = torch.ones(2, 2, 16, 64, device="cuda").bfloat16()
    c = lap.cache_pack(x, x, 4)
    k, v = c["k"], c["v"]
    q, w = torch.ones(2, 4, 64, device="cuda").bfloat16(), torch.ones(2, 2, 16, device="cuda")
    three = q[:, :, None].expand(2, 4, 3, 64).contiguous()
    step = lap.attention_step_packed
    for call in (lambda: step(q[0], k, v), lambda: step(q.cpu(), k, v), lambda: step(q.float(), k, v), lambda: step(q, k[0], v[0]), lambda: step(q, k[:1], v[:1]),
                 lambda: step(q, k, v[:, :, :8]), lambda: step(q, k.view(torch.int8), v), lambda: step(q, k[..., :32], v[..., :32]), lambda: step(q, k, v, w[..., :8]),
                 lambda: step(q, k, v, w.half()), lambda: step(q, k, v, positions=torch.zeros(2, 2, 16, dtype=torch.int64, device="cuda")),
                 lambda: step(q, k, v, lens=i32([1])), lambda: step(three, k, v, q_lens=i32([1, 2, 3])), lambda: step(torch.ones(2, 4, 72, device="cuda").bfloat16(), k, v),
                 lambda: step(q, k, v, ws=torch.zeros(64, device="cuda")), lambda: step(q, k, v, out=dict(out=q.half(), lse=w[:, 0, :4].contiguous()))):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: step(three, k, v, positions=torch.zeros(2, 2, 16, dtype=torch.int32, device="cuda")), -9), (lambda: step(q, k, v, scale=0.0), -9),
                       (lambda: step(torch.ones(2, 3, 64, device="cuda").bfloat16(), k, v), -9), (lambda: step(q[:, :, None].expand(2, 4, 200, 64), k, v), -2),
                       (lambda: step(q[:, :, None][:, :, :0], k, v), -9),
                       (lambda: step(q, k, v, w, out=dict(out=torch.empty_like(q), lse=torch.empty(2, 4, device="cuda"))), -1)):
        with pytest.raises(lap.LapError) as e:
            call()
        assert e.value.status == code
    with pytest.warns(UserWarning):
        step(q.clone().requires_grad_(), k, v)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        step(q, k, v)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("kind", [BF, HF])
def test_serving(lap, kind, bits):
    """A ragged batch of prompts packed, then tokens one by one and a few at once, as a server does, beside the numbers that the rows
    stand for in a cache of 16 bits."""
    gen = torch.Generator().manual_seed(bits)
    b, kv, h, d, slots = 3, 2, 8, 128, 150
    lens = i32([100, 1, 37])
    rows_of = lambda heads, n: torch.randn(b, heads, n, d, generator=gen).to(kind).cuda()
    k, v = rows_of(kv, 100), rows_of(kv, 100)
    cache = lap.cache_pack(k, v, bits, slots=slots, lens=lens)
    weights = torch.zeros(b, kv, slots, device="cuda")
    for new in (1, 1, 4, 1, 3, 2):
        kn, vn = rows_of(kv, new), rows_of(kv, new)
        lap.cache_pack(kn, vn, first=lens, out=cache, sync=False)
        lens += new
        q = rows_of(h, new)
        got = lap.attention_step_packed(q, cache["k"], cache["v"], weights, lens=lens, sync=False)
        full = lap.cache_unpack(cache["k"], cache["v"], kind, d, lens=lens)
        plain = lap.attention(q, full["k"], full["v"], causal=True, k_lens=lens)
        want = ref.Case(q, full["k"], full["v"], causal=True, k_lens=lens.tolist())
        within(got["out"], want.out, want.out_bound, "out")
        within(plain["out"], want.out, want.out_bound, "plain")
        added = lap.attention_weights(q, full["k"], plain["lse"], before=weights, causal=True, k_lens=lens)["weights"]
        assert torch.allclose(got["weights"], added, rtol=1e-4, atol=1e-4)
        weights = got["weights"]


@pytest.mark.parametrize("bits", [4, 8])
def test_a_packed_cache_held_to_a_number_of_slots(lap, bits):
    """Eviction, insertion and steps on packed rows choose and move what they do on rows of 16 bits."""
    gen = torch.Generator().manual_seed(bits)
    b, kv, h, d, n, keep, recent = 2, 2, 8, 80, 300, 64, 9
    k, v = (torch.randn(b, kv, n, d, generator=gen).bfloat16().cuda() for _ in range(2))
    w = torch.rand(b, kv, n, generator=gen).cuda()
    packed = lap.cache_pack(k, v, bits)
    small = lap.cache_evict(packed["k"], packed["v"], w, keep, recent, lens=i32([300, 40]))
    plain = lap.cache_evict(k, v, w, keep, recent, lens=i32([300, 40]))
    assert all(torch.equal(small[x], plain[x]) for x in ("positions", "weights", "lens"))
    again = lap.cache_pack(plain["k"], plain["v"], bits)
    used = plain["positions"] >= 0
    assert torch.equal(small["k"][used], again["k"][used]) and torch.equal(small["v"][used], again["v"][used]) and not small["k"][~used].any()
    position = i32([300, 40])
    for t in range(30):
        new = [torch.randn(b, kv, 1, d, generator=gen).bfloat16().cuda() for _ in range(2)]
        one = lap.cache_pack(*new, bits)
        a = lap.cache_insert(one["k"][:, :, 0], one["v"][:, :, 0], small["k"], small["v"], small["weights"], small["positions"], position, recent)
        c = lap.cache_insert(new[0][:, :, 0], new[1][:, :, 0], plain["k"], plain["v"], plain["weights"], plain["positions"], position, recent)
        assert torch.equal(a["slots"], c["slots"])
        q = torch.randn(b, h, d, generator=gen).bfloat16().cuda()
        got = lap.attention_step_packed(q, small["k"], small["v"], small["weights"], positions=small["positions"])
        full = lap.cache_unpack(small["k"], small["v"], BF, d)
        want = lap.attention_step(q, full["k"], full["v"], small["weights"], positions=small["positions"])
        assert torch.allclose(got["weights"], want["weights"], rtol=1e-4, atol=1e-4) and torch.allclose(got["lse"], want["lse"], rtol=1e-5, atol=1e-4)
        assert torch.allclose(got["out"].float(), want["out"].float(), rtol=2 ** -6, atol=2 ** -6)
        small["weights"] = got["weights"]
        plain["weights"] = got["weights"].clone()
        position += 1


@pytest.mark.parametrize("kind,bits,d,heads,kv,b,n", [(BF, 4, 16, 8, 8, 8191, 5), (HF, 8, 64, 3, 1, 65535, 3), (BF, 4, 64, 1, 1, 20000, 1100)])
def test_as_many_caches_as_a_call_takes(lap, kind, bits, d, heads, kv, b, n):
    """Each one's results those of a call for it and a few others."""
    gen = torch.Generator(device="cuda").manual_seed(b)
    k, v = (torch.randn(1, kv, n, d, generator=gen, device="cuda").to(kind).expand(b, kv, n, d) for _ in range(2))
    times = torch.rand(b, 1, 1, 1, generator=gen, device="cuda").to(kind)
    held = lap.cache_pack(k * times, v * (1 - times), bits)
    q = torch.randn(b, heads, d, generator=gen, device="cuda").to(kind)
    lens = torch.randint(0, n + 1, (b,), generator=gen, device="cuda").int()
    w = torch.rand(b, kv, n, generator=gen, device="cuda")
    got = lap.attention_step_packed(q, held["k"], held["v"], w, lens=lens)
    for at in (0, b // 2, b - 7):
        one = slice(at, at + 7)
        few = lap.cache_pack((k * times)[one], (v * (1 - times))[one], bits)
        assert torch.equal(few["k"], held["k"][one]) and torch.equal(few["v"], held["v"][one])
        kn, vn = (packed_ref.unpack(few[x], kind, d, bits) for x in "kv")
        want = ref.Case(q[one, :, None], kn, vn, causal=True, k_lens=lens[one].tolist())
        check({name: x[one] for name, x in got.items()}, want, w[one], (7, heads, 1, d))


@pytest.mark.parametrize("b,heads,kv,tokens,d", [(2, 40, 1, 1, 128), (3, 256, 1, 1, 64), (2, 16, 2, 5, 96), (64, 64, 8, 5, 128), (257, 40, 1, 1, 64), (600, 40, 1, 1, 128)])
@pytest.mark.parametrize("lengths", [False, True])
def test_without_slots_and_many_rows(lap, b, heads, kv, tokens, d, lengths):
    """More than 32 rows to a key head, which never have a workgroup for a whole cache: of few key heads and of more than there are places."""
    c = torch.zeros(b, kv, 0, packed_ref.row_bytes(d, 4), dtype=torch.uint8, device="cuda")
    q = torch.ones(b, heads, tokens, d, device="cuda").half()
    lens = i32([i % 3 for i in range(b)]) if lengths else None
    got = lap.attention_step_packed(q, c, c, torch.zeros(b, kv, 0, device="cuda"), lens=lens)
    assert (got["out"] == 0).all() and torch.isneginf(got["lse"]).all() and got["weights"].shape == (b, kv, 0)


@pytest.mark.parametrize("n,heads,tokens", [(900, 8, 1), (1000, 16, 1), (6000, 8, 3), (6000, 80, 1)])
@pytest.mark.parametrize("lengths", [False, True])
def test_workspace_without_weights(lap, n, heads, tokens, lengths):
    """A workspace that just does for a call without weights, and one with room to spare: equal results, and nothing behind it is written."""
    gen = torch.Generator().manual_seed(n)
    b, kv = 3, 2
    k, v, _, _ = make(lap, gen, b, kv, n, 128, BF, 4, numbers=0)
    q = rows(gen, b, heads, tokens, 128, BF, times=1.5)
    lens = i32([n, 0, n // 2]) if lengths else None
    weighted = lap.attention_step_packed(q, k, v, torch.zeros(b, kv, n, device="cuda"), lens=lens)
    need = lap.attention_workspace_bytes(lap.AT_STEP_PACKED_UNWEIGHTED, q.shape, (b, kv, n, 128), BF)
    whole = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    for ws in (whole[:need], None):
        got = lap.attention_step_packed(q, k, v, lens=lens, ws=ws)
        assert torch.equal(got["out"], weighted["out"]) and torch.equal(got["lse"], weighted["lse"])
    assert (whole[need:] == 0xA5).all()
    if need:
        with pytest.raises(lap.LapError):
            lap.attention_step_packed(q, k, v, lens=lens, ws=whole[:need - 256])
