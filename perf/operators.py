"""Performance cases of the attention operators and of the cache they read, in training and in serving.

One case is one pass through one operator on tensors that are resident on the GPU:

  forward  attention of a training step or a prompt: output rows and the logarithms of the softmax sums
  grad     its backward pass from the output's gradient, the probabilities recomputed
  weights  the attention weight that every key of a prompt has received
  step     one new token of every sequence against the cache, adding its weights to those of the slots
  evict    a prompt's keys and values into a cache of fewer slots, those of the highest weight
  insert   one new token into every full cache, in the place of the slot of the lowest weight

Tensors are [batch, heads, length, head size].  Query heads share key/value heads in equal groups, queries are aligned to
the end of the keys, and rows beyond a sequence's length are padding.  `run` makes one pass: plain torch operations in 32
bits, or with `own` the calls of the framework.
"""
import math
from types import SimpleNamespace

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
MINUS_INF = float("-inf")


def listed():
    return [
        # a short encoder-like call, where launches and latency count: odd length, every key visible
        dict(name="forward-short", op="forward", batch=2, heads=16, kv_heads=16, queries=77, keys=77, size=64, type="f16",
             causal=False, window=0, ragged=False),
        # one layer of the transformer that the traces of this repository are shaped like
        dict(name="forward-layer", op="forward", batch=8, heads=16, kv_heads=16, queries=2048, keys=2048, size=128,
             type="bf16", causal=True, window=0, ragged=False),
        # a long prompt behind a cached prefix, shared key heads
        dict(name="forward-long", op="forward", batch=1, heads=32, kv_heads=8, queries=12_345, keys=13_370, size=128,
             type="bf16", causal=True, window=0, ragged=False),
        # a ragged training batch, padded to its longest sequence, one of them empty; a head size that is no power of two
        dict(name="grad-ragged", op="grad", batch=6, heads=12, kv_heads=4, queries=1001, keys=1001, size=80, type="f16",
             causal=True, window=0, ragged=True),
        # the backward pass of that layer
        dict(name="grad-layer", op="grad", batch=8, heads=16, kv_heads=16, queries=2048, keys=2048, size=128, type="bf16",
             causal=True, window=0, ragged=False),
        # short ragged prompts
        dict(name="weights-ragged", op="weights", batch=4, heads=16, kv_heads=16, queries=333, keys=333, size=64, type="f16",
             causal=True, window=0, ragged=True),
        # a long prompt of a model with shared key heads
        dict(name="weights-prompt", op="weights", batch=2, heads=32, kv_heads=8, queries=8192, keys=8192, size=128,
             type="bf16", causal=True, window=0, ragged=False),
        # one user's token: latency counts
        dict(name="step-single", op="step", batch=1, heads=16, kv_heads=16, keys=1000, size=128, type="bf16", ragged=False),
        # a serving batch of sequences of many lengths
        dict(name="step-batch", op="step", batch=64, heads=32, kv_heads=8, keys=4096, size=128, type="bf16", ragged=True),
        # few sequences over a long cache: the work has to be split over its length
        dict(name="step-long", op="step", batch=2, heads=32, kv_heads=8, keys=131_072, size=128, type="f16", ragged=False),
        # long prompts into caches of an eighth of their length
        dict(name="evict-prompt", op="evict", batch=8, kv_heads=8, keys=16_384, keep=2048, recent=256, size=128, type="bf16",
             ragged=True),
        # a serving batch's new tokens into full caches
        dict(name="insert-batch", op="insert", batch=64, kv_heads=8, keep=2048, recent=128, size=128, type="bf16"),
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _no(n):
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["forward", "forward", "grad", "grad", "weights", "step", "step", "evict", "insert"])
    case = dict(op=op, type=rng.choice(["bf16", "f16"]))
    kv = rng.choice([1, 2, 4, 8, 16])
    size = rng.choice([64, 64, 128, 128, 128, 8 * rng.randint(4, 16)])
    if op in ("forward", "grad", "weights"):
        group = rng.choice([1, 1, 2, 4, 8]) if kv < 16 else 1
        heads = kv * group
        causal = rng.random() < 0.75
        # query-key pairs of all heads
        most = {"forward": 2.5e9, "grad": 2.5e8, "weights": 1.2e9}[op] * (2 if causal else 1)
        keys = _no(_between(rng, 33, min(12_345, int(math.sqrt(most / heads)))))
        queries = keys if op == "grad" or rng.random() < 0.6 else _no(_between(rng, max(1, keys // 8), keys))
        batch = _between(rng, 1, max(1, min(32, int(most / (heads * keys * queries)))))
        window = _between(rng, 16, keys) if causal and rng.random() < 0.25 else 0
        case.update(batch=batch, heads=heads, kv_heads=kv, queries=queries, keys=keys, size=size, causal=causal, window=window,
                    ragged=batch > 1 and rng.random() < 0.5)
        return case
    if op == "step":
        keys = _no(_between(rng, 17, 131_072))
        batch = _between(rng, 1, max(1, min(64, 2_000_000 // (keys * kv))))
        case.update(batch=batch, heads=kv * rng.choice([1, 2, 4, 7, 8]), kv_heads=kv, keys=keys, size=size,
                    ragged=batch > 1 and rng.random() < 0.6)
        return case
    if op == "evict":
        keys = _no(_between(rng, 100, 60_000))
        keep = _no(_between(rng, max(2, keys // 32), max(2, min(keys * 3 // 4, 120_000 // kv))))
        batch = _between(rng, 1, max(1, min(16, 800_000 // (keys * kv), 120_000 // (keep * kv))))
        case.update(batch=batch, kv_heads=kv, keys=keys, keep=keep, recent=_between(rng, 1, max(1, keep // 2)), size=size,
                    ragged=batch > 1 and rng.random() < 0.5)
        return case
    keep = _no(_between(rng, 64, 16_384))
    batch = _between(rng, 1, max(1, min(128, 1_000_000 // (keep * kv))))
    case.update(batch=batch, kv_heads=kv, keep=keep, recent=_between(rng, 1, max(1, keep // 2)), size=size)
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _lengths(case, most, none):
    """Lengths of a ragged batch: evenly spread up to the longest, in no order; `none`: one sequence is empty."""
    b = case["batch"]
    if not case.get("ragged"):
        return [most] * b
    spread = [max(1, most * (i + 1) // b) for i in range(b)]
    if none and b > 2:
        spread[0] = 0
    return spread[1::2] + spread[0::2][::-1]


def _scale(case):
    return 1.0 / math.sqrt(case["size"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    b, kv, d = case["batch"], case["kv_heads"], case["size"]
    kind = TYPES[case["type"]]

    def normal(*shape, times=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * times).to(kind)

    def lens(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    s = SimpleNamespace(case=case)
    if case["op"] in ("forward", "grad", "weights"):
        nq, nk = case["queries"], case["keys"]
        s.q = normal(b, case["heads"], nq, d, times=1.5)
        s.k, s.v = normal(b, kv, nk, d), normal(b, kv, nk, d)
        s.k_lens = s.q_lens = None
        if case["ragged"]:
            k_lens = _lengths(case, nk, True)
            s.k_lens, s.q_lens = lens(k_lens), lens([min(nq, x) for x in k_lens])
        if case["op"] != "forward":
            got = _attention(s)
            s.out, s.lse = got["out"], got["lse"]
        if case["op"] == "grad":
            s.dout = normal(b, case["heads"], nq, d)
        return s
    if case["op"] == "step":
        n = case["keys"]
        s.q = normal(b, case["heads"], d, times=1.5)
        s.k, s.v = normal(b, kv, n, d), normal(b, kv, n, d)
        s.lens = lens(_lengths(case, n, False))
        s.weights = torch.rand(b, kv, n, generator=gen, device="cuda") * 4
        return s
    if case["op"] == "evict":
        n = case["keys"]
        s.k, s.v = normal(b, kv, n, d), normal(b, kv, n, d)
        s.lens = lens(_lengths(case, n, True))
        # weights of a prompt: most keys get little, a few get nearly all of it; many of the small ones are equal
        w = torch.rand(b, kv, n, generator=gen, device="cuda").pow(-0.7) * 0.01
        s.weights = torch.where(w < 0.012, torch.zeros_like(w), w)
        return s
    n = case["keep"]
    s.k_cache, s.v_cache = normal(b, kv, n, d), normal(b, kv, n, d)
    s.weights = torch.rand(b, kv, n, generator=gen, device="cuda").pow(-0.7) * 0.01
    # each head has kept positions of its own out of the four times as many that have gone by, and the newest ones
    start = 4 * n
    kept = torch.argsort(torch.rand(b, kv, start - n, generator=gen, device="cuda"), dim=-1)[..., :n]
    slot = torch.arange(n, device="cuda")
    newest = case["recent"]
    s.positions = torch.where(slot < n - newest, kept, start - n + slot).to(torch.int32)
    s.position = torch.full((b,), start, dtype=torch.int32, device="cuda")
    s.k_new, s.v_new = normal(b, kv, d), normal(b, kv, d)
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _grouped(x, kv_heads):
    """[batch, heads, rows, size] -> [batch, kv_heads, group * rows, size] in 32 bits."""
    b, h, n, d = x.shape
    return x.float().reshape(b, kv_heads, (h // kv_heads) * n, d)


def _visible(s):
    """[batch, 1, 1, queries, keys]: which keys a query sees."""
    case = s.case
    nq, nk = case["queries"], case["keys"]
    i = torch.arange(nq, device="cuda").view(1, 1, 1, nq, 1)
    j = torch.arange(nk, device="cuda").view(1, 1, 1, 1, nk)
    full = lambda n: torch.full((case["batch"],), n, dtype=torch.int32, device="cuda")
    kl = (full(nk) if s.k_lens is None else s.k_lens).view(-1, 1, 1, 1, 1)
    ql = (full(nq) if s.q_lens is None else s.q_lens).view(-1, 1, 1, 1, 1)
    seen = (j < kl) & (i < ql)
    if case["causal"]:
        at = i + kl - ql
        seen = seen & (j <= at)
        if case["window"]:
            seen = seen & (j > at - case["window"])
    return seen


def _masked_scores(s, kf):
    case = s.case
    b, kv, nq, nk = case["batch"], case["kv_heads"], case["queries"], case["keys"]
    scores = torch.matmul(_grouped(s.q, kv), kf.transpose(-1, -2)).mul_(_scale(case)).view(b, kv, -1, nq, nk)
    return scores.masked_fill_(~_visible(s), MINUS_INF)


def _attention(s):
    case = s.case
    b, kv, h, nq, nk = case["batch"], case["kv_heads"], case["heads"], case["queries"], case["keys"]
    scores = _masked_scores(s, s.k.float())
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == MINUS_INF, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(b, kv, -1, nk), s.v.float()).view(b, kv, -1, nq, case["size"])
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return dict(out=out.reshape(s.q.shape).to(s.q.dtype), lse=(top + total.log()).view(b, h, nq))


def _probabilities(s, kf):
    case = s.case
    lse = s.lse.view(case["batch"], case["kv_heads"], -1, case["queries"], 1)
    scores = _masked_scores(s, kf)
    return scores.sub_(torch.where(lse == MINUS_INF, torch.zeros_like(lse), lse)).exp_()


def _attention_grad(s):
    case = s.case
    b, kv, nq, nk, d = case["batch"], case["kv_heads"], case["queries"], case["keys"], case["size"]
    kf, vf = s.k.float(), s.v.float()
    qg, dog = _grouped(s.q, kv), _grouped(s.dout, kv)
    p = _probabilities(s, kf).view(b, kv, -1, nk)
    dv = torch.matmul(p.transpose(-1, -2), dog)
    delta = (dog * _grouped(s.out, kv)).sum(-1, keepdim=True)
    ds = torch.matmul(dog, vf.transpose(-1, -2)).sub_(delta).mul_(p).mul_(_scale(case))
    dq = torch.matmul(ds, kf)
    dk = torch.matmul(ds.transpose(-1, -2), qg)
    return dict(dq=dq.view(b, case["heads"], nq, d).to(s.q.dtype), dk=dk.to(s.k.dtype), dv=dv.to(s.v.dtype))


def _attention_weights(s):
    return dict(weights=_probabilities(s, s.k.float()).sum(dim=(2, 3)))


def _attention_step(s):
    case = s.case
    b, kv, n = case["batch"], case["kv_heads"], case["keys"]
    q = s.q.float().view(b, kv, -1, case["size"])
    scores = torch.matmul(q, s.k.float().transpose(-1, -2)).mul_(_scale(case))
    live = torch.arange(n, device="cuda").view(1, 1, 1, n) < s.lens.view(-1, 1, 1, 1)
    scores = scores.masked_fill_(~live, MINUS_INF)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub(top).exp_()
    total = p.sum(-1, keepdim=True)
    p = p / total
    out = torch.matmul(p, s.v.float())
    return dict(out=out.view(s.q.shape).to(s.q.dtype), lse=(top + total.log()).view(b, -1),
                weights=s.weights + p.sum(2))


def _cache_evict(s):
    case = s.case
    n, keep, d = case["keys"], case["keep"], case["size"]
    slot = torch.arange(n, device="cuda").view(1, 1, n)
    lens = s.lens.view(-1, 1, 1)
    # highest first, equal ones in their order: the newest, the others by weight, what is padding last
    rank = torch.where(slot >= lens - case["recent"], torch.full_like(s.weights, math.inf), s.weights)
    rank = torch.where(slot < lens, rank, torch.full_like(rank, MINUS_INF))
    kept = torch.argsort(rank, dim=-1, descending=True, stable=True)[..., :keep].sort(dim=-1).values
    live = kept < lens
    rows = kept.unsqueeze(-1).expand(-1, -1, -1, d)
    k = torch.where(live.unsqueeze(-1), s.k.gather(2, rows), torch.zeros((), dtype=s.k.dtype, device="cuda"))
    v = torch.where(live.unsqueeze(-1), s.v.gather(2, rows), torch.zeros((), dtype=s.v.dtype, device="cuda"))
    return dict(k=k, v=v, weights=torch.where(live, s.weights.gather(2, kept), torch.zeros_like(s.weights[..., :keep])),
                positions=torch.where(live, kept, torch.full_like(kept, -1)).to(torch.int32),
                lens=s.lens.clamp(max=keep))


def _cache_insert(s):
    case = s.case
    n = case["keep"]
    slot = torch.arange(n, device="cuda").view(1, 1, n)
    at = s.position.view(-1, 1, 1)
    newest = s.positions > at - case["recent"]
    rank = torch.where(newest, torch.full_like(s.weights, math.inf), s.weights)
    low = rank.amin(-1, keepdim=True)
    last = torch.where(rank == low, slot, torch.full_like(slot, -1)).amax(-1)
    empty = torch.where(s.positions < 0, slot, torch.full_like(slot, n)).amin(-1)
    chosen = torch.where(empty < n, empty, last).unsqueeze(-1)
    rows = chosen.unsqueeze(-1).expand(-1, -1, 1, case["size"])
    s.k_cache.scatter_(2, rows, s.k_new.unsqueeze(2))
    s.v_cache.scatter_(2, rows, s.v_new.unsqueeze(2))
    s.weights.scatter_(2, chosen, 0.0)
    s.positions.scatter_(2, chosen, at.expand(-1, case["kv_heads"], 1))
    return chosen.squeeze(-1).to(torch.int32)


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(s):
    case = s.case
    op = case["op"]
    if own:
        import paper_1903_06631_amd as lap
        if op in ("forward", "grad", "weights"):
            mask = dict(causal=case["causal"], window=case["window"], q_lens=s.q_lens, k_lens=s.k_lens)
            if op == "forward":
                return lap.attention(s.q, s.k, s.v, **mask, sync=False)
            if op == "grad":
                return lap.attention_grad(s.dout, s.q, s.k, s.v, s.out, s.lse, **mask, sync=False)
            return lap.attention_weights(s.q, s.k, s.lse, **mask, sync=False)
        if op == "step":
            return lap.attention_step(s.q, s.k, s.v, s.weights, lens=s.lens, sync=False)
        if op == "evict":
            return lap.cache_evict(s.k, s.v, s.weights, case["keep"], case["recent"], lens=s.lens, sync=False)
        slots = lap.cache_insert(s.k_new, s.v_new, s.k_cache, s.v_cache, s.weights, s.positions, s.position,
                                 case["recent"], sync=False)["slots"]
    elif op == "insert":
        slots = _cache_insert(s)
    else:
        return {"forward": _attention, "grad": _attention_grad, "weights": _attention_weights, "step": _attention_step,
                "evict": _cache_evict}[op](s)
    s.position.add_(1)      # the next token's
    return dict(slots=slots, k=s.k_cache, v=s.v_cache, weights=s.weights, positions=s.positions)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def _pairs(case):
    """Query-key pairs that are visible, of one head, and the query and key rows in use."""
    nq, nk = case["queries"], case["keys"]
    k_lens = _lengths(case, nk, True)
    pairs = 0
    for kl in k_lens:
        ql = min(nq, kl)
        if not case["causal"]:
            pairs += ql * kl
            continue
        at = torch.arange(ql, dtype=torch.int64) + (kl - ql)
        low = (at - case["window"] + 1).clamp(min=0) if case["window"] else torch.zeros_like(at)
        pairs += int((at + 1 - low).clamp(min=0).sum())
    return pairs, sum(min(nq, kl) for kl in k_lens), sum(k_lens)


def work(case):
    b, kv, d = case["batch"], case["kv_heads"], case["size"]
    if case["op"] in ("forward", "grad", "weights"):
        pairs, rows, keys = _pairs(case)
        h = case["heads"]
        q, o, k = 2 * d * h * rows, 2 * d * h * b * case["queries"], 2 * d * kv * keys
        if case["op"] == "forward":
            return dict(bytes=q + 2 * k + o + 4 * h * b * case["queries"], flops=4 * d * h * pairs)
        if case["op"] == "grad":
            return dict(bytes=3 * q + 2 * k + 4 * h * rows + o + 2 * 2 * d * kv * b * case["keys"], flops=10 * d * h * pairs)
        return dict(bytes=q + k + 4 * h * rows + 4 * kv * b * case["keys"], flops=2 * d * h * pairs)
    if case["op"] == "step":
        h, keys = case["heads"], sum(_lengths(case, case["keys"], False))
        return dict(bytes=4 * d * kv * keys + 4 * d * h * b + 4 * h * b + 8 * kv * b * case["keys"], flops=4 * d * h * keys)
    if case["op"] == "evict":
        lens = _lengths(case, case["keys"], True)
        kept = sum(min(n, case["keep"]) for n in lens)
        return dict(bytes=kv * (4 * sum(lens) + 4 * d * kept + b * case["keep"] * (4 * d + 8)) + 8 * b, flops=kv * sum(lens))
    return dict(bytes=b * kv * (8 * case["keep"] + 8 * d + 12) + 4 * b, flops=b * kv * case["keep"])


# ---- in 64 bits ------------------------------------------------------------------------------------------------------

def exact(case, seed):
    """From the definition in 64 bits, one head and a block of query rows at a time; None where nothing is computed (an
    eviction or insertion chooses and copies)."""
    if case["op"] in ("evict", "insert"):
        return None
    s = prepare(case, seed)
    group = case["heads"] // case["kv_heads"]
    f64 = dict(dtype=torch.float64, device="cuda")
    if case["op"] == "step":
        out, lse = torch.zeros(s.q.shape, **f64), torch.zeros(s.q.shape[:2], **f64)
        weights = s.weights.double()
        for b, n in enumerate(s.lens.tolist()):
            for g in range(case["kv_heads"]):
                rows = slice(g * group, (g + 1) * group)
                e = torch.exp(_scale(case) * torch.mm(s.q[b, rows].double(), s.k[b, g, :n].double().t().contiguous()))
                z = e.sum(1)
                out[b, rows] = torch.mm(e, s.v[b, g, :n].double()) / z[:, None]
                lse[b, rows] = torch.log(z)
                weights[b, g, :n] += (e / z[:, None]).sum(0)
        return dict(out=out, lse=lse, weights=weights)

    nq, nk = case["queries"], case["keys"]
    out, lse = torch.zeros(s.q.shape, **f64), torch.full(s.q.shape[:3], MINUS_INF, **f64)
    dq, dk, dv = torch.zeros(s.q.shape, **f64), torch.zeros(s.k.shape, **f64), torch.zeros(s.k.shape, **f64)
    weights = torch.zeros(s.k.shape[:3], **f64)
    k_lens = [nk] * case["batch"] if s.k_lens is None else s.k_lens.tolist()
    q_lens = [nq] * case["batch"] if s.q_lens is None else s.q_lens.tolist()
    for b, (ql, kl) in enumerate(zip(q_lens, k_lens)):
        for h in range(case["heads"]):
            k = s.k[b, h // group, :kl].double()
            v = s.v[b, h // group, :kl].double()
            for first in range(0, ql, 4096):
                r = slice(first, min(first + 4096, ql))
                q = s.q[b, h, r].double()
                e = torch.exp(_scale(case) * torch.mm(q, k.t().contiguous()))
                if case["causal"]:
                    at = torch.arange(r.start, r.stop, device="cuda")[:, None] + (kl - ql)
                    j = torch.arange(kl, device="cuda")[None, :]
                    hide = j > at
                    if case["window"]:
                        hide |= j <= at - case["window"]
                    e[hide] = 0
                z = e.sum(1)
                some = z > 0
                p = e / torch.where(some, z, torch.ones_like(z))[:, None]
                lse[b, h, r] = torch.where(some, torch.log(z), torch.full_like(z, MINUS_INF))
                if case["op"] == "forward":
                    out[b, h, r] = torch.mm(p, v)
                elif case["op"] == "weights":
                    weights[b, h // group, :kl] += p.sum(0)
                else:
                    do = s.dout[b, h, r].double()
                    dp = torch.mm(do, v.t().contiguous())
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) * _scale(case)
                    dq[b, h, r] = torch.mm(ds, k)
                    dk[b, h // group, :kl] += torch.mm(ds.t().contiguous(), q)
                    dv[b, h // group, :kl] += torch.mm(p.t().contiguous(), do)
    if case["op"] == "forward":
        return dict(out=out, lse=lse)
    if case["op"] == "weights":
        return dict(weights=weights)
    return dict(dq=dq, dk=dk, dv=dv)
