"""Attention within a memory limit, in training and in serving.

Training: the attention of a stack of layers as a trace of variables (Section III-A of the paper), once as it is where the
probabilities are kept for the backward pass and once as it is here.  Both are planned with plan_pool; the second is then
run, forward and backward, with every tensor at its planned offset in one pool.

Serving: a prompt's keys and values go into a cache of a fixed number of slots, those that have received the most attention;
then one token after the other is inserted, in place of the slot of the least weight, and attended.  And into a cache of few
bits: prompts of many lengths packed, then a few tokens at a time behind each.

    python examples/attention_within_a_limit.py
"""
import math
import os
import sys
from types import SimpleNamespace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1903_06631_amd as lap  # noqa: E402
from traces import make_orderings  # noqa: E402

GRANULE = 512


class Recorder:
    """Variables of one iteration: sizes in bytes and the steps from which and up to which they live."""

    def __init__(self):
        self.names, self.sizes, self.allocs, self.frees = [], [], [], []

    def add(self, name, nbytes, alloc, free):
        self.names.append(name)
        self.sizes.append(max(1, -(-int(nbytes) // GRANULE)) * GRANULE)
        self.allocs.append(alloc)
        self.frees.append(free)

    def trace(self, steps):
        u32 = lambda x: np.asarray(x, np.uint32)
        return SimpleNamespace(n_vars=len(self.names), n_steps=steps, size=np.asarray(self.sizes, np.uint64), alloc=u32(self.allocs),
                               free=u32(self.frees), gap_lo=None, gap_hi=None, step_ns=None)


def record(layers, batch, heads, tokens, size, keep_probabilities):
    """Attention alone: layer l runs forward at step l and backward at step 2 layers - 1 - l."""
    r, steps = Recorder(), 2 * layers
    shape, numbers = (batch, heads, tokens, size), batch * heads * tokens * 4
    rows = math.prod(shape) * 2
    ws = [lap.attention_workspace_bytes(call, shape, shape, torch.bfloat16, causal=True) for call in (lap.AT_FORWARD, lap.AT_GRAD)]
    for l in range(layers):
        back = steps - 1 - l
        for name in ("q", "k", "v", "out"):
            r.add(f"{name}{l}", rows, l, back + 1)
        if keep_probabilities:
            r.add(f"scores{l}", rows // size * tokens, l, l + 1)
            r.add(f"p{l}", rows // size * tokens, l, back + 1)
            r.add(f"dp{l}", rows // size * tokens, back, back + 1)
        else:
            r.add(f"lse{l}", numbers, l, back + 1)
            r.add(f"forward ws{l}", ws[0], l, l + 1)
            r.add(f"ws{l}", ws[1], back, back + 1)
        for name in ("dout", "dq", "dk", "dv"):
            r.add(f"{name}{l}", rows, back, min(back + 2, steps))
    return r, r.trace(steps)


def plan(trace, orderings=64):
    """Footprint, peak load and the offset of every variable under the best of the orders."""
    dt = lap.DeviceTrace(trace)
    kinds, seeds = make_orderings(orderings)
    got = lap.plan_pool(dt, kinds, seeds, want_all=False)
    return int(got["best_footprint"].item()), int(lap.load_profile(dt)["peak"].item()), got["best_offsets"].cpu().numpy()


def train(layers=4, batch=2, heads=8, tokens=1024, size=64):
    """Runs the layers' attention inside the planned pool; returns the gradients of every layer and what they are without
    a pool, and the two plans' footprints."""
    kept = plan(record(layers, batch, heads, tokens, size, True)[1])
    recorder, trace = record(layers, batch, heads, tokens, size, False)
    footprint, peak, offsets = plan(trace)
    pool = torch.empty(footprint, dtype=torch.uint8, device="cuda")
    shape = (batch, heads, tokens, size)

    def at(name, dtype=torch.bfloat16, shape=shape):
        i = recorder.names.index(name)
        off = int(offsets[i])
        if dtype is torch.uint8:
            return pool[off:off + recorder.sizes[i]]
        n = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
        return pool[off:off + n].view(dtype).view(shape)

    gen = torch.Generator(device="cuda").manual_seed(1)
    # what the layers around would compute: each layer's q, k, v and the gradient of its output
    given = [[torch.randn(shape, generator=gen, device="cuda").bfloat16() for _ in range(4)] for _ in range(layers)]
    for l in range(layers):
        for name, x in zip("qkv", given[l]):
            at(f"{name}{l}").copy_(x)
        lap.attention(at(f"q{l}"), at(f"k{l}"), at(f"v{l}"), causal=True, sync=False, ws=at(f"forward ws{l}", torch.uint8),
                      out=dict(out=at(f"out{l}"), lse=at(f"lse{l}", torch.float32, shape[:3])))
    grads = []
    for l in reversed(range(layers)):
        at(f"dout{l}").copy_(given[l][3])
        g = lap.attention_grad(at(f"dout{l}"), at(f"q{l}"), at(f"k{l}"), at(f"v{l}"), at(f"out{l}"), at(f"lse{l}", torch.float32, shape[:3]),
                               causal=True, sync=False, grads={n: at(f"{n}{l}") for n in ("dq", "dk", "dv")}, ws=at(f"ws{l}", torch.uint8))
        grads.append({n: x.clone() for n, x in g.items()})      # the optimiser's use of them, before their memory is given on
    alone = []
    for q, k, v, dout in reversed(given):
        f = lap.attention(q, k, v, causal=True, sync=False)
        alone.append(lap.attention_grad(dout, q, k, v, f["out"], f["lse"], causal=True, sync=False))
    torch.cuda.synchronize()
    return grads, alone, dict(footprint=footprint, peak=peak, footprint_kept=kept[0], peak_kept=kept[1])


def serve(batch=2, heads=8, kv_heads=2, prompt=1500, slots=256, recent=64, new=40, size=64):
    """One layer of a prompt and `new` tokens; returns the last token's output from the cache and from all keys."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    rows = lambda h, n: torch.randn(batch, h, n, size, generator=gen, device="cuda").bfloat16()
    q, k, v = rows(heads, prompt + new), rows(kv_heads, prompt + new), rows(kv_heads, prompt + new)
    # a few keys that most queries look at, as trained models have them
    common = torch.randn(size, generator=gen, device="cuda").bfloat16()
    q += 0.75 * common
    k[:, :, torch.randint(0, prompt, (12,), generator=gen, device="cuda")] += 1.25 * common
    pq, pk, pv = (x[:, :, :prompt] for x in (q, k, v))
    first = lap.attention(pq, pk, pv, causal=True, sync=False)
    weights = lap.attention_weights(pq, pk, first["lse"], causal=True, sync=False)["weights"]
    cache = lap.cache_evict(pk, pv, weights, slots, recent, sync=False)
    position = torch.full((batch,), prompt, dtype=torch.int32, device="cuda")
    for t in range(prompt, prompt + new):
        lap.cache_insert(k[:, :, t], v[:, :, t], cache["k"], cache["v"], cache["weights"], cache["positions"], position, recent, sync=False)
        step = lap.attention_step(q[:, :, t].contiguous(), cache["k"], cache["v"], cache["weights"], positions=cache["positions"], sync=False)
        cache["weights"] = step["weights"]
        position += 1
    full = lap.attention_step(q[:, :, -1].contiguous(), k, v)
    torch.cuda.synchronize()
    return step["out"], full["out"], cache, k.shape[2]


def serve_packed(bits=4, lengths=(1500, 40, 700), heads=8, kv_heads=2, slots=1600, new=(1, 1, 3, 1), size=128):
    """One layer of a ragged batch of prompts and of tokens in a packed cache; returns the last tokens' output from it, from the
    numbers that its rows stand for and from the numbers that were packed, and the bytes of the cache and of one in 16 bits."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    batch = len(lengths)
    rows = lambda h, n: torch.randn(batch, h, n, size, generator=gen, device="cuda").bfloat16()
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    k, v = rows(kv_heads, max(lengths)), rows(kv_heads, max(lengths))
    cache = lap.cache_pack(k, v, bits, slots=slots, lens=lens, sync=False)
    plain = [torch.zeros(batch, kv_heads, slots, size, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for full, x in zip(plain, (k, v)):
        full[:, :, :x.shape[2]] = x
    for tokens in new:
        k, v = rows(kv_heads, tokens), rows(kv_heads, tokens)
        lap.cache_pack(k, v, first=lens, out=cache, sync=False)
        at = (lens.long()[:, None] + torch.arange(tokens, device="cuda"))[:, None, :, None].expand(-1, kv_heads, -1, size)
        for full, x in zip(plain, (k, v)):
            full.scatter_(2, at, x)
        lens += tokens
        q = rows(heads, tokens)
        out = lap.attention_step_packed(q, cache["k"], cache["v"], lens=lens, sync=False)["out"]
    held = lap.cache_unpack(cache["k"], cache["v"], q.dtype, size, lens=lens, sync=False)
    from_held = lap.attention(q, held["k"], held["v"], causal=True, k_lens=lens, sync=False)["out"]
    from_all = lap.attention(q, *plain, causal=True, k_lens=lens)["out"]
    return out, from_held, from_all, 2 * cache["k"].numel(), 4 * plain[0].numel()


def main():
    grads, alone, plans = train()
    same = all(torch.equal(a[n], b[n]) for a, b in zip(grads, alone) for n in a)
    mib = lambda x: f"{x / 2 ** 20:.1f} MiB"
    print(f"training: pool of {mib(plans['footprint'])} (peak load {mib(plans['peak'])}); with kept probabilities "
          f"{mib(plans['footprint_kept'])}; gradients in the pool equal those outside: {same}")
    out, full, cache, tokens = serve()
    err = float((out.float() - full.float()).norm() / full.float().norm())
    print(f"serving: {cache['k'].shape[2]} slots in place of {tokens}; the last token's output differs from full attention's by {err:.2f} of its norm")
    for bits in (4, 8):
        out, _, full, packed, plain = serve_packed(bits)
        err = float((out.float() - full.float()).norm() / full.float().norm())
        print(f"serving: {mib(packed)} in {bits} bits in place of {mib(plain)}; the last tokens' outputs differ from those of all 16 bits by {err:.3f} of their norm")


if __name__ == "__main__":
    main()
