"""Attention, its gradient and the caches' choices in 64 bits on the CPU, one row at a time from the definition, with bounds
on how far a kernel may be off that rounds probabilities and results to the element type and holds the rest in 32 bits.

u is the type's unit roundoff.  A rounded probability is off by at most u of itself, so out is off by u (sum p |v| + |out|);
the other products likewise.  What 32 bits add is a few 2^-24 for each of head_dim products and of the sums' terms (`E`)."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E = 1e-5
TINY = {torch.bfloat16: 1e-30, torch.float16: 2.0 ** -24}      # below binary16's normal range rounding is absolute: half of it


def visible(nq, nk, ql, kl, causal, window):
    """[nq, nk] truth values."""
    i, j = torch.arange(nq)[:, None], torch.arange(nk)[None, :]
    see = (i < ql) & (j < kl)
    if causal:
        at = i + kl - ql
        see = see & (j <= at)
        if window:
            see = see & (j > at - window)
    return see


def clean(x, n):
    """x in 64 bits with what is beyond row n replaced by zeros (it may hold anything)."""
    y = x.detach().cpu().double().clone()
    y[n:] = 0
    return y


class Case:
    """Results and bounds of one call, [batch, heads, ...] in 64 bits."""

    def __init__(self, q, k, v, *, causal=False, window=0, scale=None, q_lens=None, k_lens=None):
        b, h, nq, d = q.shape
        kv, nk = k.shape[1], k.shape[2]
        self.scale = 1 / math.sqrt(d) if scale is None else scale
        self.u, self.tiny = U[q.dtype], TINY[q.dtype]
        self.group = h // kv
        self.lens = [(nq if q_lens is None else max(0, min(nq, int(q_lens[i]))), nk if k_lens is None else max(0, min(nk, int(k_lens[i]))))
                     for i in range(b)]
        self.q = torch.stack([torch.stack([clean(q[i, j], self.lens[i][0]) for j in range(h)]) for i in range(b)])
        self.k = torch.stack([torch.stack([clean(k[i, j], self.lens[i][1]) for j in range(kv)]) for i in range(b)])
        self.v = torch.stack([torch.stack([clean(v[i, j], self.lens[i][1]) for j in range(kv)]) for i in range(b)])
        self.see = torch.stack([visible(nq, nk, *self.lens[i], causal, window) for i in range(b)])[:, None]
        kg, vg = self.k.repeat_interleave(self.group, 1), self.v.repeat_interleave(self.group, 1)
        self.kg, self.vg = kg, vg
        s = self.scale * self.q @ kg.transpose(-1, -2)
        # how far a score in 32 bits may be off: each of d products, and the scaled sum
        self.ds = E * (1 + self.scale * (self.q.abs() @ kg.abs().transpose(-1, -2)))
        s = s.masked_fill(~self.see, -math.inf)
        top = s.amax(-1, keepdim=True) if nk else torch.full(s.shape[:-1] + (1,), -math.inf, dtype=torch.float64)
        e = torch.exp(s - top.masked_fill(top == -math.inf, 0))
        z = e.sum(-1, keepdim=True)
        self.p = torch.where(z > 0, e / z, torch.zeros_like(e))
        self.out = self.p @ vg
        self.lse = (top + z.log()).squeeze(-1)
        self.lse_bound = torch.where(self.see, self.ds, torch.zeros_like(self.ds)).amax(-1) if nk else torch.zeros_like(self.lse)
        spread = self.p * self.ds * 2
        self.out_bound = self.u * (self.p @ vg.abs() + self.out.abs()) + spread @ vg.abs() + spread.sum(-1, keepdim=True) * self.out.abs() \
            + E * (self.p @ vg.abs()) + self.tiny * (1 + self.see.double() @ vg.abs())

    def shared(self, x):
        """Sum over the query heads of a key head."""
        b, h = x.shape[:2]
        return x.view(b, h // self.group, self.group, *x.shape[2:]).sum(2)

    def weights(self):
        return self.shared(self.p).sum(2), self.shared(self.p * self.ds * 2).sum(2) + E * self.shared(self.p).sum(2)

    def grads(self, dout, out):
        """{name: (value, bound)}; out is what the forward pass returned."""
        b, h, nq, d = self.q.shape
        g = torch.stack([torch.stack([clean(dout[i, j], self.lens[i][0]) for j in range(h)]) for i in range(b)])
        o = torch.stack([torch.stack([clean(out[i, j], self.lens[i][0]) for j in range(h)]) for i in range(b)])
        p, u = self.p, self.u
        dp = g @ self.vg.transpose(-1, -2)
        delta = (g * o).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        # in 32 bits: the probability, the two products and their difference
        off = ds.abs() * self.ds * 2 + p * E * (g.abs() @ self.vg.abs().transpose(-1, -2) + (g * o).abs().sum(-1, keepdim=True))
        t = lambda x: x.transpose(-1, -2)
        dv, dv_b = self.shared(t(p) @ g), self.shared(t(p) @ g.abs())
        dv_off = self.shared(t(p * self.ds * 2) @ g.abs())
        dq, dq_b = self.scale * ds @ self.kg, self.scale * ds.abs() @ self.kg.abs()
        dk, dk_b = self.scale * self.shared(t(ds) @ self.q), self.scale * self.shared(t(ds.abs()) @ self.q.abs())
        see = self.see.double().expand(p.shape)
        return dict(dq=(dq, (u + E) * dq_b + u * dq.abs() + self.scale * off @ self.kg.abs() + self.tiny * (1 + self.scale * see @ self.kg.abs())),
                    dk=(dk, (u + E) * dk_b + u * dk.abs() + self.scale * self.shared(t(off) @ self.q.abs()) + self.tiny * (1 + self.scale * self.shared(t(see) @ self.q.abs()))),
                    dv=(dv, (u + E) * dv_b + u * dv.abs() + dv_off + self.tiny * (1 + self.shared(t(see) @ g.abs()))))


def rank(weights, positions, newest, recent):
    """Sort keys of the slots of one row, least first: the order in which slots are given up."""
    keys = []
    for i, (w, p) in enumerate(zip(weights, positions)):
        if p < 0:
            keys.append((0, 0.0, i))
        elif p > newest - recent:
            keys.append((3, 0.0, -i))
        else:
            keys.append((1, 0.0, -i) if math.isnan(w) else (2, w, -i))
    return keys


def evict(weights, positions, length, keep, recent):
    """Slots of one row that stay, ascending."""
    pos = [i if positions is None else int(positions[i]) for i in range(length)]
    w = [float(weights[i]) for i in range(length)]
    keys = rank(w, pos, max(pos, default=-1), recent)
    used = [i for i in range(length) if pos[i] >= 0]
    return sorted(sorted(used, key=lambda i: keys[i], reverse=True)[:keep])


def insert(weights, positions, position, recent):
    """The slot that a new token takes."""
    pos = [int(p) for p in positions]
    keys = rank([float(w) for w in weights], pos, position, recent)
    return min(range(len(pos)), key=lambda i: keys[i])
