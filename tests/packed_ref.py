"""Rows in 4 or 8 bits an element, from their definition on the CPU: numbers to bytes and back, one group at a time."""
import math

import numpy as np
import torch

GROUP = 32
WIDEST = 2.0 ** 100


def row_bytes(d, bits):
    groups = -(-d // GROUP)
    return -(-groups * (GROUP * bits // 8 + 4) // 16) * 16


def number(bits16, kind):
    """The number of this type with these 16 bits."""
    return float(torch.tensor([bits16 if bits16 < 1 << 15 else bits16 - (1 << 16)], dtype=torch.int16).view(kind))


def bits_of(x, kind):
    return int(torch.tensor([x]).to(kind).view(torch.int16)) & 0xFFFF


def least_from(want, kind):
    """Bits of the least number of the type from `want` (not negative) on."""
    b = bits_of(want, kind)
    return b + 1 if number(b, kind) < want else b


def pack_row(x, bits):
    """A row (a CPU tensor of one dimension) as bytes."""
    kind, d = x.dtype, x.shape[0]
    most = 2 ** bits - 1
    words, ends = [], []
    for start in range(0, d, GROUP):
        g = x[start:start + GROUP].float().numpy()
        low, high = np.float32(g.min()) + np.float32(0), np.float32(g.max()) + np.float32(0)      # no minus zero
        with np.errstate(all="ignore"):
            span = np.float32(high - low)
            u = np.zeros(GROUP, np.int64)
            if not span <= WIDEST:
                lo, step = bits_of(math.nan, kind), 0
            else:
                lo, step = bits_of(float(low), kind), least_from(float(span / np.float32(most)), kind)
                if math.isinf(float(torch.tensor(float(low) + most * number(step, kind), dtype=torch.float32).to(kind))):
                    step -= 1
                if step:
                    u[:len(g)] = np.minimum(np.rint((g - low) / np.float32(number(step, kind))), most)
        each = 32 // bits
        for w in range(0, GROUP, each):
            word = 0
            for i in range(each):
                word |= int(u[w + i]) << (bits * (i // 2) + 16 * (i % 2))
            words.append(word)
        ends.append(lo | step << 16)
    raw = np.array(words + ends, np.uint32).tobytes()
    return torch.frombuffer(bytearray(raw + bytes(row_bytes(d, bits) - len(raw))), dtype=torch.uint8)


def unpack_row(row, kind, d, bits):
    """What a row of bytes stands for: a tensor of d numbers of the type."""
    raw = np.frombuffer(row.numpy().tobytes(), np.uint32)
    groups, each = -(-d // GROUP), 32 // bits
    out = []
    for e in range(d):
        u = int(raw[e // each]) >> (bits * (e % each // 2) + 16 * (e % 2)) & (2 ** bits - 1)
        ends = int(raw[groups * bits + e // GROUP])
        out.append(number(ends & 0xFFFF, kind) + u * number(ends >> 16, kind))
    return torch.tensor(out, dtype=torch.float64).to(kind)


def pack(x, bits):
    flat = x.detach().cpu().reshape(-1, x.shape[-1])
    rows = [pack_row(r, bits) for r in flat]
    out = torch.stack(rows) if rows else torch.zeros(0, row_bytes(x.shape[-1], bits), dtype=torch.uint8)
    return out.view(*x.shape[:-1], -1) if rows else out.view(*x.shape[:-1], row_bytes(x.shape[-1], bits))


def unpack(rows, kind, d, bits):
    """Many rows of bytes at once."""
    rows = rows.detach().cpu().contiguous()
    flat = rows.view(-1, rows.shape[-1]).numpy().view(np.uint32)
    groups, each = -(-d // GROUP), 32 // bits
    e = np.arange(d)
    shift = (bits * (e % each // 2) + 16 * (e % 2)).astype(np.uint32)
    u = (flat[:, e // each] >> shift) & np.uint32(2 ** bits - 1)
    ends = flat[:, groups * bits + e // GROUP]
    as_kind = lambda x: torch.from_numpy((x & 0xFFFF).astype(np.uint16).view(np.int16).copy()).view(kind).double()
    out = as_kind(ends) + torch.from_numpy(u.astype(np.float64)) * as_kind(ends >> 16)
    return out.to(kind).view(*rows.shape[:-1], d)
