"""Which strides of rows are taken and which refused.  Nothing is enqueued: where rows are right, the workspace is missing, and
that is looked at after the rows (status -3; -10: the rows)."""
import itertools
import random

import pytest
import torch

from test_attention_abi import FAKE, cache, lib, rows, shape  # noqa: F401

TAKEN, REFUSED = -3, -10


def grad(lib, s, **kw):
    good = lambda n: rows(batch=1 << 18, head=1 << 14, row=64)
    a = {n: kw.get(n, good(n)) for n in ("dout", "q", "k", "v", "out", "dq", "dk", "dv")}
    return lib.lap_attention_grad(s, a["dout"], a["q"], a["k"], a["v"], a["out"], FAKE, a["dq"], a["dk"], a["dv"], None, 0, None)


def overlap(batch, heads, length, d, strides):
    taken = set()
    for at in itertools.product(range(batch), range(heads), range(length)):
        first = sum(i * s for i, s in zip(at, strides))
        for e in range(first, first + d):
            if e in taken:
                return True
            taken.add(e)
    return False


def test_outputs_whose_rows_overlap(lib):
    s = shape(kv_heads=4)
    for strides in ((64, 64, 64), (1 << 16, 64, 64), (1 << 16, 64, 128), (128, 1 << 12, 64), (1 << 12, 1 << 12, 64), (1 << 16, 64, 192), (256, 64, 256)):
        for name in ("dq", "dk", "dv"):
            assert grad(lib, s, **{name: rows(FAKE, *strides)}) == REFUSED, (name, strides)
        for name in ("dout", "q", "k", "v", "out"):
            assert grad(lib, s, **{name: rows(FAKE, *strides)}) == TAKEN, (name, strides)
    for strides in ((1 << 16, 64, 256), (256, 64, 512), (64, 128, 512), (5 * 256, 64, 256)):
        for name in ("dq", "dk", "dv"):
            assert grad(lib, s, **{name: rows(FAKE, *strides)}) == (REFUSED if overlap(2, 4, 5 if name == "dq" else 7, 64, strides) else TAKEN), (name, strides)
    # rows of one head between those of another
    far = shape(q_heads=2, kv_heads=2, q_len=130, k_len=130)
    assert grad(lib, far, dq=rows(FAKE, 1 << 31, 64, (1 << 24) - 8)) == TAKEN
    assert grad(lib, far, dq=rows(FAKE, ((1 << 24) - 8) * 100, 64, (1 << 24) - 8)) == REFUSED
    assert grad(lib, far, dq=rows(FAKE, ((1 << 24) - 8) * 100 + 128, 64, (1 << 24) - 8)) == TAKEN
    assert lib.lap_cache_evict(cache(), None, 4, 0, cache(slots=8, v=rows(FAKE, 1 << 16, 64, 64)), FAKE, None, 0, None) == REFUSED
    assert lib.lap_cache_evict(cache(), None, 4, 0, cache(slots=8, v=rows(FAKE, 1 << 16, 64, 128)), FAKE, None, 0, None) == TAKEN


def test_any_strides(lib):
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(3000):
        b, h, n = rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 6)
        strides = [8 * rng.choice([rng.randint(0, 5), rng.randint(2, 40), rng.randint(30, 400)]) for _ in range(3)]
        want = overlap(b, h, n, 16, strides)
        seen[want] += 1
        s = shape(batch=b, q_heads=h, kv_heads=h, q_len=n, k_len=7, head_dim=16)
        assert grad(lib, s, dq=rows(FAKE, *strides)) == (REFUSED if want else TAKEN), (b, h, n, strides)
    assert min(seen) > 500


def test_strides_of_one_place_do_not_matter(lib):
    for odd in (4, -8, 1 << 40, 0, 1):
        one = shape(batch=1, q_heads=1, kv_heads=1, q_len=1, k_len=1)
        good = dict(batch=1 << 16, head=1 << 12, row=64)
        for place in ("batch", "head", "row"):
            for name in ("dout", "q", "k", "v", "out", "dq", "dk", "dv"):
                assert grad(lib, one, **{name: rows(**{**good, place: odd})}) == TAKEN, (name, place, odd)
        long = shape(q_len=1, causal=0, k_len=3000)
        call = lambda **kw: lib.lap_attention_step(long, kw.get("q", rows()), rows(), rows(), None, None, kw.get("out", rows()), FAKE, None, None, 0, None)
        assert call(q=rows(row=odd)) == TAKEN and call(out=rows(row=odd)) == TAKEN
    # and those of more places do
    for bad in (4, -8):
        assert grad(lib, shape(), q=rows(batch=bad)) == REFUSED and grad(lib, shape(), q=rows(head=bad)) == REFUSED and grad(lib, shape(), q=rows(row=bad)) == REFUSED
    assert grad(lib, shape(), q=rows(row=1 << 24)) == REFUSED


@pytest.mark.gpu
def test_results_with_strides_that_are_not_used():
    import paper_1903_06631_amd as lap
    gen = torch.Generator().manual_seed(1)
    make = lambda n: torch.randn(1, 1, n, 64, generator=gen).to(torch.bfloat16).cuda()
    for n, m in ((1, 1), (1, 70), (70, 1)):
        q, k, v, g = make(n), make(m), make(m), make(n)
        odd = [x.as_strided(x.shape, (12345, 3, 64 if x.shape[2] > 1 else (1 << 33) + 5, 1)) for x in (q, k, v, g)]
        a, b = lap.attention(q, k, v), lap.attention(*odd[:3])
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
        a, b = lap.attention_grad(g, q, k, v, a["out"], a["lse"]), lap.attention_grad(odd[3], *odd[:3], a["out"], a["lse"])
        assert all(torch.equal(a[x], b[x]) for x in a)


def test_workspaces_by_shape(lib):
    import paper_1903_06631_amd as lap
    q, kv = (2, 4, 5, 64), (2, 2, 7, 64)
    for which in range(4):
        assert lap.attention_workspace_bytes(which, q, kv, torch.bfloat16, causal=True) == lib.lap_attention_workspace_bytes(which, shape())
    long = shape(type=1, q_len=1, k_len=3000, causal=0)
    assert lap.attention_workspace_bytes(lap.AT_STEP, (2, 4, 64), (2, 2, 3000, 64), torch.float16) == lib.lap_attention_workspace_bytes(3, long) > 0
