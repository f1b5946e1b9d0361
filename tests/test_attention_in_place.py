"""Outputs in the memory of operands that other rows still need are refused, before anything is enqueued; outputs in memory
next to each other are right."""
import pytest
import torch

from test_attention_abi import FAKE, cache, lib, rows, shape  # noqa: F401

REFUSED, WS, MANY = -10, FAKE << 8, 1 << 30


def at(i):
    return rows((1 + i) << 24)


def test_prompts(lib):
    for bad in (1, 2):
        places = [at(3 if i == bad else i) for i in range(4)]
        assert lib.lap_attention(shape(), *places, FAKE, WS, MANY, None) == REFUSED, bad


def test_gradients(lib):
    names = ("dout", "q", "k", "v", "out", "dq", "dk", "dv")
    place = {n: i for i, n in enumerate(names)}
    def call(**kw):
        a = {n: at(kw.get(n, i)) for n, i in place.items()}
        return lib.lap_attention_grad(shape(), a["dout"], a["q"], a["k"], a["v"], a["out"], FAKE, a["dq"], a["dk"], a["dv"], WS, MANY, None)
    for output, others in (("dq", ("dout", "q", "k", "v", "dk", "dv")), ("dk", ("dout", "q", "dv")), ("dv", ("dout", "q", "dk"))):
        for other in others:
            assert call(**{output: place[other]}) == REFUSED, (output, other)


def test_weights_and_steps(lib):
    assert lib.lap_attention_weights(shape(), at(0), at(1), FAKE, None, FAKE, WS, MANY, None) == REFUSED
    one = shape(q_len=1, causal=0)
    for bad in (1, 2):
        q, k, v, out = (at(3 if i == bad else i) for i in range(4))
        assert lib.lap_attention_step(one, q, k, v, None, None, out, FAKE, None, WS, MANY, None) == REFUSED, bad


def test_caches(lib):
    src = cache(k=at(0), v=at(1), weights=FAKE, positions=FAKE << 1)
    for bad in (dict(k=at(0)), dict(k=at(1)), dict(v=at(0)), dict(v=at(1)), dict(v=at(2)), dict(weights=FAKE), dict(positions=FAKE << 1)):
        to = dict(slots=8, k=at(2), v=at(3), weights=FAKE << 2, positions=FAKE << 3)
        assert lib.lap_cache_evict(src, None, 4, 0, cache(**{**to, **bad}), FAKE << 4, WS, MANY, None) == REFUSED, bad


@pytest.mark.gpu
def test_one_tensor_for_all_gradients():
    """dq, dk and dv as slices of one tensor, as those of a joined projection are: rows of one between those of another."""
    import paper_1903_06631_amd as lap
    gen = torch.Generator().manual_seed(1)
    qkv = torch.randn(2, 150, 3, 4, 64, generator=gen).to(torch.bfloat16).cuda()
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    g = torch.randn(2, 4, 150, 64, generator=gen).to(torch.bfloat16).cuda()
    f = lap.attention(q, k, v, causal=True)
    want = lap.attention_grad(g, q, k, v, f["out"], f["lse"], causal=True)
    into = torch.full_like(qkv, 7)
    lap.attention_grad(g, q, k, v, f["out"], f["lse"], causal=True, grads={n: into[:, :, i].transpose(1, 2) for i, n in enumerate(("dq", "dk", "dv"))})
    assert all(torch.equal(into[:, :, i].transpose(1, 2), want[n]) for i, n in enumerate(("dq", "dk", "dv")))
    with pytest.raises(lap.LapError) as e:
        lap.attention_grad(g, q, k, v, f["out"], f["lse"], causal=True, grads=dict(dq=q, dk=want["dk"], dv=want["dv"]))
    assert e.value.status == -10
