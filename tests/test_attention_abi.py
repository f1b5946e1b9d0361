"""Refusals of the attention and cache calls: all before anything is enqueued, so none of these needs a GPU."""
import ctypes as C
import os

import pytest

FAKE = 0x10000      # never dereferenced


@pytest.fixture(scope="module")
def lib():
    import paper_1903_06631_amd as lap
    if not os.path.exists(lap.lib_path()):
        from paper_1903_06631_amd import build
        build.build()
    return lap.load_library()


def shape(**kw):
    from paper_1903_06631_amd.attention_ops import _Shape
    s = dict(type=0, batch=2, q_heads=4, kv_heads=2, q_len=5, k_len=7, head_dim=64, causal=1, window=0, scale=0.125, q_lens=None, k_lens=None)
    s.update(kw)
    return _Shape(**s)


def rows(data=FAKE, batch=1 << 16, head=1 << 12, row=64):
    from paper_1903_06631_amd.attention_ops import _Rows
    return _Rows(data, batch, head, row)


def forward(lib, s=None, q=None, k=None, v=None, out=None, lse=FAKE):
    return lib.lap_attention(s or shape(), q or rows(), k or rows(), v or rows(), out or rows(), lse, None, 0, None)


def test_shapes(lib):
    for bad in (dict(type=2), dict(q_heads=3), dict(causal=2), dict(causal=0, window=4), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf"))):
        assert forward(lib, shape(**bad)) == -9, bad
    for bad in (dict(batch=0), dict(q_heads=0, kv_heads=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=136), dict(q_len=(1 << 30) + 1),
                dict(k_len=0xFFFFFFFF), dict(batch=1 << 20, q_heads=1 << 10, kv_heads=1)):
        assert forward(lib, shape(**bad)) == -2, bad
    assert forward(lib, shape(head_dim=60)) == -10
    assert lib.lap_attention(None, rows(), rows(), rows(), rows(), FAKE, None, 0, None) == -1
    assert lib.lap_attention_workspace_bytes(1, shape()) >= 2 * 4 * 5 * 8
    assert lib.lap_attention_workspace_bytes(1, shape(type=7)) == 0 and lib.lap_attention_workspace_bytes(9, shape()) == 0


def test_rows_and_pointers(lib):
    for name in ("q", "k", "v", "out"):
        assert forward(lib, **{name: rows(data=None)}) == -1, name
        for bad in (dict(data=FAKE + 8), dict(row=68), dict(head=4), dict(batch=-8), dict(row=1 << 24)):
            assert forward(lib, **{name: rows(**bad)}) == -10, (name, bad)
    for bad in (dict(row=0), dict(head=0), dict(batch=0), dict(row=56)):
        assert forward(lib, out=rows(**bad)) == -10, bad
    assert forward(lib, lse=None) == -1
    assert lib.lap_attention(shape(), None, rows(), rows(), rows(), FAKE, None, 0, None) == -1
    few = shape(batch=1, k_len=3000)      # few rows on many keys: the keys in parts, joined in a workspace
    assert lib.lap_attention_workspace_bytes(0, shape()) == 0 and lib.lap_attention_workspace_bytes(0, few) > 0
    assert forward(lib, few) == -3
    assert forward(lib, shape(q_len=0), q=rows(data=None), out=rows(data=None), lse=None) == 0      # nothing to do


def test_gradient(lib):
    def call(s=None, ws=FAKE << 8, have=1 << 30, lse=FAKE, **kw):
        a = {n: kw.get(n, rows()) for n in ("dout", "q", "k", "v", "out", "dq", "dk", "dv")}
        return lib.lap_attention_grad(s or shape(), a["dout"], a["q"], a["k"], a["v"], a["out"], lse, a["dq"], a["dk"], a["dv"], ws, have, None)
    for name in ("dout", "q", "k", "v", "out", "dq", "dk", "dv"):
        assert call(**{name: None}) == -1 and call(**{name: rows(data=None)}) == -1 and call(**{name: rows(row=12)}) == -10, name
    for name in ("dq", "dk", "dv"):
        assert call(**{name: rows(row=0)}) == -10, name
    assert call(lse=None) == -1
    need = lib.lap_attention_workspace_bytes(1, shape())
    assert call(ws=None) == -3 and call(ws=(FAKE << 8) + 16) == -3 and call(have=need - 1) == -3
    assert call(shape(q_len=0, k_len=0), ws=None, have=0) == 0


def test_weights(lib):
    call = lambda s=None, q=None, k=None, lse=FAKE, w=FAKE: lib.lap_attention_weights(s or shape(), q or rows(), k or rows(), lse, None, w, None, 0, None)
    assert call(lse=None) == -1 and call(w=None) == -1 and call(q=rows(data=None)) == -1 and call(k=rows(data=FAKE + 2)) == -10
    assert call(shape(batch=1, q_heads=8, kv_heads=1, q_len=2000)) == -3      # the rows in parts, no workspace
    assert call(shape(scale=2e6)) == -9 and call(shape(k_len=0), k=rows(data=None), w=None) == 0


def test_step(lib):
    one = dict(q_len=1, causal=0)
    def call(s=None, ws=FAKE << 8, have=1 << 30, before=FAKE, weights=FAKE, lse=FAKE, **kw):
        a = {n: kw.get(n, rows()) for n in ("q", "k", "v", "out")}
        return lib.lap_attention_step(s or shape(**one), a["q"], a["k"], a["v"], None, before, a["out"], lse, weights, ws, have, None)
    for bad in (dict(q_len=2, causal=0), dict(q_len=1, causal=1), dict(q_lens=FAKE, **one), dict(type=5, **one)):
        assert call(shape(**bad)) == -9, bad
    assert call(shape(q_heads=514, kv_heads=2, **one)) == -2
    assert call(before=None) == -1 and call(weights=None) == -1 and call(lse=None) == -1 and call(k=rows(data=None)) == -1
    assert call(out=rows(head=0)) == -10
    many = shape(k_len=3000, **one)      # few caches of many slots: in chunks, joined in a workspace
    assert lib.lap_attention_workspace_bytes(3, shape(**one)) == 0 and lib.lap_attention_workspace_bytes(3, many) > 0
    assert call(many, have=lib.lap_attention_workspace_bytes(3, many) - 1) == -3


def cache(**kw):
    from paper_1903_06631_amd.attention_ops import _Cache
    c = dict(type=0, batch=2, kv_heads=2, slots=16, head_dim=64, k=rows(), v=rows(), weights=FAKE, positions=FAKE)
    c.update(kw)
    return _Cache(**c)


def test_evict(lib):
    def call(src=None, dst=None, keep=8, recent=2, lens_out=FAKE, ws=FAKE << 8, have=1 << 20):
        return lib.lap_cache_evict(src or cache(), None, keep, recent, dst or cache(slots=8), lens_out, ws, have, None)
    assert call(keep=0) == -2 and call(keep=9) == -2 and call(recent=9) == -2 and call(cache(batch=0)) == -2
    assert call(cache(batch=1 << 15)) == -2 and call(cache(slots=1 << 31)) == -2
    assert call(cache(type=1)) == -9 and call(cache(kv_heads=1)) == -9 and call(cache(head_dim=72)) == -9 and call(cache(type=2)) == -9
    assert call(cache(weights=None)) == -1 and call(dst=cache(slots=8, positions=None)) == -1 and call(lens_out=None) == -1
    assert call(dst=cache(slots=8, weights=None)) == -1 and call(cache(k=rows(data=None))) == -1
    assert call(dst=cache(slots=8, v=rows(row=0))) == -10 and call(cache(head_dim=20)) == -10
    assert call(ws=None) == -3 and call(have=64) == -3
    assert lib.lap_cache_evict(None, None, 1, 1, cache(), FAKE, None, 0, None) == -1


def test_insert(lib):
    def call(c=None, k=None, v=None, position=FAKE, recent=2, slots=FAKE):
        return lib.lap_cache_insert(c or cache(), k or rows(), v or rows(), position, recent, slots, None)
    assert call(recent=17) == -2 and call(cache(slots=0), recent=0) == -2
    assert call(position=None) == -1 and call(slots=None) == -1 and call(cache(positions=None)) == -1 and call(k=rows(data=None)) == -1
    assert call(cache(k=rows(row=0))) == -10 and call(v=rows(head=12)) == -10 and call(cache(type=3)) == -9
    assert lib.lap_cache_insert(None, rows(), rows(), FAKE, 0, FAKE, None) == -1


def test_binding_refuses_before_the_library():
    import torch
    import paper_1903_06631_amd as lap
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lap.attention(x, x, x)      # not on the GPU
    with pytest.raises(ValueError):
        lap.cache_evict(x, x, torch.zeros(1, 2, 3), 2, 1)
