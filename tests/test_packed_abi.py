"""Refusals of the packed cache's calls: all before anything is enqueued, so none of these needs a GPU."""
import pytest

import packed_ref as ref
from test_attention_abi import FAKE, cache, lib, rows, shape      # noqa: F401


def packed(**kw):
    from paper_1903_06631_amd.attention_ops import _Packed
    row = dict(batch=1 << 16, head=1 << 12, row=48)      # 64 elements in 4 bits: 40 bytes and what makes 48
    c = dict(type=0, bits=4, batch=2, kv_heads=2, slots=7, head_dim=64, k=rows(FAKE, **row), v=rows(FAKE * 2, **row))
    c.update(kw)
    return _Packed(**c)


def other(**kw):
    return rows(**{"data": FAKE * 3, **kw})


def test_row_bytes(lib):      # noqa: F811
    for bits in (4, 8):
        for d in range(8, 129, 8):
            assert lib.lap_packed_row_bytes(bits, d) == ref.row_bytes(d, bits), (bits, d)
    for bits, d in ((4, 0), (4, 4), (4, 136), (8, 60), (5, 64), (0, 64), (16, 64)):
        assert lib.lap_packed_row_bytes(bits, d) == 0
    assert len({ref.row_bytes(d, 4) for d in (128,)} & {ref.row_bytes(d, 8) for d in (128,)}) == 0
    for d in range(8, 129, 8):
        assert ref.row_bytes(d, 4) != ref.row_bytes(d, 8)      # so a row's bytes tell its bits


@pytest.mark.parametrize("name", ["lap_cache_pack", "lap_cache_unpack"])
def test_pack_and_unpack(lib, name):      # noqa: F811
    def call(c=None, k=None, v=None, n=5):
        k, v = k or other(), v or other(data=FAKE * 4)
        if name == "lap_cache_pack":
            return lib.lap_cache_pack(c or packed(), k, v, n, None, None, None)
        return lib.lap_cache_unpack(c or packed(), n, None, None, k, v, None)
    for bad in (dict(type=2), dict(type=9), dict(bits=5), dict(bits=16), dict(bits=0)):
        assert call(packed(**bad)) == -9, bad
    for bad in (dict(batch=0), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=136), dict(slots=1 << 31), dict(batch=1 << 16)):
        assert call(packed(**bad)) == -2, bad
    assert call(n=(1 << 30) + 1) == -2
    assert call(packed(head_dim=60)) == -10
    for x in ("k", "v"):
        assert call(packed(**{x: rows(data=None)})) == -1
        for bad in (dict(data=FAKE + 8), dict(row=56), dict(head=24), dict(batch=-16), dict(row=1 << 25)):
            assert call(packed(**{x: rows(**{"row": 48, **bad})})) == -10, bad
        for bad in (dict(data=FAKE + 8), dict(row=68), dict(head=4), dict(batch=-8)):
            assert call(**{x: other(**bad)}) == -10, bad
        assert call(**{x: rows(data=None)}) == -1
        overlapping = dict(row=32) if name == "lap_cache_pack" else dict(row=0)
        if name == "lap_cache_pack":
            assert call(packed(**{x: rows(FAKE * 5, row=32)})) == -10
        else:
            assert call(**{x: other(**overlapping)}) == -10
    # an output where something is read, and both outputs at one place
    if name == "lap_cache_pack":
        assert call(k=rows(data=FAKE)) == -10 and call(v=rows(data=FAKE)) == -10 and call(k=rows(data=2 * FAKE)) == -10
        assert call(packed(v=rows(FAKE, row=48))) == -10
        assert lib.lap_cache_pack(None, other(), other(), 5, None, None, None) == -1
    else:
        assert call(k=other(data=FAKE)) == -10 and call(v=other(data=2 * FAKE)) == -10 and call(v=other()) == -10
        assert lib.lap_cache_unpack(None, 5, None, None, other(), other(), None) == -1
    assert call(n=0, k=rows(data=None), v=rows(data=None)) == 0      # nothing to do


def test_step(lib):      # noqa: F811
    def call(s=None, c=None, positions=None, ws=FAKE << 8, have=1 << 30, before=FAKE, weights=FAKE, lse=FAKE, **kw):
        a = {n: kw.get(n, other()) for n in ("q", "out")}
        return lib.lap_attention_step_packed(s or shape(), a["q"], c or packed(), positions, before, a["out"], lse, weights, ws, have, None)
    for bad in (dict(q_len=0), dict(causal=0), dict(window=3), dict(type=5), dict(scale=0.0), dict(type=1), dict(batch=1), dict(k_len=8),
                dict(kv_heads=4), dict(head_dim=72)):
        assert call(shape(**bad)) == -9, bad
    assert call(shape(kv_heads=1), packed(kv_heads=2)) == -9
    assert call(positions=FAKE) == -9      # several tokens, and slots that stand in no order
    assert call(shape(q_heads=514, q_len=1)) == -2 and call(shape(q_heads=64, q_len=9)) == -2
    for bad in (dict(bits=3), dict(type=2)):
        assert call(c=packed(**bad)) == -9
    assert call(c=packed(k=rows(FAKE, row=40))) == -10 and call(c=packed(v=rows(None))) == -1
    assert call(before=None) == -1 and call(weights=None) == -1 and call(lse=None) == -1 and call(q=rows(data=None)) == -1
    assert call(out=other(row=0)) == -10 and call(out=rows(FAKE)) == -10 and call(out=rows(2 * FAKE)) == -10
    many = shape(k_len=9000)      # few caches of many slots: in chunks, joined in a workspace
    need = lib.lap_attention_workspace_bytes(4, many)
    assert need > 0 and call(many, packed(slots=9000), have=need - 1) == -3 and call(many, packed(slots=9000), ws=None) == -3
    assert lib.lap_attention_workspace_bytes(4, shape(causal=0)) == 0


def test_moved_rows_of_bytes(lib):      # noqa: F811
    """Eviction and insertion take packed rows as bytes."""
    row = dict(row=48)
    byte = lambda **kw: cache(**{"type": 2, "head_dim": 48, "k": rows(FAKE, **row), "v": rows(FAKE * 2, **row), **kw})
    def evict(src=None, dst=None):
        return lib.lap_cache_evict(src or byte(), None, 8, 2, dst or byte(slots=8, k=rows(FAKE * 3, **row), v=rows(FAKE * 4, **row)), FAKE, FAKE << 8, 64, None)
    assert evict() == -3      # nothing else to find fault with
    assert evict(byte(head_dim=40)) == -10 and evict(byte(head_dim=272)) == -2 and evict(byte(head_dim=64)) == -9 and evict(byte(type=0)) == -9
    assert evict(byte(k=rows(FAKE, row=56))) == -10 and evict(byte(v=rows(FAKE + 8, row=48))) == -10
    assert evict(dst=byte(slots=8, k=rows(FAKE * 3, row=32), v=rows(FAKE * 4, **row))) == -10
    insert = lambda c, k=None, v=None, recent=17: lib.lap_cache_insert(c, k or rows(FAKE * 5, **row), v or rows(FAKE * 6, **row), FAKE, recent, FAKE, None)
    assert insert(byte()) == -2 and insert(byte(), k=rows(FAKE, head=40), recent=2) == -10 and insert(byte(), v=rows(None), recent=2) == -1


def test_binding_refuses_before_the_library():
    import torch
    import paper_1903_06631_amd as lap
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    c = torch.zeros(1, 2, 3, 48, dtype=torch.uint8)
    for call in (lambda: lap.cache_pack(x, x, 4), lambda: lap.cache_pack(x, x), lambda: lap.cache_unpack(c, c, torch.bfloat16, 64),
                 lambda: lap.cache_unpack(c, c, torch.float32, 64), lambda: lap.attention_step_packed(x, c, c), lambda: lap.packed_row_bytes(4, 20),
                 lambda: lap.packed_row_bytes(3, 64), lambda: lap.attention_step_packed(x[0, 0], c, c)):
        with pytest.raises(ValueError):
            call()
    assert lap.packed_row_bytes(4, 128) == 80 and lap.packed_row_bytes(8, 128) == 144


@pytest.mark.parametrize("q_shape,kv_shape", [((2, 40, 1, 128), (2, 1, 0, 128)), ((64, 64, 5, 128), (64, 8, 0, 128)), ((257, 40, 1, 128), (257, 1, 0, 128)),
                                              ((600, 256, 1, 64), (600, 1, 0, 64)), ((1, 65535, 64, 8), (1, 65535, 0, 8))])
def test_workspace_without_slots(q_shape, kv_shape):
    """Caches without slots and more than 32 rows to a key head, of few key heads and of more than there are places for workgroups: a
    workspace like any other's.  (In a process of its own: a division by zero in the library ends it.)"""
    import os
    import subprocess
    import sys
    code = ("import torch, paper_1903_06631_amd as lap\n"
            f"print(lap.attention_workspace_bytes(lap.AT_STEP_PACKED, {q_shape}, {kv_shape}, torch.bfloat16))")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, f"ended with {r.returncode}: {r.stderr[-500:]}"
    need = int(r.stdout.split()[-1])
    assert need > 0 and need % 256 == 0


def test_workspace_of_a_call_without_weights(lib):      # noqa: F811
    """No room for the scores, which only the weights need: 64 rows of 131072 slots are more than the packed rows themselves."""
    import torch
    import paper_1903_06631_amd as lap
    for q_shape, kv_shape in (((16, 32, 5, 128), (16, 8, 8192, 128)), ((2, 64, 8, 128), (2, 8, 131072, 128)), ((64, 512, 128), (64, 8, 4096, 128))):
        need = [lap.attention_workspace_bytes(x, q_shape, kv_shape, torch.bfloat16) for x in (lap.AT_STEP_PACKED, lap.AT_STEP_PACKED_UNWEIGHTED)]
        queries = q_shape[0] * q_shape[1] * (q_shape[2] if len(q_shape) == 4 else 1)
        assert need[0] - need[1] == queries * kv_shape[2] * 4 and 0 < need[1] < 1 << 27
    many, c = shape(k_len=9000), packed(slots=9000)
    need = [lib.lap_attention_workspace_bytes(x, many) for x in (4, 5)]
    def call(have, w):      # (the last of the checks, after the workspace's, refuses an output in the place of the keys)
        return lib.lap_attention_step_packed(many, other(), c, None, w, rows(FAKE), FAKE, w, FAKE << 8, have, None)
    assert need[1] < need[0] and call(need[1] - 1, None) == -3 and call(need[1], None) == -10
    assert call(need[0] - 1, FAKE) == -3 and call(need[0], FAKE) == -10
    assert lib.lap_attention_workspace_bytes(5, shape(causal=0)) == 0 and lib.lap_attention_workspace_bytes(6, many) == 0
