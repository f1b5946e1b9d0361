"""ctypes binding of liblap's attention and cache operators: argument marshalling only.

Tensors are [batch, heads, length, head_dim] in torch.bfloat16 or torch.float16 with elements of a row side by side; other
strides are free (a [batch, length, heads, head_dim] tensor goes in as its transpose(1, 2)).  Lengths, positions and slots
are torch.int32, weights and logarithms of softmax sums torch.float32, all contiguous.  Work is enqueued on the current
stream of q's device; `sync=False` returns without waiting for it.  `out` takes result tensors that the caller owns, `ws` a
workspace (uint8, 256-byte aligned, at least attention_workspace_bytes; cache_evict: 4 bytes for every slot of the new cache,
rounded up to a multiple of 256).  Autograd does not see these calls: their results have no gradient, attention_grad computes
it, and a torch.autograd.Function around the two is the caller's (a result that would be expected to have one is warned of).
What a library call cannot see (types, shapes, devices) raises
ValueError here; the rest is LapError from the library.

A cache in 4 or 8 bits an element is a pair of torch.uint8 tensors [batch, kv_heads, slots, packed_row_bytes], strides that are
multiples of 16; a call knows the bits by that size.  cache_evict and cache_insert take such rows as well.
"""
from __future__ import annotations

import ctypes as C
import struct
import warnings
from types import SimpleNamespace
from typing import Optional

from . import binding

AT_FORWARD, AT_GRAD, AT_WEIGHTS, AT_STEP, AT_STEP_PACKED, AT_STEP_PACKED_UNWEIGHTED = range(6)


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64), ("row", C.c_int64)]


class _Shape(C.Structure):
    _fields_ = [("type", C.c_uint32), ("batch", C.c_uint32), ("q_heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("q_len", C.c_uint32), ("k_len", C.c_uint32), ("head_dim", C.c_uint32), ("causal", C.c_uint32),
                ("window", C.c_uint32), ("scale", C.c_float), ("q_lens", C.c_void_p), ("k_lens", C.c_void_p)]


class _Cache(C.Structure):
    _fields_ = [("type", C.c_uint32), ("batch", C.c_uint32), ("kv_heads", C.c_uint32), ("slots", C.c_uint32),
                ("head_dim", C.c_uint32), ("k", _Rows), ("v", _Rows), ("weights", C.c_void_p), ("positions", C.c_void_p)]


class _Packed(C.Structure):
    _fields_ = [("type", C.c_uint32), ("bits", C.c_uint32), ("batch", C.c_uint32), ("kv_heads", C.c_uint32), ("slots", C.c_uint32),
                ("head_dim", C.c_uint32), ("k", _Rows), ("v", _Rows)]


torch = None      # set when the library is loaded, which loads torch first

# The same structures as bytes, which a call's arguments are put together from: that and its checks are what the smallest
# calls take longest for, and a ctypes object is twice as long in the making.
_pack_rows = struct.Struct("@P3q").pack
_pack_shape = struct.Struct("@9If2P").pack
_pack_cache = struct.Struct("@5I4x").pack
_pack_two = struct.Struct("@2P").pack
_pack_pair = struct.Struct("@P3qP3q").pack
_pack_packed = struct.Struct("@6IP3qP3q").pack
_NOWHERE = _pack_rows(0, 0, 0, 0)
_ROWS = len(_NOWHERE)
assert len(_NOWHERE) == C.sizeof(_Rows) and len(_pack_shape(*[0] * 12)) == C.sizeof(_Shape)
assert len(_pack_cache(*[0] * 5) + 2 * _NOWHERE + _pack_two(0, 0)) == C.sizeof(_Cache)
assert len(_pack_packed(*[0] * 14)) == C.sizeof(_Packed) and _pack_pair(*range(8)) == _pack_rows(0, 1, 2, 3) + _pack_rows(4, 5, 6, 7)

_calls = SimpleNamespace()      # the library's calls, which take those bytes


def declare(lib) -> None:
    global torch, _stream, _device, _kinds, _moved
    import torch
    _kinds = {torch.bfloat16: 0, torch.float16: 1}
    _moved = dict(_kinds)
    _moved[torch.uint8] = 2
    # the handle alone, where torch has a call for it: a stream object takes 2 us to make
    _stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    p, u32, size, rows, shape, cache = C.c_void_p, C.c_uint32, C.c_size_t, C.POINTER(_Rows), C.POINTER(_Shape), C.POINTER(_Cache)
    packed = C.POINTER(_Packed)
    ws = [p, size, p]
    for name, result, args in (("lap_attention_workspace_bytes", size, [C.c_int, shape]),
                               ("lap_cache_workspace_bytes", size, [cache]),
                               ("lap_attention", C.c_int, [shape, rows, rows, rows, rows, p] + ws),
                               ("lap_attention_grad", C.c_int, [shape] + [rows] * 5 + [p] + [rows] * 3 + ws),
                               ("lap_attention_weights", C.c_int, [shape, rows, rows, p, p, p] + ws),
                               ("lap_attention_step", C.c_int, [shape, rows, rows, rows, p, p, rows, p, p] + ws),
                               ("lap_cache_evict", C.c_int, [cache, p, u32, u32, cache, p] + ws),
                               ("lap_cache_insert", C.c_int, [cache, rows, rows, p, u32, p, p]),
                               ("lap_packed_row_bytes", size, [u32, u32]),
                               ("lap_cache_pack", C.c_int, [packed, rows, rows, u32, p, p, p]),
                               ("lap_cache_unpack", C.c_int, [packed, u32, p, p, rows, rows, p]),
                               ("lap_attention_step_packed", C.c_int, [shape, rows, packed, p, p, rows, p, p] + ws)):
        call = getattr(lib, name)
        call.restype, call.argtypes = result, args
        call = lib[name]
        call.restype, call.argtypes = result, [p if x in (rows, shape, cache, packed) else x for x in args]
        setattr(_calls, name, call)


def _lib():
    if binding._lib is None:
        binding.load_library()
    return _calls


def _on(index: int, call, *args) -> int:
    """The call with its tensors' GPU as the current one, which is where the library launches (every GPU's default stream has
    the same handle)."""
    if _device() == index:
        return call(*args)
    with torch.cuda.device(index):
        return call(*args)


def _warn_of_autograd(name: str, where: str) -> None:
    if torch.is_grad_enabled():
        warnings.warn(f"{name}: the result has no gradient for autograd; {where}", stacklevel=3)


def _done(rc: int, where: str, index: int, sync: bool) -> None:
    if rc:
        raise binding.LapError(rc, where)
    if sync:
        torch.cuda.current_stream(index).synchronize()


# A call's arguments are looked at on every call, of a few microseconds each: the texts of refusals are put together only
# where one is due.

def _refuse(name: str, x, expected) -> None:
    raise ValueError(f"{name}: {tuple(x.shape)} {x.dtype} on {x.device} with strides {x.stride()}, expected {expected}")


def _rows(x, name: str, dtype, shape, index: int):
    """lap_rows of x, which has to be a tensor of this type and shape on this GPU, elements of a row side by side."""
    if x.dtype is not dtype or x.shape != shape or x.get_device() != index:
        _refuse(name, x, f"{tuple(shape)} {dtype} on GPU {index}")
    st = x.stride()
    if st[-1] != 1 and x.numel():
        _refuse(name, x, "the elements of a row side by side")
    return _pack_rows(x.data_ptr(), st[0], st[1], st[2] if len(st) == 4 else 0)


def _plain(x, name: str, dtype, shape, index: int):
    """Address of a contiguous tensor of this type and shape, None for None."""
    if x is None:
        return None
    if x.dtype is not dtype or x.shape != shape or x.get_device() != index or not x.is_contiguous():
        _refuse(name, x, f"a contiguous {dtype} of {tuple(shape)} on GPU {index}")
    return x.data_ptr()


def _type(x, name: str, kinds=None):
    """lap's number for x's type, the type, the GPU."""
    t, index = x.dtype, x.get_device()
    kind = (kinds or _kinds).get(t)
    if kind is None:
        _refuse(name, x, "torch.bfloat16 or torch.float16" + (" (packed rows: torch.uint8)" if kinds else ""))
    if index < 0:
        _refuse(name, x, "a tensor on the GPU")
    return kind, t, index


def _four(x, name: str):
    shape = x.shape
    if len(shape) != 4:
        _refuse(name, x, "[batch, heads, length, head_dim]")
    return shape


def _count(x, name: str) -> int:
    if not 0 <= x <= 0xFFFFFFFF or int(x) != x:      # what the library takes; its own limits are lower
        raise ValueError(f"{name} is a number of keys or slots, not {x}")
    return int(x)


def _scale(scale: Optional[float], d: int) -> float:
    return C.c_float(scale).value if scale is not None else d ** -0.5 if d else 0.0


def _shape(q, k, causal, window, scale, q_lens, k_lens):
    """lap_attention_shape, the type, the shapes of queries and keys, the GPU."""
    qs, ks = _four(q, "q"), _four(k, "k")
    b, h, n, d = qs
    _, kv, m, _ = ks
    kind, t, index = _type(q, "q")
    s = _pack_shape(kind, b, h, kv, n, m, d, 1 if causal else 0, _count(window, "window") if window else 0, _scale(scale, d),
                    0 if q_lens is None else _plain(q_lens, "q_lens", torch.int32, (b,), index),
                    0 if k_lens is None else _plain(k_lens, "k_lens", torch.int32, (b,), index))
    return s, t, qs, (b, kv, m, d), index


def _workspace(ws, need: int, index: int, like):
    """The workspace, its size and its address."""
    if ws is None:
        if not need:
            return None, 0, None
        ws = like.new_empty(need, dtype=torch.uint8)
    elif ws.dtype is not torch.uint8 or ws.get_device() != index or not ws.is_contiguous():
        _refuse("ws", ws, f"a contiguous torch.uint8 on GPU {index}")
    return ws, ws.numel(), ws.data_ptr()


def attention_workspace_bytes(which: int, q_shape, kv_shape, dtype, *, causal: bool = False) -> int:
    """lap_attention_workspace_bytes: of a call (AT_FORWARD, AT_GRAD, AT_WEIGHTS, AT_STEP, AT_STEP_PACKED, or of a packed step without
    weights AT_STEP_PACKED_UNWEIGHTED) on queries and keys of these shapes, [batch, heads, length, head_dim], for a step's queries without a length.  dtype and head_dim are the elements',
    also of a packed cache.  0: none, also where the call is refused."""
    lib = _lib()
    b, h, *n, d = q_shape
    s = _pack_shape(_kinds[dtype], b, h, kv_shape[1], n[0] if n else 1, kv_shape[2], d, 1 if causal or which >= AT_STEP_PACKED else 0, 0,
                    1.0, 0, 0)
    return int(lib.lap_attention_workspace_bytes(which, s))


def attention(q, k, v, *, causal: bool = False, window: int = 0, scale: Optional[float] = None, q_lens=None, k_lens=None,
              out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention: returns dict(out like q, lse [batch, q_heads, q_len]), without gradients for autograd.  scale None:
    1 / sqrt(head_dim)."""
    lib = _lib()
    if q.requires_grad or k.requires_grad or v.requires_grad:
        _warn_of_autograd("attention", "attention_grad computes that of q, k and v")
    s, t, qs, kv, index = _shape(q, k, causal, window, scale, q_lens, k_lens)
    if out is None:
        out = dict(out=torch.empty_like(q), lse=q.new_empty(qs[:3], dtype=torch.float32))
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_FORWARD, s), index, q)
    rc = _on(index, lib.lap_attention, s, _rows(q, "q", t, qs, index), _rows(k, "k", t, kv, index), _rows(v, "v", t, kv, index),
             _rows(out["out"], "out", t, qs, index), _plain(out["lse"], "lse", torch.float32, qs[:3], index),
             at, have, _stream(index))
    if rc or sync:
        _done(rc, "lap_attention", index, sync)
    return out


def attention_grad(dout, q, k, v, out, lse, *, causal: bool = False, window: int = 0, scale: Optional[float] = None, q_lens=None,
                   k_lens=None, grads: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention_grad: returns dict(dq, dk, dv); out and lse are attention's, the other arguments as there.  grads takes
    result tensors that the caller owns."""
    lib = _lib()
    s, t, qs, kv, index = _shape(q, k, causal, window, scale, q_lens, k_lens)
    if grads is None:
        grads = dict(dq=torch.empty_like(q), dk=q.new_empty(kv), dv=q.new_empty(kv))
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_GRAD, s), index, q)
    rc = _on(index, lib.lap_attention_grad, s, _rows(dout, "dout", t, qs, index), _rows(q, "q", t, qs, index), _rows(k, "k", t, kv, index),
             _rows(v, "v", t, kv, index), _rows(out, "out", t, qs, index),
             _plain(lse, "lse", torch.float32, qs[:3], index), _rows(grads["dq"], "dq", t, qs, index),
             _rows(grads["dk"], "dk", t, kv, index), _rows(grads["dv"], "dv", t, kv, index),
             at, have, _stream(index))
    if rc or sync:
        _done(rc, "lap_attention_grad", index, sync)
    return grads


def attention_weights(q, k, lse, *, before=None, causal: bool = False, window: int = 0, scale: Optional[float] = None, q_lens=None,
                      k_lens=None, weights=None, ws=None, sync: bool = True):
    """lap_attention_weights: returns dict(weights [batch, kv_heads, k_len]) = before (None: zeros) + what the keys receive."""
    lib = _lib()
    s, t, qs, ks, index = _shape(q, k, causal, window, scale, q_lens, k_lens)
    kv = ks[:3]
    if weights is None:
        weights = q.new_empty(kv, dtype=torch.float32)
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_WEIGHTS, s), index, q)
    rc = _on(index, lib.lap_attention_weights, s, _rows(q, "q", t, qs, index), _rows(k, "k", t, ks, index),
             _plain(lse, "lse", torch.float32, qs[:3], index), _plain(before, "before", torch.float32, kv, index),
             _plain(weights, "weights", torch.float32, kv, index), at, have, _stream(index))
    if rc or sync:
        _done(rc, "lap_attention_weights", index, sync)
    return dict(weights=weights)


def attention_step(q, k_cache, v_cache, weights=None, *, lens=None, positions=None, scale: Optional[float] = None,
                   out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention_step: q [batch, q_heads, head_dim] of one token against caches [batch, kv_heads, slots, head_dim].  Returns
    dict(out like q, lse [batch, q_heads], weights = the given ones + this token's, a new tensor unless out holds one; None
    where none are given)."""
    lib = _lib()
    if q.requires_grad or k_cache.requires_grad or v_cache.requires_grad:
        _warn_of_autograd("attention_step", "there is none of a step")
    if q.dim() != 3:
        _refuse("q", q, "[batch, heads, head_dim]")
    qs, ks = q.shape, _four(k_cache, "k_cache")
    b, h, d = qs
    _, kv, n, _ = ks
    kind, t, index = _type(q, "q")
    s = _pack_shape(kind, b, h, kv, 1, n, d, 0, 0, _scale(scale, d), 0, _plain(lens, "lens", torch.int32, (b,), index) or 0)
    slots, kv = (b, kv, n), (b, kv, n, d)
    if out is None:
        out = dict(out=torch.empty_like(q), lse=q.new_empty((b, h), dtype=torch.float32),
                   weights=None if weights is None else q.new_empty(slots, dtype=torch.float32))
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_STEP, s), index, q)
    rc = _on(index, lib.lap_attention_step, s, _rows(q, "q", t, qs, index), _rows(k_cache, "k_cache", t, kv, index), _rows(v_cache, "v_cache", t, kv, index),
             _plain(positions, "positions", torch.int32, slots, index), _plain(weights, "weights", torch.float32, slots, index),
             _rows(out["out"], "out", t, qs, index), _plain(out["lse"], "lse", torch.float32, (b, h), index),
             _plain(out.get("weights"), "out weights", torch.float32, slots, index), at, have, _stream(index))
    if rc or sync:
        _done(rc, "lap_attention_step", index, sync)
    return out


def _cache(k, v, weights, positions, name: str = ""):
    b, h, n, d = shape = _four(k, name + "k")
    kind, t, index = _type(k, name + "k", _moved)
    slots = (b, h, n)
    return (_pack_cache(kind, b, h, n, d) + _rows(k, name + "k", t, shape, index) + _rows(v, name + "v", t, shape, index)
            + _pack_two(_plain(weights, name + "weights", torch.float32, slots, index) or 0,
                        _plain(positions, name + "positions", torch.int32, slots, index) or 0))


def cache_evict(k, v, weights, keep: int, recent: int, *, lens=None, positions=None, slots: Optional[int] = None,
                out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_cache_evict: the `keep` rows of highest weight of k and v, the newest `recent` among them, into a cache of `slots`
    (None: keep).  Returns dict(k, v, weights, positions [batch, kv_heads, slots], lens [batch]: the lengths given, up to keep).
    Where a head has fewer slots in use than that, only `positions` tells attention_step which are empty."""
    lib = _lib()
    src = _cache(k, v, weights, positions)
    keep, recent = _count(keep, "keep"), _count(recent, "recent")
    b, h, n, d = k.shape
    index = k.get_device()
    if out is None:
        m = keep if slots is None else _count(slots, "slots")
        out = dict(k=k.new_empty((b, h, m, d)), v=k.new_empty((b, h, m, d)), weights=k.new_empty((b, h, m), dtype=torch.float32),
                   positions=k.new_empty((b, h, m), dtype=torch.int32), lens=k.new_empty(b, dtype=torch.int32))
    if out["k"].dtype is not k.dtype or out["k"].get_device() != index:
        _refuse("out k", out["k"], f"{k.dtype} on GPU {index}")
    dst = _cache(out["k"], out["v"], out["weights"], out["positions"], "out ")
    ws, have, at = _workspace(ws, lib.lap_cache_workspace_bytes(dst), index, k)
    rc = _on(index, lib.lap_cache_evict, src, _plain(lens, "lens", torch.int32, (b,), index), keep, recent, dst,
             _plain(out["lens"], "out lens", torch.int32, (b,), index), at, have, _stream(index))
    if rc or sync:
        _done(rc, "lap_cache_evict", index, sync)
    return out


def cache_insert(k_new, v_new, k_cache, v_cache, weights, positions, position, recent: int, *, slots=None, sync: bool = True):
    """lap_cache_insert: one token [batch, kv_heads, head_dim] into every cache, in place; position [batch] is the token's.
    Returns dict(slots [batch, kv_heads]): where it went."""
    lib = _lib()
    cache = _cache(k_cache, v_cache, weights, positions)
    b, h, _, d = k_cache.shape
    index = k_cache.get_device()
    if slots is None:
        slots = k_cache.new_empty((b, h), dtype=torch.int32)
    rc = _on(index, lib.lap_cache_insert, cache, _rows(k_new, "k_new", k_cache.dtype, (b, h, d), index), _rows(v_new, "v_new", k_cache.dtype, (b, h, d), index),
             _plain(position, "position", torch.int32, (b,), index), _count(recent, "recent"),
             _plain(slots, "slots", torch.int32, (b, h), index), _stream(index))
    if rc or sync:
        _done(rc, "lap_cache_insert", index, sync)
    return dict(slots=slots)


_row_bits = {}      # (bytes of a row, head_dim): bits


def packed_row_bytes(bits: int, head_dim: int) -> int:
    """lap_packed_row_bytes: of a row of head_dim elements in 4 or 8 bits each."""
    need = int(_lib().lap_packed_row_bytes(_count(bits, "bits"), _count(head_dim, "head_dim")))
    if not need:
        raise ValueError(f"there are no packed rows of {head_dim} elements in {bits} bits: 4 or 8 bits, a multiple of 8 up to 128 elements")
    return need


_CACHE, _OUT = ("k_cache", "v_cache"), ("out k_cache", "out v_cache")


def _pair(k, v, names, dtype, shape, index: int):
    """Address and strides of k, then of v, tensors of [batch, heads, length, elements] that are as _rows wants them."""
    if not (k.dtype is dtype is v.dtype and k.shape == shape == v.shape and k.get_device() == index == v.get_device()):
        _rows(k, names[0], dtype, shape, index), _rows(v, names[1], dtype, shape, index)
    a, b = k.stride(), v.stride()
    if a[3] != 1 or b[3] != 1:
        _rows(k, names[0], dtype, shape, index), _rows(v, names[1], dtype, shape, index)
    return k.data_ptr(), a[0], a[1], a[2], v.data_ptr(), b[0], b[1], b[2]


def _packed(kind: int, d: int, k, v, index: int, names=_CACHE):
    """lap_packed_cache of rows of bytes that stand for d elements each, the shape of the rows."""
    shape = k.shape
    if len(shape) != 4:
        _refuse(names[0], k, "[batch, heads, length, bytes of a row]")
    b, h, n, row = shape
    bits = _row_bits.get((row, d))
    if bits is None:
        for bits in (4, 8):
            if _lib().lap_packed_row_bytes(bits, d) == row:
                break
        else:
            _refuse(names[0], k, f"rows of packed_row_bytes of 4 or 8 bits and {d} elements")
        _row_bits[row, d] = bits
    return _pack_packed(kind, bits, b, h, n, d, *_pair(k, v, names, torch.uint8, shape, index)), shape


def cache_pack(k, v, bits: Optional[int] = None, *, lens=None, first=None, slots: Optional[int] = None, out: Optional[dict] = None,
               sync: bool = True):
    """lap_cache_pack: rows k and v [batch, kv_heads, length, head_dim] into a cache in `bits` (4 or 8) an element, row i of sequence b into
    slot first[b] + i (None: i).  Returns dict(k, v), the cache: out's, whose other slots stay as they are, or a new one of
    `slots` slots (None: length), zeros elsewhere."""
    lib = _lib()
    if k.requires_grad or v.requires_grad:
        _warn_of_autograd("cache_pack", "there is none of a cache")
    b, h, n, d = shape = _four(k, "k")
    kind, t, index = _type(k, "k")
    if out is None:
        if bits is None:
            raise ValueError("cache_pack: bits, or out, says how many an element takes")
        m, row = n if slots is None else _count(slots, "slots"), packed_row_bytes(bits, d)
        out = dict(k=k.new_zeros((b, h, m, row), dtype=torch.uint8), v=k.new_zeros((b, h, m, row), dtype=torch.uint8))
    elif slots is not None:
        raise ValueError("cache_pack: the slots are out's")
    cache, rows = _packed(kind, d, out["k"], out["v"], index, _OUT)
    if rows[0] != b or rows[1] != h or (bits is not None and rows[3] != packed_row_bytes(bits, d)):
        _refuse("out k_cache", out["k"], f"a cache of {b} sequences and {h} heads" + (f" in {bits} bits" if bits is not None else ""))
    rows = _pack_pair(*_pair(k, v, "kv", t, shape, index))
    args = (cache, rows, rows[_ROWS:], n, _plain(lens, "lens", torch.int32, (b,), index), _plain(first, "first", torch.int32, (b,), index), _stream(index))
    rc = lib.lap_cache_pack(*args) if _device() == index else _on(index, lib.lap_cache_pack, *args)
    if rc or sync:
        _done(rc, "lap_cache_pack", index, sync)
    return out


def cache_unpack(k_cache, v_cache, dtype, head_dim: int, *, lens=None, first=None, length: Optional[int] = None, out: Optional[dict] = None,
                 sync: bool = True):
    """lap_cache_unpack: what the slots first[b] + i of a packed cache stand for, as rows [batch, kv_heads, length, head_dim] of dtype
    (None: as many as there are slots); rows i from lens[b] on are zeros.  Returns dict(k, v)."""
    lib = _lib()
    kind = _kinds.get(dtype)
    if kind is None:
        raise ValueError(f"cache_unpack: {dtype}, expected torch.bfloat16 or torch.float16")
    index = k_cache.get_device()
    if index < 0:
        _refuse("k_cache", k_cache, "a tensor on the GPU")
    d = _count(head_dim, "head_dim")
    cache, (b, h, m, _) = _packed(kind, d, k_cache, v_cache, index)
    n = m if length is None else _count(length, "length")
    shape = (b, h, n, d)
    if out is None:      # contiguous, and nothing to check
        k = k_cache.new_empty(shape, dtype=dtype)
        v, row = torch.empty_like(k), n * d
        out = dict(k=k, v=v)
        rows = _pack_pair(k.data_ptr(), h * row, row, d, v.data_ptr(), h * row, row, d)
    else:
        rows = _pack_pair(*_pair(out["k"], out["v"], ("out k", "out v"), dtype, shape, index))
    args = (cache, n, _plain(lens, "lens", torch.int32, (b,), index), _plain(first, "first", torch.int32, (b,), index), rows, rows[_ROWS:], _stream(index))
    rc = lib.lap_cache_unpack(*args) if _device() == index else _on(index, lib.lap_cache_unpack, *args)
    if rc or sync:
        _done(rc, "lap_cache_unpack", index, sync)
    return out


def attention_step_packed(q, k_cache, v_cache, weights=None, *, lens=None, positions=None, q_lens=None, scale: Optional[float] = None,
                          out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention_step_packed: attention_step on a packed cache, for q [batch, q_heads, head_dim] of one token of every sequence, or
    [batch, q_heads, tokens, head_dim] of its last few, whose keys and values are in the cache already (q_lens: how many of them are in
    use).  Returns dict(out like q, lse [batch, q_heads] or [batch, q_heads, tokens], weights as there)."""
    lib = _lib()
    if q.requires_grad:
        _warn_of_autograd("attention_step_packed", "there is none of a step")
    qs = q.shape
    if len(qs) not in (3, 4):
        _refuse("q", q, "[batch, heads, head_dim] or [batch, heads, tokens, head_dim]")
    b, h, d = qs[0], qs[1], qs[-1]
    tokens = qs[2] if len(qs) == 4 else None
    kind, t, index = _type(q, "q")
    cache, (cb, kv, n, _) = _packed(kind, d, k_cache, v_cache, index)
    if cb != b:
        _refuse("k_cache", k_cache, f"a cache of {b} sequences")
    s = _pack_shape(kind, b, h, kv, 1 if tokens is None else tokens, n, d, 1, 0, _scale(scale, d), 0 if q_lens is None else _plain(q_lens, "q_lens", torch.int32, (b,), index),
                    0 if lens is None else _plain(lens, "lens", torch.int32, (b,), index))
    slots, lse = (b, kv, n), (b, h) if tokens is None else (b, h, tokens)
    before = _plain(weights, "weights", torch.float32, slots, index)
    if out is None:      # nothing to check
        o, sums = torch.empty_like(q), q.new_empty(lse, dtype=torch.float32)
        after = None if weights is None else torch.empty_like(weights)
        out = dict(out=o, lse=sums, weights=after)
        st = o.stride()
        results = _pack_rows(o.data_ptr(), st[0], st[1], st[2] if tokens is not None else 0), sums.data_ptr(), None if after is None else after.data_ptr()
    else:
        results = (_rows(out["out"], "out", t, qs, index), _plain(out["lse"], "lse", torch.float32, lse, index),
                   _plain(out.get("weights"), "out weights", torch.float32, slots, index))
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_STEP_PACKED_UNWEIGHTED if weights is None else AT_STEP_PACKED, s), index, q)
    args = (s, _rows(q, "q", t, qs, index), cache, _plain(positions, "positions", torch.int32, slots, index), before, *results, at, have, _stream(index))
    rc = lib.lap_attention_step_packed(*args) if _device() == index else _on(index, lib.lap_attention_step_packed, *args)
    if rc or sync:
        _done(rc, "lap_attention_step_packed", index, sync)
    return out
