"""ctypes binding of liblap's attention and cache operators: argument marshalling only.

Tensors are [batch, heads, length, head_dim] in torch.bfloat16 or torch.float16 with elements of a row side by side; other
strides are free (a [batch, length, heads, head_dim] tensor goes in as its transpose(1, 2)).  Lengths, positions and slots
are torch.int32, weights and logarithms of softmax sums torch.float32, all contiguous.  Work is enqueued on the current
stream of q's device; `sync=False` returns without waiting for it.  `out` takes result tensors that the caller owns, `ws` a
workspace (uint8, at least as large as the call asks for).  What a library call cannot see (types, shapes, devices) raises
ValueError here; the rest is LapError from the library.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

from . import binding

AT_FORWARD, AT_GRAD, AT_WEIGHTS, AT_STEP = range(4)


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64), ("row", C.c_int64)]


class _Shape(C.Structure):
    _fields_ = [("type", C.c_uint32), ("batch", C.c_uint32), ("q_heads", C.c_uint32), ("kv_heads", C.c_uint32),
                ("q_len", C.c_uint32), ("k_len", C.c_uint32), ("head_dim", C.c_uint32), ("causal", C.c_uint32),
                ("window", C.c_uint32), ("scale", C.c_float), ("q_lens", C.c_void_p), ("k_lens", C.c_void_p)]


class _Cache(C.Structure):
    _fields_ = [("type", C.c_uint32), ("batch", C.c_uint32), ("kv_heads", C.c_uint32), ("slots", C.c_uint32),
                ("head_dim", C.c_uint32), ("k", _Rows), ("v", _Rows), ("weights", C.c_void_p), ("positions", C.c_void_p)]


torch = None      # set when the library is loaded, which loads torch first


def declare(lib) -> None:
    global torch, _stream
    import torch
    # the handle alone, where torch has a call for it: a stream object takes 2 us to make
    _stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    p, rows, shape, cache = C.c_void_p, C.POINTER(_Rows), C.POINTER(_Shape), C.POINTER(_Cache)
    ws = [p, C.c_size_t, p]
    lib.lap_attention_workspace_bytes.restype = C.c_size_t
    lib.lap_attention_workspace_bytes.argtypes = [C.c_int, shape]
    lib.lap_cache_workspace_bytes.restype = C.c_size_t
    lib.lap_cache_workspace_bytes.argtypes = [cache]
    for name, args in (("lap_attention", [shape, rows, rows, rows, rows, p] + ws),
                       ("lap_attention_grad", [shape] + [rows] * 5 + [p] + [rows] * 3 + ws),
                       ("lap_attention_weights", [shape, rows, rows, p, p, p] + ws),
                       ("lap_attention_step", [shape, rows, rows, rows, p, p, rows, p, p] + ws),
                       ("lap_cache_evict", [cache, p, C.c_uint32, C.c_uint32, cache, p] + ws),
                       ("lap_cache_insert", [cache, rows, rows, p, C.c_uint32, p, p])):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = args


def _lib():
    return binding._lib or binding.load_library()


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
    return _Rows(x.data_ptr(), st[0], st[1], st[2] if len(st) == 4 else 0)


def _plain(x, name: str, dtype, shape, index: int):
    """Address of a contiguous tensor of this type and shape, None for None."""
    if x is None:
        return None
    if x.dtype is not dtype or x.shape != shape or x.get_device() != index or not x.is_contiguous():
        _refuse(name, x, f"a contiguous {dtype} of {tuple(shape)} on GPU {index}")
    return x.data_ptr()


def _type(x, name: str) -> int:
    if x.dtype is torch.bfloat16:
        kind = 0
    elif x.dtype is torch.float16:
        kind = 1
    else:
        _refuse(name, x, "torch.bfloat16 or torch.float16")
    if not x.is_cuda:
        _refuse(name, x, "a tensor on the GPU")
    return kind


def _four(x, name: str):
    if x.dim() != 4:
        _refuse(name, x, "[batch, heads, length, head_dim]")
    return x.shape


def _scale(scale: Optional[float], d: int) -> float:
    return float(scale) if scale is not None else d ** -0.5 if d else 0.0


def _shape(q, k, causal, window, scale, q_lens, k_lens):
    """lap_attention_shape, the type, the shapes of queries and keys, the GPU."""
    qs, ks = _four(q, "q"), _four(k, "k")
    b, h, n, d = qs
    _, kv, m, _ = ks
    kind, index = _type(q, "q"), q.get_device()
    if window < 0:
        raise ValueError("window is 0 (none) or a number of keys")
    i32 = torch.int32
    s = _Shape(kind, b, h, kv, n, m, d, 1 if causal else 0, window, _scale(scale, d),
               None if q_lens is None else _plain(q_lens, "q_lens", i32, (b,), index),
               None if k_lens is None else _plain(k_lens, "k_lens", i32, (b,), index))
    return s, q.dtype, qs, (b, kv, m, d), index


def _workspace(ws, need: int, index: int):
    """The workspace, its size and its address."""
    if ws is None:
        if not need:
            return None, 0, None
        ws = torch.empty(need, dtype=torch.uint8, device=index)
    elif ws.dtype is not torch.uint8 or ws.get_device() != index or not ws.is_contiguous():
        _refuse("ws", ws, f"a contiguous torch.uint8 on GPU {index}")
    return ws, ws.numel(), ws.data_ptr()


def attention(q, k, v, *, causal: bool = False, window: int = 0, scale: Optional[float] = None, q_lens=None, k_lens=None,
              out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention: returns dict(out like q, lse [batch, q_heads, q_len]).  scale None: 1 / sqrt(head_dim)."""
    lib = _lib()
    s, t, qs, kv, index = _shape(q, k, causal, window, scale, q_lens, k_lens)
    if out is None:
        out = dict(out=torch.empty_like(q), lse=torch.empty(qs[:3], dtype=torch.float32, device=index))
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_FORWARD, s), index)
    rc = lib.lap_attention(s, _rows(q, "q", t, qs, index), _rows(k, "k", t, kv, index), _rows(v, "v", t, kv, index),
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
        grads = dict(dq=torch.empty_like(q), dk=torch.empty(kv, dtype=t, device=index),
                     dv=torch.empty(kv, dtype=t, device=index))
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_GRAD, s), index)
    rc = lib.lap_attention_grad(s, _rows(dout, "dout", t, qs, index), _rows(q, "q", t, qs, index), _rows(k, "k", t, kv, index),
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
        weights = torch.empty(kv, dtype=torch.float32, device=index)
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_WEIGHTS, s), index)
    rc = lib.lap_attention_weights(s, _rows(q, "q", t, qs, index), _rows(k, "k", t, ks, index),
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
    if q.dim() != 3:
        _refuse("q", q, "[batch, heads, head_dim]")
    qs, ks = q.shape, _four(k_cache, "k_cache")
    b, h, d = qs
    _, kv, n, _ = ks
    kind, t, index = _type(q, "q"), q.dtype, q.get_device()
    slots, kv = (b, kv, n), (b, kv, n, d)
    s = _Shape(kind, b, h, kv[1], 1, n, d, 0, 0, _scale(scale, d), None, _plain(lens, "lens", torch.int32, (b,), index))
    if out is None:
        out = dict(out=torch.empty_like(q), lse=torch.empty((b, h), dtype=torch.float32, device=index),
                   weights=None if weights is None else torch.empty(slots, dtype=torch.float32, device=index))
    ws, have, at = _workspace(ws, lib.lap_attention_workspace_bytes(AT_STEP, s), index)
    rc = lib.lap_attention_step(s, _rows(q, "q", t, qs, index), _rows(k_cache, "k_cache", t, kv, index), _rows(v_cache, "v_cache", t, kv, index),
                                _plain(positions, "positions", torch.int32, slots, index), _plain(weights, "weights", torch.float32, slots, index),
                                _rows(out["out"], "out", t, qs, index), _plain(out["lse"], "lse", torch.float32, (b, h), index),
                                _plain(out.get("weights"), "out weights", torch.float32, slots, index), at, have, _stream(index))
    if rc or sync:
        _done(rc, "lap_attention_step", index, sync)
    return out


def _cache(k, v, weights, positions, name: str = ""):
    b, h, n, d = shape = _four(k, name + "k")
    kind, t, index = _type(k, name + "k"), k.dtype, k.get_device()
    return _Cache(kind, b, h, n, d, _rows(k, name + "k", t, shape, index), _rows(v, name + "v", t, shape, index),
                  _plain(weights, name + "weights", torch.float32, (b, h, n), index),
                  _plain(positions, name + "positions", torch.int32, (b, h, n), index))


def cache_evict(k, v, weights, keep: int, recent: int, *, lens=None, positions=None, slots: Optional[int] = None,
                out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_cache_evict: the `keep` rows of highest weight of k and v, the newest `recent` among them, into a cache of `slots`
    (None: keep).  Returns dict(k, v, weights, positions [batch, kv_heads, slots], lens [batch])."""
    lib = _lib()
    src = _cache(k, v, weights, positions)
    if keep < 0 or recent < 0:
        raise ValueError("keep and recent are numbers of slots")
    b, h, n, d = k.shape
    index = k.get_device()
    if out is None:
        m = int(keep if slots is None else slots)
        out = dict(k=torch.empty((b, h, m, d), dtype=k.dtype, device=index), v=torch.empty((b, h, m, d), dtype=k.dtype, device=index),
                   weights=torch.empty((b, h, m), dtype=torch.float32, device=index),
                   positions=torch.empty((b, h, m), dtype=torch.int32, device=index), lens=torch.empty(b, dtype=torch.int32, device=index))
    if out["k"].dtype is not k.dtype or out["k"].get_device() != index:
        _refuse("out k", out["k"], f"{k.dtype} on GPU {index}")
    dst = _cache(out["k"], out["v"], out["weights"], out["positions"], "out ")
    ws, have, at = _workspace(ws, lib.lap_cache_workspace_bytes(dst), index)
    rc = lib.lap_cache_evict(src, _plain(lens, "lens", torch.int32, (b,), index), int(keep), int(recent), dst,
                             _plain(out["lens"], "out lens", torch.int32, (b,), index), at, have, _stream(index))
    if rc or sync:
        _done(rc, "lap_cache_evict", index, sync)
    return out


def cache_insert(k_new, v_new, k_cache, v_cache, weights, positions, position, recent: int, *, slots=None, sync: bool = True):
    """lap_cache_insert: one token [batch, kv_heads, head_dim] into every cache, in place; position [batch] is the token's.
    Returns dict(slots [batch, kv_heads]): where it went."""
    lib = _lib()
    cache = _cache(k_cache, v_cache, weights, positions)
    if recent < 0:
        raise ValueError("recent is a number of slots")
    b, h, _, d = k_cache.shape
    index = k_cache.get_device()
    if slots is None:
        slots = torch.empty((b, h), dtype=torch.int32, device=index)
    rc = lib.lap_cache_insert(cache, _rows(k_new, "k_new", k_cache.dtype, (b, h, d), index), _rows(v_new, "v_new", k_cache.dtype, (b, h, d), index),
                              _plain(position, "position", torch.int32, (b,), index), int(recent),
                              _plain(slots, "slots", torch.int32, (b, h), index), _stream(index))
    if rc or sync:
        _done(rc, "lap_cache_insert", index, sync)
    return dict(slots=slots)
