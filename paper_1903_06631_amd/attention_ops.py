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
import math
from typing import Optional

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


def declare(lib) -> None:
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
    from .binding import load_library
    return load_library()


def _torch():
    import torch
    return torch


def _done(rc: int, where: str, torch, device, sync: bool) -> None:
    if rc:
        from .binding import LapError
        raise LapError(rc, where)
    if sync:
        torch.cuda.current_stream(device).synchronize()


def _check(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _rows(x, name: str, like, shape):
    """lap_rows of x, which has to be a tensor of this shape and of like's type and device."""
    _check(x.dtype == like.dtype and x.device == like.device, f"{name}: {x.dtype} on {x.device}, expected {like.dtype} on {like.device}")
    _check(tuple(x.shape) == tuple(shape), f"{name}: shape {tuple(x.shape)}, expected {tuple(shape)}")
    st = x.stride()
    _check(st[-1] == 1 or x.numel() == 0, f"{name}: the elements of a row have to lie side by side")
    return _Rows(x.data_ptr(), st[0], st[1], st[2] if len(shape) == 4 else 0)


def _plain(x, name: str, dtype, shape, device):
    """Address of a contiguous tensor of this type and shape, None for None."""
    if x is None:
        return None
    _check(x.dtype == dtype and x.device == device and tuple(x.shape) == tuple(shape) and x.is_contiguous(),
           f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return x.data_ptr()


def _type(torch, x) -> int:
    _check(x.is_cuda, "tensors have to be on the GPU")
    _check(x.dtype in (torch.bfloat16, torch.float16), f"{x.dtype}: expected torch.bfloat16 or torch.float16")
    return 0 if x.dtype == torch.bfloat16 else 1


def _shape(torch, q, k, causal, window, scale, q_lens, k_lens):
    _check(q.dim() == 4 and k.dim() == 4, "q and k are [batch, heads, length, head_dim]")
    b, h, n, d = q.shape
    kind = _type(torch, q)
    _check(window >= 0, "window is 0 (none) or a number of keys")
    return _Shape(kind, b, h, k.shape[1], n, k.shape[2], d, bool(causal), int(window),
                  1.0 / math.sqrt(d) if scale is None and d else (scale or 0.0),
                  _plain(q_lens, "q_lens", torch.int32, (b,), q.device), _plain(k_lens, "k_lens", torch.int32, (b,), q.device))


def _workspace(torch, ws, need: int, device):
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    elif need:
        _check(ws.dtype == torch.uint8 and ws.device == device and ws.is_contiguous(), "ws: expected contiguous torch.uint8 on the tensors' device")
    return ws, (0 if ws is None else ws.numel()), (None if ws is None else ws.data_ptr())


def _stream(torch, device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def attention(q, k, v, *, causal: bool = False, window: int = 0, scale: Optional[float] = None, q_lens=None, k_lens=None,
              out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention: returns dict(out like q, lse [batch, q_heads, q_len]).  scale None: 1 / sqrt(head_dim)."""
    torch, lib = _torch(), _lib()
    s = _shape(torch, q, k, causal, window, scale, q_lens, k_lens)
    kv = (s.batch, s.kv_heads, s.k_len, s.head_dim)
    if out is None:
        out = dict(out=torch.empty_like(q), lse=torch.empty(q.shape[:3], dtype=torch.float32, device=q.device))
    ws, have, at = _workspace(torch, ws, lib.lap_attention_workspace_bytes(AT_FORWARD, s), q.device)
    rc = lib.lap_attention(s, _rows(q, "q", q, q.shape), _rows(k, "k", q, kv), _rows(v, "v", q, kv),
                           _rows(out["out"], "out", q, q.shape), _plain(out["lse"], "lse", torch.float32, q.shape[:3], q.device),
                           at, have, _stream(torch, q.device))
    _done(rc, "lap_attention", torch, q.device, sync)
    return out


def attention_grad(dout, q, k, v, out, lse, *, causal: bool = False, window: int = 0, scale: Optional[float] = None, q_lens=None,
                   k_lens=None, grads: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention_grad: returns dict(dq, dk, dv); out and lse are attention's, the other arguments as there.  grads takes
    result tensors that the caller owns."""
    torch, lib = _torch(), _lib()
    s = _shape(torch, q, k, causal, window, scale, q_lens, k_lens)
    kv = (s.batch, s.kv_heads, s.k_len, s.head_dim)
    if grads is None:
        grads = dict(dq=torch.empty_like(q), dk=torch.empty(kv, dtype=q.dtype, device=q.device),
                     dv=torch.empty(kv, dtype=q.dtype, device=q.device))
    ws, have, at = _workspace(torch, ws, lib.lap_attention_workspace_bytes(AT_GRAD, s), q.device)
    rc = lib.lap_attention_grad(s, _rows(dout, "dout", q, q.shape), _rows(q, "q", q, q.shape), _rows(k, "k", q, kv), _rows(v, "v", q, kv),
                                _rows(out, "out", q, q.shape), _plain(lse, "lse", torch.float32, q.shape[:3], q.device),
                                _rows(grads["dq"], "dq", q, q.shape), _rows(grads["dk"], "dk", q, kv), _rows(grads["dv"], "dv", q, kv),
                                at, have, _stream(torch, q.device))
    _done(rc, "lap_attention_grad", torch, q.device, sync)
    return grads


def attention_weights(q, k, lse, *, before=None, causal: bool = False, window: int = 0, scale: Optional[float] = None, q_lens=None,
                      k_lens=None, weights=None, ws=None, sync: bool = True):
    """lap_attention_weights: returns dict(weights [batch, kv_heads, k_len]) = before (None: zeros) + what the keys receive."""
    torch, lib = _torch(), _lib()
    s = _shape(torch, q, k, causal, window, scale, q_lens, k_lens)
    kv = (s.batch, s.kv_heads, s.k_len)
    if weights is None:
        weights = torch.empty(kv, dtype=torch.float32, device=q.device)
    ws, have, at = _workspace(torch, ws, lib.lap_attention_workspace_bytes(AT_WEIGHTS, s), q.device)
    rc = lib.lap_attention_weights(s, _rows(q, "q", q, q.shape), _rows(k, "k", q, kv + (s.head_dim,)),
                                   _plain(lse, "lse", torch.float32, q.shape[:3], q.device), _plain(before, "before", torch.float32, kv, q.device),
                                   _plain(weights, "weights", torch.float32, kv, q.device), at, have, _stream(torch, q.device))
    _done(rc, "lap_attention_weights", torch, q.device, sync)
    return dict(weights=weights)


def attention_step(q, k_cache, v_cache, weights=None, *, lens=None, positions=None, scale: Optional[float] = None,
                   out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_attention_step: q [batch, q_heads, head_dim] of one token against caches [batch, kv_heads, slots, head_dim].  Returns
    dict(out like q, lse [batch, q_heads], weights = the given ones + this token's, a new tensor unless out holds one; None
    where none are given)."""
    torch, lib = _torch(), _lib()
    _check(q.dim() == 3 and k_cache.dim() == 4, "q is [batch, heads, head_dim], caches are [batch, heads, slots, head_dim]")
    b, h, d = q.shape
    dev = q.device
    slots = (b, k_cache.shape[1], k_cache.shape[2])
    s = _Shape(_type(torch, q), b, h, slots[1], 1, slots[2], d, 0, 0, 1.0 / math.sqrt(d) if scale is None and d else (scale or 0.0),
               None, _plain(lens, "lens", torch.int32, (b,), dev))
    if out is None:
        out = dict(out=torch.empty_like(q), lse=torch.empty((b, h), dtype=torch.float32, device=dev),
                   weights=None if weights is None else torch.empty(slots, dtype=torch.float32, device=dev))
    ws, have, at = _workspace(torch, ws, lib.lap_attention_workspace_bytes(AT_STEP, s), dev)
    rc = lib.lap_attention_step(s, _rows(q, "q", q, q.shape), _rows(k_cache, "k_cache", q, slots + (d,)), _rows(v_cache, "v_cache", q, slots + (d,)),
                                _plain(positions, "positions", torch.int32, slots, dev), _plain(weights, "weights", torch.float32, slots, dev),
                                _rows(out["out"], "out", q, q.shape), _plain(out["lse"], "lse", torch.float32, (b, h), dev),
                                _plain(out.get("weights"), "out weights", torch.float32, slots, dev), at, have, _stream(torch, dev))
    _done(rc, "lap_attention_step", torch, dev, sync)
    return out


def _cache(torch, k, v, weights, positions, name: str = ""):
    _check(k.dim() == 4, "caches are [batch, heads, slots, head_dim]")
    b, h, n, d = k.shape
    kind = _type(torch, k)
    return _Cache(kind, b, h, n, d, _rows(k, name + "k", k, k.shape), _rows(v, name + "v", k, k.shape),
                  _plain(weights, name + "weights", torch.float32, (b, h, n), k.device),
                  _plain(positions, name + "positions", torch.int32, (b, h, n), k.device))


def cache_evict(k, v, weights, keep: int, recent: int, *, lens=None, positions=None, slots: Optional[int] = None,
                out: Optional[dict] = None, ws=None, sync: bool = True):
    """lap_cache_evict: the `keep` rows of highest weight of k and v, the newest `recent` among them, into a cache of `slots`
    (None: keep).  Returns dict(k, v, weights, positions [batch, kv_heads, slots], lens [batch])."""
    torch, lib = _torch(), _lib()
    src = _cache(torch, k, v, weights, positions)
    _check(keep >= 0 and recent >= 0, "keep and recent are numbers of slots")
    b, h, n, d = k.shape
    dev = k.device
    if out is None:
        m = int(keep if slots is None else slots)
        out = dict(k=torch.empty((b, h, m, d), dtype=k.dtype, device=dev), v=torch.empty((b, h, m, d), dtype=k.dtype, device=dev),
                   weights=torch.empty((b, h, m), dtype=torch.float32, device=dev),
                   positions=torch.empty((b, h, m), dtype=torch.int32, device=dev), lens=torch.empty(b, dtype=torch.int32, device=dev))
    _check(out["k"].dtype == k.dtype and out["k"].device == dev, "out k: type or device")
    dst = _cache(torch, out["k"], out["v"], out["weights"], out["positions"], "out ")
    ws, have, at = _workspace(torch, ws, lib.lap_cache_workspace_bytes(dst), dev)
    rc = lib.lap_cache_evict(src, _plain(lens, "lens", torch.int32, (b,), dev), int(keep), int(recent), dst,
                             _plain(out["lens"], "out lens", torch.int32, (b,), dev), at, have, _stream(torch, dev))
    _done(rc, "lap_cache_evict", torch, dev, sync)
    return out


def cache_insert(k_new, v_new, k_cache, v_cache, weights, positions, position, recent: int, *, slots=None, sync: bool = True):
    """lap_cache_insert: one token [batch, kv_heads, head_dim] into every cache, in place; position [batch] is the token's.
    Returns dict(slots [batch, kv_heads]): where it went."""
    torch, lib = _torch(), _lib()
    cache = _cache(torch, k_cache, v_cache, weights, positions)
    _check(recent >= 0, "recent is a number of slots")
    b, h, _, d = k_cache.shape
    dev = k_cache.device
    if slots is None:
        slots = torch.empty((b, h), dtype=torch.int32, device=dev)
    rc = lib.lap_cache_insert(cache, _rows(k_new, "k_new", k_cache, (b, h, d)), _rows(v_new, "v_new", k_cache, (b, h, d)),
                              _plain(position, "position", torch.int32, (b,), dev), int(recent),
                              _plain(slots, "slots", torch.int32, (b, h), dev), _stream(torch, dev))
    _done(rc, "lap_cache_insert", torch, dev, sync)
    return dict(slots=slots)
