"""Operators on the cache itself (ctypes binding of include/hill.h, as hill.py):

    hill_window_attn(q, k, v, window=, n_sink=)          -> out   one token over the first tokens and a window
    hill_window_prefill(q, k, v, window=, n_sink=)       -> out   the same for a chunk's tokens
    new_packed_cache / pack_kv / unpack_kv                        K and V held in 4 bits
    hill_packed_attn(q, cache, ...)                      -> out   one token over a packed cache [S += weights]
    hill_evict(s, k_keep, k=, v= | cache=, pos=)         -> idx   the k_keep heaviest tokens stay, in place

Shapes: q [B, Hq, D] (prefill: [B, Hq, T, D], any strides with D contiguous);
k, v [B, Hkv, Ncap, D]; lens [B] int32; s [B, R, >= n] fp32; out fp32
[B, Hq, D] (prefill: q's dtype and layout).  Calls run on the tensors' device, on its
current stream or on ``stream``; a workspace that is not given is allocated
there for the call.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import Optional

import torch

from .hill import (DTYPES, GRANS, HILL_OK, HillDesc, PackedDesc, PrefillDesc, _check, _ptr, _stream_ptr, load_library)

_NO_CONTEXT = contextlib.nullcontext()
_DESC_BYTES = ctypes.sizeof(HillDesc)


def _on(dev: torch.device, stream):
    """Context with the call's device and stream current, so that what is allocated in it belongs to that stream."""
    if stream is None:
        return _NO_CONTEXT if dev.index == torch._C._cuda_getDevice() else torch.cuda.device(dev)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=dev) if stream else torch.cuda.default_stream(dev)
    if stream.device != dev:
        raise ValueError("stream is on %s, the tensors are on %s" % (stream.device, dev))
    return torch.cuda.stream(stream)


def _device_of(*named) -> torch.device:
    """The one GPU that every given (name, tensor) is on."""
    dev = None
    for name, t in named:
        if t is None:
            continue
        if t.device.type != "cuda":
            raise ValueError("libhill works on GPU tensors only (%s is on %s)" % (name, t.device))
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError("%s is on %s, not on %s" % (name, t.device, dev))
    return dev


def _desc(B, Hq, Hkv, D, n, dtype, *, q_st=None, k_st=None, v_st=None, s_st=(0, 0), granularity="token", sm_scale=0.0,
          n_sink=0, n_recent=0) -> HillDesc:
    rows = (Hkv * n * D, n * D, D)
    k_st = rows if k_st is None else k_st
    v_st = k_st if v_st is None else v_st
    return HillDesc(_DESC_BYTES, B, Hq, Hkv, D, n, DTYPES.get(dtype, -1), 0, GRANS[granularity], sm_scale,
                    *((Hq * D, D) if q_st is None else q_st), *k_st, *v_st, *s_st, n_sink, n_recent)


def _rows(name, t, dims, dtype=None):
    """Strides of t before its contiguous last axis."""
    if t.dim() != dims:
        raise ValueError("%s must have %d dimensions, not %d" % (name, dims, t.dim()))
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s must be %s, not %s" % (name, dtype, t.dtype))
    st = t.stride()
    if st[-1] != 1:
        raise ValueError("%s must have a contiguous last axis" % name)
    return st[:-1]


def _int32(name, t, shape):
    if t.dtype != torch.int32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 tensor of shape %s" % (name, tuple(shape)))


def _tokens(n_tokens, most, what):
    n = most if n_tokens is None else int(n_tokens)
    if not 0 <= n <= most:
        raise ValueError("n_tokens %d is not among the %d of %s" % (n, most, what))
    return n


def _count(name, x):
    """A token count as the C structure holds it (more than any cache holds: all)."""
    x = int(x)
    if x < 0:
        raise ValueError("%s must be >= 0" % name)
    return min(x, 2 ** 31 - 1)


def _workspace(fn, args, like, ws):
    """ws, or one of the size that fn says on like's device (None for none)."""
    if ws is not None:
        if not ws.is_contiguous():
            raise ValueError("ws must be contiguous")
        return ws, ws.numel() * ws.element_size()
    need = ctypes.c_size_t(0)
    _check(fn(*args, ctypes.byref(need)))
    if need.value == 0:
        return None, 0
    return like.new_empty(need.value, dtype=torch.uint8), need.value


def _kv_strides(k, v, B, D, dtype):
    k_st, v_st = _rows("k", k, 4, dtype), _rows("v", v, 4, dtype)
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        raise ValueError("k and v must be [%d, Hkv, n, %d] alike, got %s and %s" % (B, D, tuple(k.shape), tuple(v.shape)))
    return k_st, v_st


def _out(out, q):
    if out is None:
        return q.new_empty(q.shape, dtype=torch.float32)
    if out.dtype != torch.float32 or out.shape != q.shape or not out.is_contiguous():
        raise ValueError("out must be a contiguous float32 tensor of q's shape")
    return out


def _window_desc(q, k, v, lens, n_tokens, window, n_sink, sm_scale, dims):
    q_st = _rows("q", q, dims)
    B, Hq, D = q.shape[0], q.shape[1], q.shape[-1]
    k_st, v_st = _kv_strides(k, v, B, D, q.dtype)
    n = _tokens(n_tokens, k.shape[2], "the cache")
    if lens is not None:
        _int32("lens", lens, (B,))
    return _desc(B, Hq, k.shape[1], D, n, q.dtype, q_st=q_st[:2], k_st=k_st, v_st=v_st, sm_scale=float(sm_scale),
                 n_sink=_count("n_sink", n_sink), n_recent=_count("window", window)), q_st


def hill_window_attn(q, k, v, *, window, n_sink=0, n_tokens=None, lens=None, sm_scale=0.0, out=None, ws=None, stream=None):
    """Attention of one token per sequence, the last of its n_tokens (or
    lens[b]) tokens, over the first n_sink and the last ``window`` of them;
    out [B, Hq, D] fp32, zero where nothing is visible."""
    lib = load_library()
    dev = _device_of(("q", q), ("k", k), ("v", v), ("lens", lens), ("out", out), ("ws", ws))
    d, _ = _window_desc(q, k, v, lens, n_tokens, window, n_sink, sm_scale, 3)
    with _on(dev, stream):
        out = _out(out, q)
        ref = ctypes.byref(d)
        ws, ws_bytes = _workspace(lib.hill_window_workspace_bytes, (ref, 0), q, ws)
        _check(lib.hill_window_attn(ref, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lens), out.data_ptr(), _ptr(ws),
                                    ws_bytes, _stream_ptr(None)))
    return out


def hill_window_prefill(q, k, v, *, window, n_sink=0, n_tokens=None, lens=None, sm_scale=0.0, out=None, ws=None,
                        stream=None):
    """Attention of the last T tokens of every sequence (q [B, Hq, T, D]; their
    K and V are in the cache), each over the first n_sink tokens and the last
    ``window`` up to itself; out like q (its dtype; its strides where they are
    dense), zero for rows before the sequence's first token."""
    lib = load_library()
    dev = _device_of(("q", q), ("k", k), ("v", v), ("lens", lens), ("out", out), ("ws", ws))
    d, q_st = _window_desc(q, k, v, lens, n_tokens, window, n_sink, sm_scale, 4)
    with _on(dev, stream):
        if out is None:
            out = torch.empty_like(q)
        if out.shape != q.shape:
            raise ValueError("out must have q's shape")
        o_st = _rows("out", out, 4, q.dtype)
        p = PrefillDesc(ctypes.sizeof(PrefillDesc), q.shape[2], q_st[2], *o_st)
        ref = ctypes.byref(d)
        ws, ws_bytes = _workspace(lib.hill_window_workspace_bytes, (ref, q.shape[2]), q, ws)
        _check(lib.hill_window_prefill(ref, ctypes.byref(p), q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lens),
                                       out.data_ptr(), _ptr(ws), ws_bytes, _stream_ptr(None)))
    return out


class PackedCache:
    """K and V of one layer held in 4 bits (include/hill.h): codes [B, Hkv,
    cap, 64] uint8 and (scale, zero) of each group of 32 elements, [B, Hkv,
    cap, 4, 2] fp16, both contiguous; 160 bytes per token and KV head.  A cache
    that is written (pack_kv, hill_evict) has four buffers that do not overlap."""

    def __init__(self, k_codes, k_params, v_codes, v_params):
        B, Hkv, cap = k_codes.shape[:3]
        _device_of(("k_codes", k_codes), ("k_params", k_params), ("v_codes", v_codes), ("v_params", v_params))
        for name, t, shape, dtype in (("k_codes", k_codes, (64,), torch.uint8), ("v_codes", v_codes, (64,), torch.uint8),
                                      ("k_params", k_params, (4, 2), torch.float16),
                                      ("v_params", v_params, (4, 2), torch.float16)):
            if tuple(t.shape) != (B, Hkv, cap) + shape or t.dtype != dtype or not t.is_contiguous():
                raise ValueError("%s must be a contiguous %s tensor of shape %s" % (name, dtype, (B, Hkv, cap) + shape))
        self.k_codes, self.k_params, self.v_codes, self.v_params = k_codes, k_params, v_codes, v_params
        self.batch, self.n_kv_heads, self.cap = B, Hkv, cap
        self.device = k_codes.device
        self.desc = PackedDesc(ctypes.sizeof(PackedDesc), cap, k_codes.data_ptr(), k_params.data_ptr(), v_codes.data_ptr(),
                               v_params.data_ptr())


def new_packed_cache(B: int, Hkv: int, cap: int, device) -> PackedCache:
    """A packed cache of ``cap`` zero rows per sequence and KV head."""
    codes = [torch.zeros((B, Hkv, cap, 64), dtype=torch.uint8, device=device) for _ in range(2)]
    params = [torch.zeros((B, Hkv, cap, 4, 2), dtype=torch.float16, device=device) for _ in range(2)]
    return PackedCache(codes[0], params[0], codes[1], params[1])


def pack_kv(k, v, cache: PackedCache, *, at=0, stream=None) -> PackedCache:
    """Writes the rows of k and v ([B, Hkv, T, D], any strides with D
    contiguous) into the cache from row ``at`` on: an int, or an int32 tensor
    [B] with each sequence's (rows that would land outside the cache are then dropped)."""
    lib = load_library()
    lens = at if isinstance(at, torch.Tensor) else None
    dev = _device_of(("k", k), ("v", v), ("cache", cache.k_codes), ("at", lens))
    k_st, v_st = _kv_strides(k, v, cache.batch, 128, k.dtype)
    B, Hkv, T, D = k.shape
    if Hkv != cache.n_kv_heads:
        raise ValueError("k has %d KV heads, the cache %d" % (Hkv, cache.n_kv_heads))
    if lens is not None:
        _int32("at", lens, (B,))
    elif not 0 <= int(at) <= cache.cap - T:
        raise ValueError("rows [%d, %d) are not inside the cache's %d" % (at, at + T, cache.cap))
    if T == 0:
        return cache
    d = _desc(B, Hkv, Hkv, D, T, k.dtype, k_st=k_st, v_st=v_st)
    with _on(dev, stream):
        _check(lib.hill_pack_kv(ctypes.byref(d), ctypes.byref(cache.desc), k.data_ptr(), v.data_ptr(), _ptr(lens),
                                0 if lens is not None else int(at), _stream_ptr(None)))
    return cache


def unpack_kv(cache: PackedCache, *, token_begin=0, token_end=None, dtype=torch.float16, k_out=None, v_out=None, stream=None):
    """Rows [token_begin, token_end) of the cache as 16-bit k and v ([B, Hkv,
    token_end - token_begin, D]); fp16 holds the values exactly."""
    lib = load_library()
    t1 = cache.cap if token_end is None else int(token_end)
    rows = t1 - int(token_begin)
    if not 0 <= int(token_begin) <= t1 <= cache.cap:
        raise ValueError("rows [%d, %d) are not inside the cache's %d" % (token_begin, t1, cache.cap))
    if (k_out is None) != (v_out is None):
        raise ValueError("k_out and v_out go together")
    dev = _device_of(("cache", cache.k_codes), ("k_out", k_out), ("v_out", v_out))
    shape = (cache.batch, cache.n_kv_heads, rows, 128)
    with _on(dev, stream):
        if k_out is None:
            k_out, v_out = (torch.empty(shape, dtype=dtype, device=dev) for _ in range(2))
        k_st, v_st = _rows("k_out", k_out, 4), _rows("v_out", v_out, 4, k_out.dtype)
        if tuple(k_out.shape) != shape or tuple(v_out.shape) != shape:
            raise ValueError("k_out and v_out must be %s" % (shape,))
        if rows == 0:
            return k_out, v_out
        d = _desc(shape[0], shape[1], shape[1], 128, rows, k_out.dtype, k_st=k_st, v_st=v_st)
        _check(lib.hill_unpack_kv(ctypes.byref(d), ctypes.byref(cache.desc), int(token_begin), t1, k_out.data_ptr(),
                                  v_out.data_ptr(), _stream_ptr(None)))
    return k_out, v_out


def _packed_desc(q, cache, n_tokens, lens, n_sink, window, idx, s, granularity, sm_scale):
    """Descriptor and list length."""
    q_st = _rows("q", q, 3)
    B, Hq, D = q.shape
    if B != cache.batch:
        raise ValueError("q has %d sequences, the cache %d" % (B, cache.batch))
    n = _tokens(n_tokens, cache.cap, "the cache")
    if lens is not None:
        _int32("lens", lens, (B,))
    R = 1 if granularity == "token" else cache.n_kv_heads
    s_st = (0, 0)
    if s is not None:
        s_st = _rows("s", s, 3, torch.float32)
        if s.shape[0] != B or s.shape[1] != R or s.shape[2] < n:
            raise ValueError("s must be [%d, %d, >= %d], not %s" % (B, R, n, tuple(s.shape)))
    k_sel = 0
    if idx is not None:
        k_sel = idx.shape[-1]
        _int32("idx", idx, (B, R, k_sel))
        if k_sel == 0:
            raise ValueError("idx lists no tokens")
    return _desc(B, Hq, cache.n_kv_heads, D, n, q.dtype, q_st=q_st, s_st=s_st, granularity=granularity,
                 sm_scale=float(sm_scale), n_sink=_count("n_sink", n_sink),
                 n_recent=_count("window", n if window is None else window)), k_sel


def hill_packed_attn(q, cache: PackedCache, *, n_tokens=None, lens=None, n_sink=0, window=None, idx=None, s=None,
                     granularity="token", sm_scale=0.0, out=None, ws=None, stream=None):
    """Attention of one token per sequence over a packed cache: over all its
    n_tokens (or lens[b]) tokens, or the first n_sink and the last ``window`` of
    them, or the tokens of ``idx`` ([B, R, k] int32, as hill_topk gives them).
    ``s``: S += the weights of the visible tokens (as hill_score).  Returns out
    [B, Hq, D] fp32."""
    lib = load_library()
    dev = _device_of(("q", q), ("cache", cache.k_codes), ("lens", lens), ("idx", idx), ("s", s), ("out", out), ("ws", ws))
    d, k_sel = _packed_desc(q, cache, n_tokens, lens, n_sink, window, idx, s, granularity, sm_scale)
    with _on(dev, stream):
        out = _out(out, q)
        ref = ctypes.byref(d)
        ws, ws_bytes = _workspace(lib.hill_packed_workspace_bytes, (ref, k_sel, int(s is not None)), q, ws)
        _check(lib.hill_packed_attn(ref, ctypes.byref(cache.desc), q.data_ptr(), _ptr(lens), _ptr(idx), k_sel, _ptr(s),
                                    out.data_ptr(), _ptr(ws), ws_bytes, _stream_ptr(None)))
    return out


def hill_evict(s, k_keep, *, k=None, v=None, cache: Optional[PackedCache] = None, pos=None, n_tokens=None,
               granularity="token", n_kv_heads=None, n_sink=0, n_recent=0, idx_out=None, ws=None, stream=None):
    """Makes the cache k_keep tokens long: the k_keep largest S of each row
    stay (the first n_sink and last n_recent always), in order and in place, in
    k and v or in ``cache``, in s (zero behind them) and in pos (int32, s's
    shape and strides).  Returns their former indices [B, R, k_keep] int32.  Calls that
    run at the same time need a ``ws`` each (the call's own, if none is given)."""
    lib = load_library()
    k_keep = int(k_keep)
    if (k is None) != (v is None) or (k is not None and cache is not None):
        raise ValueError("give k and v, or cache, or neither")
    dev = _device_of(("s", s), ("k", k), ("v", v), ("cache", None if cache is None else cache.k_codes), ("pos", pos),
                     ("idx_out", idx_out), ("ws", ws))
    s_st = _rows("s", s, 3, torch.float32)
    B, R, cap = s.shape
    n = _tokens(n_tokens, cap, "s")
    if not 1 <= k_keep <= n:
        raise ValueError("k_keep %d not in [1, n_tokens=%d]" % (k_keep, n))
    k_st = v_st = None
    Hkv, dtype = n_kv_heads, torch.float16
    if k is not None:
        Hkv, dtype = k.shape[1], k.dtype
        k_st, v_st = _kv_strides(k, v, B, 128, dtype)
        _tokens(n, k.shape[2], "k")
    elif cache is not None:
        Hkv = cache.n_kv_heads
        if cache.batch != B:
            raise ValueError("s has %d sequences, the cache %d" % (B, cache.batch))
        _tokens(n, cache.cap, "the cache")
    elif Hkv is None:
        Hkv = R
    if R != (1 if granularity == "token" else Hkv):
        raise ValueError("s has %d rows per sequence, granularity %s needs %d" % (R, granularity, 1 if granularity == "token"
                                                                                  else Hkv))
    p_st = (0, 0)
    if pos is not None:
        p_st = _rows("pos", pos, 3, torch.int32)
        if pos.shape[:2] != s.shape[:2] or pos.shape[2] < n:
            raise ValueError("pos must be [%d, %d, >= %d], not %s" % (B, R, n, tuple(pos.shape)))
    d = _desc(B, Hkv, Hkv, 128, n, dtype, k_st=k_st, v_st=v_st, s_st=s_st, granularity=granularity,
              n_sink=_count("n_sink", n_sink), n_recent=_count("n_recent", n_recent))
    with _on(dev, stream):
        if idx_out is None:
            idx_out = torch.empty((B, R, k_keep), dtype=torch.int32, device=dev)
        else:
            _int32("idx_out", idx_out, (B, R, k_keep))
        ref = ctypes.byref(d)
        ws, ws_bytes = _workspace(lib.hill_evict_workspace_bytes, (ref, k_keep), s, ws)
        _check(lib.hill_evict(ref, s.data_ptr(), k_keep, idx_out.data_ptr(), _ptr(k), _ptr(v),
                              None if cache is None else ctypes.byref(cache.desc), _ptr(pos), *p_st, _ptr(ws), ws_bytes,
                              _stream_ptr(None)))
    return idx_out


class _AttnCall:
    """A call marshalled once, for per-step loops: only the query pointer
    changes (and what lens, on the device, says).  Runs on the device and the stream that
    it was made for; its workspace and ``out`` are its own."""

    def _marshal(self, fn, dev, keep, before, after):
        self._fn, self._dev, self._keep, self._before = fn, dev.index, keep, before
        self._after = tuple(ctypes.c_void_p(_ptr(x)) if x is None or isinstance(x, torch.Tensor) else x for x in after)

    def __call__(self, q_ptr: int):
        if torch._C._cuda_getDevice() != self._dev:
            with torch.cuda.device(self._dev):
                return self(q_ptr)
        st = self._fn(*self._before, q_ptr, *self._after)
        if st != HILL_OK:
            _check(st)


class WindowAttnCall(_AttnCall):
    """hill_window_attn for queries of q's shape and strides."""

    def __init__(self, q, k, v, *, window, n_sink=0, n_tokens=None, lens=None, sm_scale=0.0, ws=None, stream=None):
        lib = load_library()
        dev = _device_of(("q", q), ("k", k), ("v", v), ("lens", lens), ("ws", ws))
        self.desc, _ = _window_desc(q, k, v, lens, n_tokens, window, n_sink, sm_scale, 3)
        with _on(dev, stream):
            self.out = _out(None, q)
            ref = ctypes.byref(self.desc)
            self.ws, ws_bytes = _workspace(lib.hill_window_workspace_bytes, (ref, 0), q, ws)
            self._marshal(lib.hill_window_attn, dev, (k, v, lens), (ref,),
                          (k, v, lens, self.out, self.ws, ctypes.c_size_t(ws_bytes), ctypes.c_void_p(_stream_ptr(None))))


class PackedAttnCall(_AttnCall):
    """hill_packed_attn for queries of q's shape and strides."""

    def __init__(self, q, cache: PackedCache, *, n_tokens=None, lens=None, n_sink=0, window=None, idx=None, s=None,
                 granularity="token", sm_scale=0.0, ws=None, stream=None):
        lib = load_library()
        dev = _device_of(("q", q), ("cache", cache.k_codes), ("lens", lens), ("idx", idx), ("s", s), ("ws", ws))
        self.desc, k_sel = _packed_desc(q, cache, n_tokens, lens, n_sink, window, idx, s, granularity, sm_scale)
        with _on(dev, stream):
            self.out = _out(None, q)
            ref = ctypes.byref(self.desc)
            self.ws, ws_bytes = _workspace(lib.hill_packed_workspace_bytes, (ref, k_sel, int(s is not None)), q, ws)
            self._marshal(lib.hill_packed_attn, dev, (cache, lens, idx, s), (ref, ctypes.byref(cache.desc)),
                          (lens, idx, ctypes.c_int32(k_sel), s, self.out, self.ws, ctypes.c_size_t(ws_bytes),
                           ctypes.c_void_p(_stream_ptr(None))))
