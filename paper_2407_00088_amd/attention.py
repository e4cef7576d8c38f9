"""Attention between the projections: thin binding of include/tmac_attn.h (argument checks and marshalling; every step runs in the
library's HIP kernels), functions that allocate results and workspace, and a holder of one layer's cache.  For inference: there is no
backward pass, and results of inputs that require gradients carry none.

  attn_prompt     attention over packed prompts
  attn_weights    the attention weight that each of their keys received
  KVCache         a cache that keeps the heaviest keys: fill (from prompts or another cache), append (one token), attend (a
                  decode step over a shared prefix, if there is one, and the cache)
"""
from __future__ import annotations

import contextlib
import ctypes as C
import math
import threading
from typing import Optional

import torch

from . import binding as B

TMAC_ELEM_F16, TMAC_ELEM_BF16 = 0, 1
_ELEM = {torch.float16: TMAC_ELEM_F16, torch.bfloat16: TMAC_ELEM_BF16}

EXPORTS = ["tmac_attn_prompt_workspace_bytes", "tmac_attn_prompt", "tmac_attn_weights_workspace_bytes", "tmac_attn_weights",
           "tmac_cache_fill_workspace_bytes", "tmac_cache_fill", "tmac_cache_append", "tmac_attn_decode_workspace_bytes",
           "tmac_attn_decode"]


class tmac_attn_desc(C.Structure):
    _fields_ = [("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("elem", C.c_int32), ("scale", C.c_float),
                ("causal", C.c_int32), ("reserved", C.c_int32 * 2)]


class tmac_view(C.Structure):
    _fields_ = [("data", C.c_void_p), ("seq", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class tmac_cache(C.Structure):
    _fields_ = [("k", tmac_view), ("v", tmac_view), ("weight_dev", C.c_void_p), ("pos_dev", C.c_void_p), ("lens_dev", C.c_void_p),
                ("seen_dev", C.c_void_p), ("B", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("capacity", C.c_int32),
                ("recent", C.c_int32), ("elem", C.c_int32), ("reserved", C.c_int32 * 2)]


class tmac_cache_source(C.Structure):
    _fields_ = [("k", tmac_view), ("v", tmac_view), ("weight", tmac_view), ("pos", tmac_view), ("cu_dev", C.c_void_p),
                ("lens_dev", C.c_void_p), ("seen_dev", C.c_void_p), ("total", C.c_int32), ("reserved", C.c_int32)]


def _declare(lib):
    D, V, K, S = (C.POINTER(t) for t in (tmac_attn_desc, tmac_view, tmac_cache, tmac_cache_source))
    P, I32, SZ = C.c_void_p, C.c_int32, C.c_size_t
    for name, result, args in [
            ("tmac_attn_prompt_workspace_bytes", SZ, [D, I32, I32, I32]),
            ("tmac_attn_prompt", C.c_int, [D, V, V, V, I32, I32, I32, P, P, V, P, P, SZ, P]),
            ("tmac_attn_weights_workspace_bytes", SZ, [D, I32, I32, I32]),
            ("tmac_attn_weights", C.c_int, [D, V, V, P, I32, I32, I32, P, P, P, P, SZ, P]),
            ("tmac_cache_fill_workspace_bytes", SZ, [K]),
            ("tmac_cache_fill", C.c_int, [K, S, P, SZ, P]),
            ("tmac_cache_append", C.c_int, [K, V, V, P]),
            ("tmac_attn_decode_workspace_bytes", SZ, [D, K, I32, I32]),
            ("tmac_attn_decode", C.c_int, [D, V, V, V, I32, K, I32, V, P, P, SZ, P])]:
        f = getattr(lib, name)
        f.restype, f.argtypes = result, args
    return lib


lib = _declare(B.lib)
# the ordinary calls go through the native side of the binding, which answers None for all others; those are checked, worded
# and made here
calls = B.calls
calls.bind_attention(tmac_attn_desc, tmac_cache, *(C.cast(getattr(lib, f), C.c_void_p).value for f in EXPORTS))


def attn_desc(Hq: int, Hkv: int, D: int, dtype, scale: Optional[float] = None, causal: bool = True) -> tmac_attn_desc:
    if dtype not in _ELEM:
        raise ValueError(f"q, k and v are float16 or bfloat16, got {dtype}")
    return tmac_attn_desc(Hq, Hkv, D, _ELEM[dtype], 1.0 / math.sqrt(D) if scale is None else scale, int(causal))


def _dims(name: str, t, order: str, shape, dtype) -> None:
    """The tensor's type, dimensions and place; -1 stands for any size.  (The C ABI takes them on trust.)"""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.dim() != len(shape) or not t.is_cuda or \
            any(want not in (-1, got) for want, got in zip(shape, t.shape)):
        got = f"{tuple(t.shape)} {t.dtype} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name} is a tensor [{order}] = {list(shape)} of {dtype} on the GPU, got {got}")


def _rows(name: str, t) -> None:
    if t.numel() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the elements of a row of {name} lie side by side: got strides {tuple(t.stride())}")


def _apart(name: str, t) -> None:
    """No two rows of a result share an element."""
    end = t.shape[-1]
    for stride, n in sorted(zip(t.stride()[:-1], t.shape[:-1])):
        if n > 1:
            if stride < end:
                raise ValueError(f"the rows of {name} do not overlap: got strides {tuple(t.stride())} for {tuple(t.shape)}")
            end += stride * (n - 1)


def _counted(**sizes) -> None:
    """The C ABI counts in 32 bits."""
    for name, n in sizes.items():
        if n >= 1 << 31:
            raise ValueError(f"{name} ({n}) does not fit 32 bits")


def _plain(name: str, t, shape, dtype) -> None:
    _dims(name, t, ", ".join(str(n) for n in shape), shape, dtype)
    if not t.is_contiguous():
        raise ValueError(f"{name} is contiguous")


def _view(t, seq: Optional[int], token: Optional[int], head: Optional[int]) -> tmac_view:
    """Strides of the given dimensions; that of a dimension of one entry is never used and may be anything in torch."""
    s = [0 if d is None or t.shape[d] == 1 else t.stride(d) for d in (seq, token, head)]
    return tmac_view(t.data_ptr(), *s)


def _same_device(*tensors) -> None:
    """All on the current device, whose stream the call goes to."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.device.index != here:
            raise ValueError(f"tensors on {t.device}, the current device is cuda:{here}")


def _workspace(n: int, device):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device)


def _on(stream):
    """Results and workspaces of a call on a stream of the caller's belong to that stream: memory of another one could be handed
    out again there while the call still runs."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _packed(q, k, cu_q, cu_k):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q is [Tq, Hq, D], k is [Tk, Hkv, D]")
    (Tq, Hq, D), (Tk, Hkv, _) = q.shape, k.shape
    if q.dtype not in _ELEM:
        raise ValueError(f"q, k and v are float16 or bfloat16, got {q.dtype}")
    _dims("q", q, "Tq, Hq, D", (Tq, Hq, D), q.dtype)
    _dims("k", k, "Tk, Hkv, D", (Tk, Hkv, D), q.dtype)
    _rows("q", q), _rows("k", k)
    S = cu_q.numel() - 1
    _plain("cu_q", cu_q, (S + 1,), torch.int32)
    _plain("cu_k", cu_k, (S + 1,), torch.int32)
    _counted(S=S, Tq=Tq, Tk=Tk, Hq=Hq, D=D)
    if Hkv == 0 or Hq % Hkv:
        raise ValueError(f"the query heads ({Hq}) are a multiple of the key heads ({Hkv})")
    return S, Tq, Tk, Hq, Hkv, D


def attn_prompt(q, k, v, cu_q, cu_k=None, causal: bool = True, scale: Optional[float] = None, out=None, lse=None, stream=None):
    """Attention over packed sequences: q [Tq, Hq, D], k and v [Tk, Hkv, D], cu_q and cu_k int32 [S + 1] (cu_k None: the queries' own).
    Returns (out [Tq, Hq, D], lse fp32 [Hq, Tq])."""
    cu_k = cu_q if cu_k is None else cu_k
    if out is None and lse is None and stream is None:
        got = calls.attn_prompt(q, k, v, cu_q, cu_k, causal, scale)
        if got is not None:
            return got
    S, Tq, Tk, Hq, Hkv, D = _packed(q, k, cu_q, cu_k)
    _dims("v", v, "Tk, Hkv, D", (Tk, Hkv, D), q.dtype)
    _rows("v", v)
    desc = attn_desc(Hq, Hkv, D, q.dtype, scale, causal)
    n = lib.tmac_attn_prompt_workspace_bytes(desc, S, Tq, Tk)
    with _on(stream):
        if out is None:
            out = torch.empty((Tq, Hq, D), dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty((Hq, Tq), dtype=torch.float32, device=q.device)
        ws = _workspace(n, q.device) if n else None
    _dims("out", out, "Tq, Hq, D", (Tq, Hq, D), q.dtype)
    _rows("out", out), _apart("out", out)
    _plain("lse", lse, (Hq, Tq), torch.float32)
    _same_device(q, k, v, cu_q, cu_k, out, lse)
    B._check(lib.tmac_attn_prompt(desc, _view(q, None, 0, 1), _view(k, None, 0, 1), _view(v, None, 0, 1), S, Tq, Tk, cu_q.data_ptr(),
                                  cu_k.data_ptr(), _view(out, None, 0, 1), lse.data_ptr(), ws.data_ptr() if n else None, n,
                                  B._stream_ptr(stream)), "tmac_attn_prompt")
    return out, lse


def attn_weights(q, k, lse, cu_q, cu_k=None, causal: bool = True, scale: Optional[float] = None, out=None, stream=None):
    """Weight [Hkv, Tk] (fp32) that each key received: exp(s - lse) summed over the queries that see it and the heads of its group;
    lse as attn_prompt returns it."""
    cu_k = cu_q if cu_k is None else cu_k
    if out is None and stream is None:
        got = calls.attn_weights(q, k, lse, cu_q, cu_k, causal, scale)
        if got is not None:
            return got
    S, Tq, Tk, Hq, Hkv, D = _packed(q, k, cu_q, cu_k)
    _plain("lse", lse, (Hq, Tq), torch.float32)
    desc = attn_desc(Hq, Hkv, D, q.dtype, scale, causal)
    n = lib.tmac_attn_weights_workspace_bytes(desc, S, Tq, Tk)
    with _on(stream):
        if out is None:
            out = torch.empty((Hkv, Tk), dtype=torch.float32, device=q.device)
        ws = _workspace(n, q.device) if n else None
    _plain("out", out, (Hkv, Tk), torch.float32)
    _same_device(q, k, lse, cu_q, cu_k, out)
    B._check(lib.tmac_attn_weights(desc, _view(q, None, 0, 1), _view(k, None, 0, 1), lse.data_ptr(), S, Tq, Tk, cu_q.data_ptr(),
                                   cu_k.data_ptr(), out.data_ptr(), ws.data_ptr() if n else None, n, B._stream_ptr(stream)),
             "tmac_attn_weights")
    return out


class KVCache:
    """Keys and values of one layer for `batch` sequences, `capacity` slots for each sequence and key head, which keep the
    `recent` last tokens and the heaviest others.

      k, v    [batch, Hkv, capacity, D]          weight  fp32 [batch, Hkv, capacity]
      pos     int32 [batch, Hkv, capacity]       lens, seen  int32 [batch, Hkv]

    The tensors may be written to, not replaced (calls go by their addresses).  Calls of one cache share its workspaces: on several streams they must not overlap.
    Calls from several threads are enqueued one after the other, each whole.
    """

    def __init__(self, batch: int, Hkv: int, D: int, capacity: int, recent: int = 0, dtype=torch.float16, Hq: Optional[int] = None,
                 scale: Optional[float] = None, device: str = "cuda"):
        if not 0 <= recent <= capacity:
            raise ValueError(f"recent ({recent}) is between 0 and the capacity ({capacity})")
        self.B, self.Hkv, self.D, self.capacity, self.recent = batch, Hkv, D, capacity, recent
        self.Hq = Hkv if Hq is None else Hq
        self.desc = attn_desc(self.Hq, Hkv, D, dtype, scale, False)
        self.k = torch.zeros((batch, Hkv, capacity, D), dtype=dtype, device=device)
        self.v = torch.zeros_like(self.k)
        self.weight = torch.zeros((batch, Hkv, capacity), dtype=torch.float32, device=device)
        self.pos = torch.zeros((batch, Hkv, capacity), dtype=torch.int32, device=device)
        self.lens = torch.zeros((batch, Hkv), dtype=torch.int32, device=device)
        self.seen = torch.zeros((batch, Hkv), dtype=torch.int32, device=device)
        self.cache = tmac_cache(_view(self.k, 0, 2, 1), _view(self.v, 0, 2, 1), self.weight.data_ptr(), self.pos.data_ptr(),
                                self.lens.data_ptr(), self.seen.data_ptr(), batch, Hkv, D, capacity, recent, _ELEM[dtype])
        # (a call is up to two launches that hand a workspace on, and the interpreter may change threads between them)
        self.lock = threading.RLock()
        self.fill_ws = None
        self.attend_ws = None
        self.outgrown = []

    def __setattr__(self, name, value):
        # (`cache.weight *= x` comes here too, with the tensor that is there)
        if name in ("k", "v", "weight", "pos", "lens", "seen") and self.__dict__.get(name, value) is not value:
            raise AttributeError(f"{name} is written to, not replaced: {name}.copy_(...)")
        super().__setattr__(name, value)

    def _grown(self, ws, n: int, stream):
        """A workspace of n bytes at least.  (One that is too small is kept: an earlier call may still run on it, or a graph that was
        captured with it be replayed.  Sizes at least double, so that what is kept stays below what is used.)"""
        if ws is not None and ws.numel() >= n:
            return ws
        if ws is not None:
            self.outgrown.append(ws)
            n = max(n, 2 * ws.numel())
        with _on(stream):
            return _workspace(n, self.k.device)

    def _fill(self, source: tmac_cache_source, stream) -> None:
        n = lib.tmac_cache_fill_workspace_bytes(self.cache)
        self.fill_ws = self._grown(self.fill_ws, n, stream)
        B._check(lib.tmac_cache_fill(self.cache, source, self.fill_ws.data_ptr(), n, B._stream_ptr(stream)), "tmac_cache_fill")

    def fill(self, k, v, weight, cu, stream=None) -> None:
        """From packed prompts: k, v [T, Hkv, D], weight fp32 [Hkv, T] (attn_weights), cu int32 [batch + 1]."""
        with self.lock:
            if stream is None and self.fill_ws is not None and calls.cache_fill(self.cache, self.k, k, v, weight, cu, self.fill_ws):
                return
            T = k.shape[0]
            _counted(T=T)
            _dims("k", k, "T, Hkv, D", (T, self.Hkv, self.D), self.k.dtype)
            _dims("v", v, "T, Hkv, D", (T, self.Hkv, self.D), self.k.dtype)
            _rows("k", k), _rows("v", v)
            _dims("weight", weight, "Hkv, T", (self.Hkv, T), torch.float32)
            _plain("cu", cu, (self.B + 1,), torch.int32)
            _same_device(self.k, k, v, weight, cu)
            self._fill(tmac_cache_source(_view(k, None, 0, 1), _view(v, None, 0, 1), _view(weight, None, 1, 0), tmac_view(), cu.data_ptr(), None,
                                         None, T), stream)

    def fill_from(self, other: "KVCache", stream=None) -> None:
        """From another cache of as many sequences and heads: its heaviest and latest tokens, as many as this one holds."""
        if other is self or (other.B, other.Hkv, other.D, other.k.dtype) != (self.B, self.Hkv, self.D, self.k.dtype):
            raise ValueError("the source is another cache of the same sequences, heads and type")
        _same_device(self.k, other.k)
        first, second = sorted((self, other), key=id)   # (the same order whichever is filled from the other)
        with first.lock, second.lock:
            self._fill(tmac_cache_source(_view(other.k, 0, 2, 1), _view(other.v, 0, 2, 1), _view(other.weight, 0, 2, 1), _view(other.pos, 0, 2, 1),
                                         None, other.lens.data_ptr(), other.seen.data_ptr(), other.capacity), stream)

    def append(self, k, v, stream=None) -> None:
        """One token for every sequence: k, v [batch, Hkv, D]."""
        with self.lock:
            if stream is None and calls.cache_append(self.cache, self.k, k, v):
                return
            for name, t in (("k", k), ("v", v)):
                _dims(name, t, "batch, Hkv, D", (self.B, self.Hkv, self.D), self.k.dtype)
                _rows(name, t)
            _same_device(self.k, k, v)
            B._check(lib.tmac_cache_append(self.cache, _view(k, 0, None, 1), _view(v, 0, None, 1), B._stream_ptr(stream)), "tmac_cache_append")

    def attend(self, q, prefix_k=None, prefix_v=None, weigh: bool = True, out=None, lse=None, stream=None):
        """One decode step: q [batch, Hq, D] over the prefix (k and v [P, Hkv, D], shared by all sequences), if there is one, and the
        slots in use; `weigh` adds the step's weights to the slots'.  Returns (out [batch, Hq, D], lse fp32 [batch, Hq])."""
        with self.lock:
            if out is None and lse is None and stream is None and self.attend_ws is not None:
                got = calls.attend(self.cache, self.k, self.desc, q, prefix_k, prefix_v, weigh, self.attend_ws)
                if got is not None:
                    return got
            dt = self.k.dtype
            _dims("q", q, "batch, Hq, D", (self.B, self.Hq, self.D), dt)
            _rows("q", q)
            P, v0, v1 = 0, tmac_view(), tmac_view()
            if (prefix_k is None) != (prefix_v is None):
                raise ValueError("a prefix has keys and values")
            if prefix_k is not None:
                P = prefix_k.shape[0]
                _counted(P=P)
                for name, t in (("prefix_k", prefix_k), ("prefix_v", prefix_v)):
                    _dims(name, t, "P, Hkv, D", (P, self.Hkv, self.D), dt)
                    _rows(name, t)
                v0, v1 = _view(prefix_k, None, 0, 1), _view(prefix_v, None, 0, 1)
            with _on(stream):
                if out is None:
                    out = torch.empty((self.B, self.Hq, self.D), dtype=dt, device=q.device)
                if lse is None:
                    lse = torch.empty((self.B, self.Hq), dtype=torch.float32, device=q.device)
            _dims("out", out, "batch, Hq, D", (self.B, self.Hq, self.D), dt)
            _rows("out", out), _apart("out", out)
            _plain("lse", lse, (self.B, self.Hq), torch.float32)
            _same_device(self.k, q, prefix_k, prefix_v, out, lse)
            n = lib.tmac_attn_decode_workspace_bytes(self.desc, self.cache, P, int(weigh))
            self.attend_ws = self._grown(self.attend_ws, n, stream)
            B._check(lib.tmac_attn_decode(self.desc, _view(q, 0, None, 1), v0, v1, P, self.cache, int(weigh), _view(out, 0, None, 1),
                                          lse.data_ptr(), self.attend_ws.data_ptr(), n, B._stream_ptr(stream)), "tmac_attn_decode")
            return out, lse
