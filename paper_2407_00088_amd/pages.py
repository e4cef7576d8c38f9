"""A paged cache of keys and values in 8 bits: thin binding of include/tmac_pages.h (argument checks and marshalling; every step runs
in the library's HIP kernels), and holders of frequencies, of the pages, and of which page belongs to which sequence.  For inference, as
attention.py.

  Rotary      rotary positions: rotate
  PagedCache  one layer's keys and values: append (tokens into their pages, keys rotated on the way), attend, read
  PageTable   pages and lengths of a batch's sequences, on the host and on the GPU
"""
from __future__ import annotations

import ctypes as C
import math
import threading
from typing import Optional, Sequence

import torch

from . import attention as A
from . import binding as B
from .attention import tmac_attn_desc, tmac_view

TMAC_CODE_I8, TMAC_CODE_E4M3 = 0, 1
BLOCK_TOKENS = 32   # tokens that share a scale
ROPE_MAX = 4        # tensors of one launch
_CODE = {"i8": TMAC_CODE_I8, "e4m3": TMAC_CODE_E4M3}

EXPORTS = ["tmac_rotate", "tmac_pages_code_bytes", "tmac_pages_scale_bytes", "tmac_pages_append", "tmac_pages_read",
           "tmac_pages_attend_workspace_bytes", "tmac_pages_attend"]


class tmac_rope(C.Structure):
    _fields_ = [("freq_dev", C.c_void_p), ("magnitude", C.c_double), ("D", C.c_int32), ("rot", C.c_int32), ("interleaved", C.c_int32),
                ("elem", C.c_int32), ("reserved", C.c_int32 * 2)]


class tmac_rope_item(C.Structure):
    _fields_ = [("x", tmac_view), ("out", tmac_view), ("H", C.c_int32), ("reserved", C.c_int32)]


class tmac_pages(C.Structure):
    _fields_ = [("codes_dev", C.c_void_p), ("scales_dev", C.c_void_p), ("pages", C.c_int32), ("page", C.c_int32), ("Hkv", C.c_int32),
                ("D", C.c_int32), ("code", C.c_int32), ("reserved", C.c_int32 * 3)]


class tmac_pages_batch(C.Structure):
    _fields_ = [("table_dev", C.c_void_p), ("table_stride", C.c_int64), ("lens_dev", C.c_void_p), ("cu_dev", C.c_void_p), ("S", C.c_int32),
                ("width", C.c_int32), ("T", C.c_int32), ("most", C.c_int32)]


def _declare(lib):
    R, I, G, N, D, V = (C.POINTER(t) for t in (tmac_rope, tmac_rope_item, tmac_pages, tmac_pages_batch, tmac_attn_desc, tmac_view))
    P, I32, SZ = C.c_void_p, C.c_int32, C.c_size_t
    for name, result, args in [
            ("tmac_rotate", C.c_int, [R, I, I32, P, I32, P]),
            ("tmac_pages_code_bytes", SZ, [G]),
            ("tmac_pages_scale_bytes", SZ, [G]),
            ("tmac_pages_append", C.c_int, [G, N, I32, V, V, R, P, V, V, I32, P]),
            ("tmac_pages_read", C.c_int, [G, N, I32, V, V, P]),
            ("tmac_pages_attend_workspace_bytes", SZ, [D, G, N]),
            ("tmac_pages_attend", C.c_int, [D, G, N, V, V, P, P, SZ, P])]:
        f = getattr(lib, name)
        f.restype, f.argtypes = result, args
    return lib


lib = _declare(B.lib)
# (the ordinary calls go through the native side of the binding, as in attention.py)
calls = B.calls
calls.bind_pages(tmac_rope, tmac_pages, *(C.cast(getattr(lib, f), C.c_void_p).value for f in (
    "tmac_rotate", "tmac_pages_append", "tmac_pages_read", "tmac_pages_attend_workspace_bytes", "tmac_pages_attend")))


def _row_view(t) -> tmac_view:
    return A._view(t, None, 0, 1)


def frequencies(rot: int, base: float = 10000.0, scaling=None):
    """(radians a position of each of the rot / 2 pairs, fp64; what cosines and sines are multiplied with) for f_i = base^(-2 i / rot) and
    `scaling`, a context `factor` times as long as the `trained` one:

      None
      ("linear", factor)                      f_i / factor
      ("base", factor)                        base * factor^(rot / (rot - 2)): the slowest pair gets 1 / factor, the fastest stays
      ("ramp", factor, trained, fast, slow)   pairs that turn more than `fast` times in `trained` positions stay, those that turn less than
                                              `slow` times get f_i / factor, between them by pair number; magnitude 0.1 ln factor + 1
      ("bands", factor, trained, low, high)   pairs that turn more than `high` times stay, less than `low` times f_i / factor, between them by
                                              the number of turns
    """
    kind = "none" if scaling is None else scaling[0]
    numbers = () if scaling is None else tuple(float(x) for x in scaling[1:])
    if len(numbers) != {"none": 0, "linear": 1, "base": 1, "ramp": 4, "bands": 4}.get(kind, -1):
        raise ValueError(f"no such scaling of frequencies: {scaling!r}")
    if not all(math.isfinite(x) and x > 0 for x in numbers) or not (math.isfinite(base) and base > 1):
        raise ValueError(f"base ({base}) above one and scaling {scaling!r} of numbers above zero")
    if kind == "base":
        if rot < 4:
            raise ValueError('scaling "base" needs two pairs')
        base *= numbers[0] ** (rot / (rot - 2))
    i = torch.arange(rot // 2, dtype=torch.float64)
    f = base ** (-2.0 * i / rot)
    if kind == "linear":
        return f / numbers[0], 1.0
    if kind == "ramp":
        factor, trained, fast, slow = numbers
        if fast <= slow:
            raise ValueError(f"fast ({fast}) is above slow ({slow})")
        # the pair that turns so often in `trained` positions
        at = [rot * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (fast, slow)]
        lo, hi = max(0, math.floor(at[0])), min(rot - 1, math.ceil(at[1]))
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0
    if kind == "bands":
        factor, trained, low, high = numbers
        if high <= low:
            raise ValueError(f"high ({high}) is above low ({low})")
        mix = ((trained * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return f * (mix + (1 - mix) / factor), 1.0
    return f, 1.0


class Rotary:
    """Rotary positions of heads of D elements, of which the first `rot` turn (None: all): pairs (i, i + rot / 2), or (2 i, 2 i + 1) where
    `interleaved`.  base, scaling: see frequencies().  What it consists of is not replaced (calls go by the address of `freq`, and by sizes that are kept beside it)."""

    def __init__(self, D: int, rot: Optional[int] = None, base: float = 10000.0, interleaved: bool = False, scaling=None, device: str = "cuda"):
        rot = D if rot is None else rot
        if not 2 <= rot <= D or rot % 2:
            raise ValueError(f"rot ({rot}) is even and between 2 and D ({D})")
        f, self.magnitude = frequencies(rot, base, scaling)
        self.D, self.rot, self.interleaved = D, rot, bool(interleaved)
        self.freq = f.to(device)
        self.rope = {dt: tmac_rope(self.freq.data_ptr(), self.magnitude, D, rot, int(self.interleaved), elem) for dt, elem in A._ELEM.items()}

    def __setattr__(self, name, value):
        if self.__dict__.get(name, value) is not value:
            raise AttributeError(f"{name} is not replaced: make another Rotary")
        super().__setattr__(name, value)

    def _rope(self, dtype) -> tmac_rope:
        rope = self.rope[dtype]
        if self.freq.data_ptr() != rope.freq_dev:
            raise ValueError("freq has been moved to other memory: make another Rotary")
        return rope

    def rotate(self, positions, *tensors, out: Optional[Sequence] = None, stream=None):
        """Tensors [T, H, D] of the same T tokens (up to four, H their own) turned by positions int64 [T].  Returns a tuple of as many; `out`:
        where they go (a tensor itself: in place)."""
        if out is None and stream is None and tensors:
            rope = self.rope.get(tensors[0].dtype)
            got = rope and calls.rotate(rope, self.freq, positions, *tensors)
            if got is not None:
                return got
        if not 1 <= len(tensors) <= ROPE_MAX:
            raise ValueError(f"one to {ROPE_MAX} tensors, got {len(tensors)}")
        if out is not None and len(out) != len(tensors):
            raise ValueError(f"as many results as tensors: {len(out)}, {len(tensors)}")
        x = tensors[0]
        if x.dim() != 3 or x.dtype not in A._ELEM:
            raise ValueError(f"tensors are [T, H, D] of float16 or bfloat16, got {tuple(x.shape)} of {x.dtype}")
        rope = self._rope(x.dtype)
        T = x.shape[0]
        A._counted(T=T)
        for i, t in enumerate(tensors):
            A._dims(f"tensor {i}", t, "T, H, D", (T, -1, self.D), x.dtype)
            A._rows(f"tensor {i}", t)
            A._counted(H=t.shape[1])
        A._plain("positions", positions, (T,), torch.int64)
        with A._on(stream):
            got = tuple(torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in tensors) if out is None else tuple(out)
        for i, (t, o) in enumerate(zip(tensors, got)):
            A._dims(f"result {i}", o, "T, H, D", tuple(t.shape), x.dtype)
            A._rows(f"result {i}", o), A._apart(f"result {i}", o)
        A._same_device(self.freq, positions, *tensors, *got)
        pairs = [(t, o) for t, o in zip(tensors, got) if t.shape[1]]
        if T and pairs:
            items = (tmac_rope_item * len(pairs))(*(tmac_rope_item(_row_view(t), _row_view(o), t.shape[1]) for t, o in pairs))
            B._check(lib.tmac_rotate(rope, items, len(pairs), positions.data_ptr(), T, B._stream_ptr(stream)), "tmac_rotate")
        return got


class PagedCache:
    """Keys and values of one layer in `pages` pages of `page` tokens, in 8 bits: `code` "e4m3" or "i8", with a scale for every block of 32
    tokens and key head, for keys and for values.  dtype: of what is appended, of queries and results.  rotary: what turns keys and
    queries on their way in (None: they come as they are to be kept).

      codes   uint8 [pages, Hkv, page / 32, bytes of a block]   (the order within a block: include/tmac_pages.h)
      scales  fp32 [pages, Hkv, page / 32, 2]

    Sequences are given by each call: table int32 [S, width] (the sequences' pages, -1: none), lens int32 [S] (their tokens, those of the
    call included), and cu int32 [S + 1], by which the rows of the call's tensors are the sequences' last tokens (None: one row each);
    `most`: most rows of a sequence, where it is known.  Calls of one cache share its workspaces: on several streams they must not overlap.  Calls from
    several threads are enqueued one after the other, each whole.
    """

    def __init__(self, pages: int, Hkv: int, D: int, page: int = 64, code: str = "e4m3", dtype=torch.float16, rotary: Optional[Rotary] = None,
                 Hq: Optional[int] = None, scale: Optional[float] = None, device: str = "cuda"):
        if code not in _CODE:
            raise ValueError(f"code is one of {sorted(_CODE)}, got {code!r}")
        if rotary is not None and rotary.D != D:
            raise ValueError(f"rotary turns heads of {rotary.D} elements, the cache has {D}")
        self.Hkv, self.D, self.page, self.Hq = Hkv, D, page, Hkv if Hq is None else Hq
        self.dtype, self.rotary = dtype, rotary
        self.desc = A.attn_desc(self.Hq, Hkv, D, dtype, scale, True)
        self.cache = tmac_pages(None, None, pages, page, Hkv, D, _CODE[code])
        blocks = max(page, 0) // BLOCK_TOKENS
        nbytes = lib.tmac_pages_code_bytes(self.cache)
        if not nbytes and (pages or page < BLOCK_TOKENS):
            raise ValueError(f"pages ({pages}) of {BLOCK_TOKENS} to 4096 tokens, a power of two (got {page}), heads of a multiple of 4 up to "
                             f"128 elements (got {D}), at least one (got {Hkv})")
        self.codes = torch.zeros((pages, Hkv, blocks, nbytes // max(pages * Hkv * blocks, 1)), dtype=torch.uint8, device=device)
        self.scales = torch.zeros((pages, Hkv, blocks, 2), dtype=torch.float32, device=device)
        self.cache.codes_dev, self.cache.scales_dev = self.codes.data_ptr(), self.scales.data_ptr()
        # (a call is up to three launches that hand a workspace on, and the interpreter may change threads between them)
        self.lock = threading.RLock()
        self.attend_ws = None
        self.outgrown = []

    def __setattr__(self, name, value):
        if name in ("codes", "scales") and self.__dict__.get(name, value) is not value:
            raise AttributeError(f"{name} is written to, not replaced: {name}.copy_(...)")
        # (what tensors are checked against, and what the kernels go by)
        if name in ("Hkv", "D", "page", "Hq", "dtype", "desc", "cache") and self.__dict__.get(name, value) is not value:
            raise AttributeError(f"{name} is not replaced: make another PagedCache")
        if name == "rotary" and value is not None and value.D != self.D:
            raise ValueError(f"rotary turns heads of {value.D} elements, the cache has {self.D}")
        super().__setattr__(name, value)

    def _grown(self, n: int, stream):
        """A workspace of n bytes at least; one that is too small is kept, as KVCache does."""
        ws = self.attend_ws
        if ws is None or ws.numel() < n:
            if ws is not None:
                self.outgrown.append(ws)
                n = max(n, 2 * ws.numel())
            with A._on(stream):
                self.attend_ws = A._workspace(n, self.codes.device)
        return self.attend_ws

    def _batch(self, T: int, table, lens, cu, most) -> tmac_pages_batch:
        if any(t.data_ptr() != (at or 0) for t, at in ((self.codes, self.cache.codes_dev), (self.scales, self.cache.scales_dev))):
            raise ValueError("codes or scales have been moved to other memory: make another PagedCache")
        S = lens.shape[0] if isinstance(lens, torch.Tensor) and lens.dim() else 0
        A._plain("lens", lens, (S,), torch.int32)
        A._dims("table", table, "S, width", (S, -1), torch.int32)
        if table.shape[1] > 1 and table.stride(1) != 1:
            raise ValueError("the entries of a row of table lie side by side")
        if cu is None:
            if T != S:
                raise ValueError(f"without cu every sequence has one row: {T} rows, {S} sequences")
        else:
            A._plain("cu", cu, (S + 1,), torch.int32)
        A._counted(S=S, T=T, width=table.shape[1])
        most = 0 if most is None else int(most)
        if not 0 <= most < 1 << 31:
            raise ValueError(f"most ({most}) is a number of rows")
        stride = table.stride(0) if S > 1 else table.shape[1]
        if stride < table.shape[1]:
            raise ValueError("the rows of table do not overlap")
        return tmac_pages_batch(table.data_ptr(), stride, lens.data_ptr(), None if cu is None else cu.data_ptr(), S, table.shape[1], T, most)

    def append(self, k, v, table, lens, cu=None, q=None, positions=None, most: Optional[int] = None, q_out=None, stream=None):
        """k, v [T, Hkv, D], the last tokens of their sequences, into the pages; with `rotary`, keys are turned on the way, and so are the
        queries q [T, Hq, D] of the same tokens, if there are any, by positions int64 [T] (None: the tokens' places in their sequences).
        Returns the turned queries, or None.  Two sequences of a call must not write to the same page."""
        with self.lock:
            if stream is None and q_out is None:
                rotary = self.rotary
                got = calls.pages_append(self.cache, self.codes, self.desc, table, lens, cu, most, k, v,
                                         None if rotary is None else rotary.rope[self.dtype], None if rotary is None else rotary.freq, q, positions)
                if got is not None:
                    return None if q is None else got
            T = k.shape[0]
            for name, t in (("k", k), ("v", v)):
                A._dims(name, t, "T, Hkv, D", (T, self.Hkv, self.D), self.dtype)
                A._rows(name, t)
            batch = self._batch(T, table, lens, cu, most)
            rope = None if self.rotary is None else self.rotary._rope(self.dtype)
            if self.rotary is None and (q is not None or positions is not None):
                raise ValueError("a cache without rotary turns no queries and needs no positions")
            if q is None and q_out is not None:
                raise ValueError("a result for queries that are not there")
            if positions is not None:
                A._plain("positions", positions, (T,), torch.int64)
            views = [None, None]
            if q is not None:
                A._dims("q", q, "T, Hq, D", (T, self.Hq, self.D), self.dtype)
                A._rows("q", q)
                if q_out is None:
                    with A._on(stream):
                        q_out = torch.empty((T, self.Hq, self.D), dtype=self.dtype, device=q.device)
                A._dims("q_out", q_out, "T, Hq, D", (T, self.Hq, self.D), self.dtype)
                A._rows("q_out", q_out), A._apart("q_out", q_out)
                views = [_row_view(q), _row_view(q_out)]
            A._same_device(self.codes, k, v, table, lens, cu, q, q_out, positions, None if self.rotary is None else self.rotary.freq)
            if T:
                B._check(lib.tmac_pages_append(self.cache, batch, A._ELEM[self.dtype], _row_view(k), _row_view(v), rope,
                                               None if positions is None else positions.data_ptr(), *views, self.Hq, B._stream_ptr(stream)),
                         "tmac_pages_append")
            return q_out

    def read(self, table, lens, cu=None, T: Optional[int] = None, most: Optional[int] = None, k=None, v=None, stream=None):
        """The last tokens of the sequences as the pages hold them: (k, v) [T, Hkv, D].  T: cu's last entry, where it is known (else it is
        fetched, which waits for the GPU)."""
        with self.lock:
            if T is None:
                T = k.shape[0] if k is not None else lens.shape[0] if cu is None else int(cu[-1])
            if stream is None and k is None and v is None:
                got = calls.pages_read(self.cache, self.codes, self.desc, table, lens, cu, most, T)
                if got is not None:
                    return got
            batch = self._batch(T, table, lens, cu, most)
            with A._on(stream):
                k, v = (torch.empty((T, self.Hkv, self.D), dtype=self.dtype, device=self.codes.device) if t is None else t for t in (k, v))
            for name, t in (("k", k), ("v", v)):
                A._dims(name, t, "T, Hkv, D", (T, self.Hkv, self.D), self.dtype)
                A._rows(name, t), A._apart(name, t)
            A._same_device(self.codes, k, v, table, lens, cu)
            if T:
                B._check(lib.tmac_pages_read(self.cache, batch, A._ELEM[self.dtype], _row_view(k), _row_view(v), B._stream_ptr(stream)),
                         "tmac_pages_read")
            return k, v

    def attend(self, q, table, lens, cu=None, most: Optional[int] = None, out=None, lse=None, stream=None):
        """q [T, Hq, D], the last tokens of their sequences, over all tokens up to each that are in the pages.  Returns (out [T, Hq, D],
        lse fp32 [Hq, T])."""
        with self.lock:
            if out is None and lse is None and stream is None and self.attend_ws is not None:
                got = calls.pages_attend(self.cache, self.codes, self.desc, table, lens, cu, most, q, self.attend_ws)
                if got is not None:
                    return got
            T = q.shape[0]
            A._dims("q", q, "T, Hq, D", (T, self.Hq, self.D), self.dtype)
            A._rows("q", q)
            batch = self._batch(T, table, lens, cu, most)
            with A._on(stream):
                if out is None:
                    out = torch.empty((T, self.Hq, self.D), dtype=self.dtype, device=q.device)
                if lse is None:
                    lse = torch.empty((self.Hq, T), dtype=torch.float32, device=q.device)
            A._dims("out", out, "T, Hq, D", (T, self.Hq, self.D), self.dtype)
            A._rows("out", out), A._apart("out", out)
            A._plain("lse", lse, (self.Hq, T), torch.float32)
            A._same_device(self.codes, q, out, lse, table, lens, cu)
            if T:
                n = lib.tmac_pages_attend_workspace_bytes(self.desc, self.cache, batch)
                B._check(lib.tmac_pages_attend(self.desc, self.cache, batch, _row_view(q), _row_view(out), lse.data_ptr(), self._grown(n, stream).data_ptr(),
                                               n, B._stream_ptr(stream)), "tmac_pages_attend")
            return out, lse


class PageTable:
    """Which pages belong to which of `batch` sequences, and how many tokens these have, on the host and on the GPU:

      table  int32 [batch, width]  pages of each sequence, -1 behind them       lens  int32 [batch]

    The tensors keep their place (a captured graph that was given them sees what extend() and the others put there since).  These copy from the host and wait for the
    GPU's stream: a step that is captured has them outside.
    """

    def __init__(self, batch: int, width: int, pages: int, page: int = 64, device: str = "cuda"):
        if min(batch, width, pages, page) < 1:
            raise ValueError(f"batch ({batch}), width ({width}), pages ({pages}) and page ({page}) are above zero")
        self.batch, self.width, self.page = batch, width, page
        self.free = list(range(pages - 1, -1, -1))
        self.owned = [[] for _ in range(batch)]
        self.length = [0] * batch
        self.table = torch.full((batch, width), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=device)

    def _write(self, table: bool) -> None:
        self.lens.copy_(torch.tensor(self.length, dtype=torch.int32))
        if table:
            self.table.copy_(torch.tensor([own + [-1] * (self.width - len(own)) for own in self.owned], dtype=torch.int32))

    def extend(self, counts: Sequence[int]):
        """Room for so many more tokens of each sequence.  Returns (cu int32 [batch + 1], the most of one sequence) for the calls that are
        about these tokens.  Without room for all of them nothing changes."""
        if len(counts) != self.batch or min(counts) < 0:
            raise ValueError(f"a count for each of {self.batch} sequences, got {list(counts)}")
        need = [-(-(n + c) // self.page) - len(own) for n, c, own in zip(self.length, counts, self.owned)]
        if any(len(own) + n > self.width for own, n in zip(self.owned, need)):
            raise ValueError(f"a sequence has at most {self.width} pages of {self.page} tokens")
        if sum(need) > len(self.free):
            raise MemoryError(f"{sum(need)} pages are needed, {len(self.free)} are free")
        for s, n in enumerate(need):
            self.owned[s] += [self.free.pop() for _ in range(n)]
            self.length[s] += counts[s]
        self._write(any(need))
        cu = torch.zeros(self.batch + 1, dtype=torch.int32)
        torch.cumsum(torch.tensor(counts, dtype=torch.int32), 0, out=cu[1:])
        return cu.to(self.lens.device), max(counts)

    def take_back(self, counts: Sequence[int]) -> None:
        """The last tokens of each sequence leave (drafts that were not accepted, or all of a sequence that has ended); pages that hold none any
        more are free again."""
        if len(counts) != self.batch or any(not 0 <= c <= n for c, n in zip(counts, self.length)):
            raise ValueError(f"of each sequence at most as many as it has ({self.length}), got {list(counts)}")
        freed = False
        for s, c in enumerate(counts):
            self.length[s] -= c
            keep = -(-self.length[s] // self.page)
            freed |= len(self.owned[s]) > keep
            self.free += reversed(self.owned[s][keep:])
            del self.owned[s][keep:]
        self._write(freed)
