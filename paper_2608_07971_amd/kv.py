"""Python binding of the paged 8-bit key/value cache (include/esp_kv.h).

The functions carry the names of the C-ABI and only marshal arguments; `Rope`
and `PagedCache` own the tensors.  A step of an offline-inference job:

    cache.resize(lengths)                            # room for the new tokens
    q = cache.append(layer, k, v, offsets, rope=rope, q=q)
    out, lse = cache.attend(layer, q, offsets, max_new=1)

`fork`, `resize` and `compact` make a changed batch or memory budget real.
There is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Optional

import torch

from . import ESP_OK, EspError, lib as _base_lib

_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice

BF16, FP16, FP32 = 0, 1, 2
_TYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}
CODES = torch.float8_e4m3fn


class esp_kv_cache(C.Structure):
    _fields_ = [("pages", C.c_int32), ("layers", C.c_int32), ("kv_heads", C.c_int32), ("page_tokens", C.c_int32),
                ("head_dim", C.c_int32), ("sequences", C.c_int32), ("table_width", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("scale", C.c_void_p), ("table", C.c_void_p),
                ("lengths", C.c_void_p), ("refs", C.c_void_p), ("status", C.c_void_p)]


class esp_kv_rope(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("magnitude", C.c_float), ("rotary_dim", C.c_int32), ("interleaved", C.c_int32)]


class esp_kv_view(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


_P, _I, _L, _V, _Z = C.c_void_p, C.c_int32, C.c_int64, esp_kv_view, C.POINTER(C.c_size_t)

# Every entry point of include/esp_kv.h with its ctypes signature.
_SIGS = {
    "esp_kv_rope_turns": [_I, C.c_double, _I, C.c_double, _I, _P, C.POINTER(C.c_float)],
    "esp_kv_rotate": [_P, _I, _L, _I, _I, _V, _P, _I, _V, _P],
    "esp_kv_append": [_P, _I, _I, _I, _L, _P, _P, _V, _V, _P, _I, _V, _V, _P],
    "esp_kv_gather": [_P, _I, _I, _I, _L, _P, _P, _P, _P, _P, _P],
    "esp_kv_attend_workspace": [_P, _I, _L, _I, _I, _I, _Z],
    "esp_kv_attend": [_P, _I, _I, _I, _L, _P, _P, _I, _V, C.c_float, _I, _I, _I, _V, _P, _P, C.c_size_t, _P],
    "esp_kv_pages_workspace": [_P, _I, _Z],
    "esp_kv_resize": [_P, _P, _P, C.c_size_t, _P],
    "esp_kv_fork": [_P, _I, _P, _P, _P, C.c_size_t, _P],
    "esp_kv_compact": [_P, _I, _P, _P, _P, _P, C.c_size_t, _P],
    "esp_kv_device_status": [_P, _P],
}

_lib = None


def lib():
    """libesp.so with the entry points of esp_kv.h (raises when it has not been built)."""
    global _lib
    if _lib is None:
        L = _base_lib()
        for name, args in _SIGS.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, C.c_int
        L.hipStreamGetCaptureInfo.argtypes = [_P, C.POINTER(C.c_int), C.POINTER(C.c_ulonglong)]
        _lib = L
    return _lib


def _capture(stream: int):
    """What tells the capture that the current stream (of this handle) is in from others; None outside of one."""
    if not torch.cuda.is_current_stream_capturing():
        return None
    status, number = C.c_int(0), C.c_ulonglong(0)
    return number.value if lib().hipStreamGetCaptureInfo(stream, C.byref(status), C.byref(number)) == 0 else object()


def _check(code: int, where: str) -> None:
    if code != ESP_OK:
        raise EspError(code, where)


def _on_stream(call):
    """call(..., s): with the handle of the stream that the work goes to, on its device, so that what the call
    allocates belongs to that stream.  The current stream of the current device costs no context.  A stream that is
    given is noted at the tensors that it is to read, so that the allocator keeps those that the caller drops."""
    @functools.wraps(call)
    def entry(first, *args, stream=None, **more):
        index = first.index
        if stream is None and _current_device() == index:
            return call(first, *args, s=_raw_stream(index), **more)
        if stream is None:
            with torch.cuda.device(index):
                return call(first, *args, s=_raw_stream(index), **more)
        own = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=first.device)
        with torch.cuda.stream(own):
            result = call(first, *args, s=int(own.cuda_stream), **more)
        for x in (first, *args, *more.values()):
            for t in (x,) if isinstance(x, torch.Tensor) else getattr(x, "tensors", ()):
                t.record_stream(own)
        return result
    return entry


def _ints(t, n: Optional[int], what: str, device) -> int:
    """Address of a contiguous int32 device vector (of n values)."""
    if t.dtype != torch.int32 or t.device != device or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{what}: contiguous int32 tensor{'' if n is None else f' of {n} values'} on {device} expected")
    return t.data_ptr()


def _view(t, tokens: int, heads: int, dim: int, what: str, device) -> esp_kv_view:
    if t.shape != (tokens, heads, dim) or t.device != device:
        raise ValueError(f"{what}: tensor [{tokens}, {heads}, {dim}] on {device} expected")
    a, b, c = t.stride()
    if c != 1 and dim > 1 and t.numel():
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return esp_kv_view(t.data_ptr(), a, b)


_NO_VIEW = esp_kv_view(None, 0, 0)


def esp_kv_rope_turns(rotary_dim: int, base: float, scaling: int, factor: float, context: int):
    turns = (C.c_double * max(1, rotary_dim // 2))()
    magnitude = C.c_float(0.0)
    _check(lib().esp_kv_rope_turns(int(rotary_dim), float(base), int(scaling), float(factor), int(context),
                                   C.cast(turns, C.c_void_p), C.byref(magnitude)), "esp_kv_rope_turns")
    return list(turns), float(magnitude.value)


class Rope:
    """Rotary positions of heads of head_dim elements, the first rotary_dim of them turned.  scaling: "none",
    "linear", "ntk" or "parts" (by factor, from a first context of `context` tokens)."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, base: float = 10000.0, interleaved: bool = False,
                 scaling: str = "none", factor: float = 1.0, context: int = 0, device="cuda:0"):
        if scaling not in SCALINGS:
            raise ValueError(f"scaling: one of {sorted(SCALINGS)} expected")
        self.head_dim, self.rotary_dim = int(head_dim), int(head_dim if rotary_dim is None else rotary_dim)
        turns, self.magnitude = esp_kv_rope_turns(self.rotary_dim, base, SCALINGS[scaling], factor, context)
        if self.rotary_dim > self.head_dim:
            raise ValueError("rotary_dim exceeds head_dim")
        self.turns = torch.tensor(turns, dtype=torch.float64, device=device)
        self.device, self.index, self.tensors = self.turns.device, self.turns.device.index, (self.turns,)
        self.c = esp_kv_rope(self.turns.data_ptr(), self.magnitude, self.rotary_dim, int(bool(interleaved)))
        self.ptr = C.addressof(self.c)


@_on_stream
def rotate(rope: Rope, x: torch.Tensor, positions: torch.Tensor, inverse: bool = False, out: Optional[torch.Tensor] = None,
           *, s: int) -> torch.Tensor:
    """x [tokens, heads, head_dim] turned by positions (int32 [tokens]); inverse: turned back, which is the gradient, and
    what backward() does.  out may be x.  stream: the current one, unless given."""
    if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
        return _Turned.apply(x, None if out is x else out, out is x, rope, positions, inverse, s)
    return _turn(rope, x, positions, inverse, out, s)


class _Turned(torch.autograd.Function):
    """rotate with its gradient: the rotation times magnitude, transposed."""

    @staticmethod
    def forward(ctx, x, out, in_place, rope, positions, inverse, s):
        if in_place:
            out = x
        if out is not None:
            ctx.mark_dirty(out)
        ctx.rope, ctx.inverse = rope, inverse
        ctx.save_for_backward(positions)
        return _turn(rope, x, positions, inverse, out, s)

    @staticmethod
    def backward(ctx, grad):
        positions, = ctx.saved_tensors
        if grad.stride(-1) != 1:
            grad = grad.contiguous()
        return rotate(ctx.rope, grad, positions, inverse=not ctx.inverse), None, None, None, None, None, None


class _NoGradient(torch.autograd.Function):
    """A result that depends on tensors that require gradients, through what has none: backward() says so."""

    @staticmethod
    def forward(ctx, what, source, result):
        ctx.what = what
        ctx.mark_dirty(result)
        return result

    @staticmethod
    def backward(ctx, grad):
        raise RuntimeError(f"{ctx.what} has no gradient: the cache holds its tokens rounded to 8 bits. Detach its inputs, or "
                           "call it under torch.no_grad()")


def _turn(rope, x, positions, inverse, out, s: int) -> torch.Tensor:
    kind = _TYPES.get(x.dtype)
    if kind is None or x.dim() != 3 or x.device != rope.device:
        raise ValueError(f"x: bfloat16, float16 or float32 tensor [tokens, heads, head_dim] on {rope.device} expected")
    T, H, D = x.shape
    if D != rope.head_dim:
        raise ValueError(f"x: heads of {rope.head_dim} elements expected")
    if out is None:
        out = torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    elif out.dtype != x.dtype:
        raise ValueError("out: the type of x expected")
    _check(lib().esp_kv_rotate(rope.ptr, kind, T, H, D, _view(x, T, H, D, "x", x.device), _ints(positions, T, "positions", x.device),
                               1 if inverse else 0, _view(out, T, H, D, "out", x.device), s), "esp_kv_rotate")
    return out


class PagedCache:
    """Pages of keys and values in 8 bits, shared by the sequences of a batch.  The tensors k, v, scale, table,
    lengths and refs are as include/esp_kv.h lays them out."""

    def __init__(self, pages: int, page_tokens: int, kv_heads: int, head_dim: int, sequences: int, table_width: int,
                 layers: int = 1, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU: the cache has no CPU path")
        d = torch.device(device)
        self._set(torch.zeros((pages, layers, kv_heads, page_tokens, head_dim), dtype=torch.uint8, device=d).view(CODES),
                  torch.zeros((pages, layers, kv_heads, head_dim, page_tokens), dtype=torch.uint8, device=d).view(CODES),
                  torch.zeros((pages, layers, 2, kv_heads), dtype=torch.float32, device=d),
                  torch.full((sequences, table_width), -1, dtype=torch.int32, device=d),
                  torch.zeros(sequences, dtype=torch.int32, device=d), torch.zeros(pages, dtype=torch.int32, device=d))

    @classmethod
    def adopt(cls, k, v, scale, table, lengths, refs) -> "PagedCache":
        """A cache over tensors that the caller filled."""
        self = cls.__new__(cls)
        self._set(k, v, scale, table, lengths, refs)
        return self

    def _set(self, k, v, scale, table, lengths, refs) -> None:
        P, L, H, T, D = k.shape
        want = {"k": (k, (P, L, H, T, D), CODES), "v": (v, (P, L, H, D, T), CODES), "scale": (scale, (P, L, 2, H), torch.float32),
                "table": (table, (table.shape[0], table.shape[-1]), torch.int32), "lengths": (lengths, (table.shape[0],), torch.int32),
                "refs": (refs, (P,), torch.int32)}
        for name, (t, shape, dtype) in want.items():
            if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous() or t.device != k.device or not t.is_cuda:
                raise ValueError(f"{name}: contiguous {dtype} device tensor of shape {shape} expected")
        self.k, self.v, self.scale, self.table, self.lengths, self.refs = k, v, scale, table, lengths, refs
        self.device, self.index = k.device, k.device.index
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.tensors = (k, v, scale, table, lengths, refs, self.status)
        self.pages, self.layers, self.kv_heads, self.page_tokens, self.head_dim = P, L, H, T, D
        self.sequences, self.table_width = table.shape
        self._work, self._graph_work, self._sizes = {}, (None, {}), {}
        self._scale, self._pages_bytes = D ** -0.5, None
        self._source = None                     # requires gradients once tokens were appended that do
        # kernels and captured graphs take the addresses by value: the tensors stay for the cache's life
        self.c = esp_kv_cache(self.pages, self.layers, self.kv_heads, self.page_tokens, self.head_dim, self.sequences,
                              self.table_width, self.k.data_ptr(), self.v.data_ptr(), self.scale.data_ptr(), self.table.data_ptr(),
                              self.lengths.data_ptr(), self.refs.data_ptr(), self.status.data_ptr())
        self.ptr = C.addressof(self.c)

    @property
    def page_bytes(self) -> int:
        """Bytes of one page: what a configuration's memory demand counts."""
        return 2 * self.layers * self.kv_heads * (self.page_tokens * self.head_dim + 4)

    def _workspace(self, kind: str, size, stream: int) -> torch.Tensor:
        """Scratch of this kind of call on this stream, kept and grown.  Calls that are captured share scratch of their
        graph instead, which may be replayed beside other work of any stream: its first use clears it in every replay."""
        capture = _capture(stream)
        if capture is None:
            kept = self._work
        else:
            if capture != self._graph_work[0]:
                self._graph_work = capture, {}
            kept = self._graph_work[1]
        w = kept.get((kind, stream))
        if w is None or w.numel() < size:
            if w is not None and capture is None:
                size = max(size, 2 * w.numel())
            w = torch.empty(max(size, 256), dtype=torch.uint8, device=self.device)
            if kind == "attend":
                w[:4 * (768 + self.kv_heads)].zero_()
            kept[(kind, stream)] = w
        return w

    def _results(self, what: str, q, *results):
        """The results of a call on q, and on what the cache holds, whose gradients would be lost."""
        if not torch.is_grad_enabled():
            return results
        source = q if q is not None and q.requires_grad else self._source
        return results if source is None else tuple(_NoGradient.apply("PagedCache." + what, source, r) for r in results)

    def _rows(self, offsets, seqs):
        rows = offsets.numel() - 1
        if rows < 0 or (seqs is None and rows > self.sequences):
            raise ValueError("offsets: [rows + 1] expected, with no more rows than sequences")
        return rows, _ints(offsets, None, "offsets", self.device), None if seqs is None else _ints(seqs, rows, "seqs", self.device)

    @_on_stream
    def append(self, layer: int, k, v, offsets, rope: Optional[Rope] = None, q=None, seqs=None, *, s: int):
        """Writes the new tokens k, v [tokens, kv_heads, head_dim], the last ones of their sequences, rows cut by
        offsets (int32 [rows + 1]); q [tokens, q_heads, head_dim] is turned too and returned.  No gradient goes through
        the cache or this turning (rotate has one): backward() raises where one would be lost."""
        kind = _TYPES.get(k.dtype)
        if kind is None or kind == FP32 or k.dim() != 3 or v.dtype != k.dtype or (q is not None and (q.dtype != k.dtype or q.dim() != 3)):
            raise ValueError("k, v and q: bfloat16 or float16 [tokens, heads, head_dim] expected, of one type")
        if rope is not None and (rope.head_dim != self.head_dim or rope.index != self.index):
            raise ValueError("rope: made for another head_dim or device")
        if q is not None and rope is None:
            raise ValueError("q is given to be turned: rope expected")
        T, H, D, dev = k.shape[0], self.kv_heads, self.head_dim, self.device
        rows, off, sq = self._rows(offsets, seqs)
        out, heads, vq, vo = None, 0, _NO_VIEW, _NO_VIEW
        if q is not None:
            heads = q.shape[1]
            if q.numel() and (q.data_ptr() % 16 or q.stride(0) % 8 or q.stride(1) % 8):
                q = q.clone(memory_format=torch.contiguous_format)    # also of one that is contiguous at an odd place
            out = torch.empty_like(q) if q.is_contiguous() else torch.empty(q.shape, dtype=q.dtype, device=dev)
            vq, vo = _view(q, T, heads, D, "q", dev), _view(out, T, heads, D, "q", dev)
        _check(lib().esp_kv_append(self.ptr, layer, kind, rows, T, off, sq, _view(k, T, H, D, "k", dev), _view(v, T, H, D, "v", dev),
                                   None if rope is None else rope.ptr, heads, vq, vo, s), "esp_kv_append")
        if torch.is_grad_enabled() and (k.requires_grad or v.requires_grad) and self._source is None:
            self._source = torch.zeros((), requires_grad=True)
        return out if out is None or not q.requires_grad else self._results("append", q, out)[0]

    @_on_stream
    def gather(self, layer: int, starts, offsets, tokens: int, dtype=torch.bfloat16, seqs=None, *, s: int):
        """Keys and values [tokens, kv_heads, head_dim] of row b's tokens from starts[b] on, as numbers; `tokens` is
        the last of offsets."""
        kind = _TYPES.get(dtype)
        if kind is None or kind == FP32:
            raise ValueError("dtype: bfloat16 or float16 expected")
        rows, off, sq = self._rows(offsets, seqs)
        both = torch.empty((2, tokens, self.kv_heads, self.head_dim), dtype=dtype, device=self.device)
        k, v = both[0], both[1]
        _check(lib().esp_kv_gather(self.ptr, layer, kind, rows, tokens, off, sq, _ints(starts, rows, "starts", self.device),
                                   k.data_ptr(), v.data_ptr(), s), "esp_kv_gather")
        return self._results("gather", None, k, v)

    @_on_stream
    def attend(self, layer: int, q, offsets, scale: Optional[float] = None, window: int = 0, max_new: Optional[int] = None,
               max_length: Optional[int] = None, out=None, lse: bool = True, seqs=None, *, s: int):
        """(out, lse) of q [tokens, q_heads, head_dim] over the cache; scale defaults to head_dim ** -0.5.  max_new and
        max_length bound the rows' tokens and the sequences' lengths (default: what the shapes allow, with which a call
        may take up to a tenth longer).  Rows that are left out leave out and lse as they were.  No gradient:
        backward() raises where one would be lost."""
        kind = _TYPES.get(q.dtype)
        if kind is None or kind == FP32 or q.dim() != 3:
            raise ValueError("q: bfloat16 or float16 [tokens, q_heads, head_dim] expected")
        T, H, D = q.shape
        rows, off, sq = self._rows(offsets, seqs)
        if scale is None:
            scale = self._scale
        if max_new is None:
            max_new = T
        if max_length is None:
            max_length = self.table_width * self.page_tokens
        shape = (rows, T, H, max_new, max_length)
        size = self._sizes.get(shape)
        if size is None:
            n = C.c_size_t(0)
            _check(lib().esp_kv_attend_workspace(self.ptr, *shape, C.byref(n)), "esp_kv_attend_workspace")
            if len(self._sizes) >= 4096:
                self._sizes.clear()
            size = self._sizes[shape] = n.value
        if out is None:
            out = torch.empty_like(q) if q.is_contiguous() else torch.empty(q.shape, dtype=q.dtype, device=self.device)
        elif out.dtype != q.dtype:
            raise ValueError("out: the type of q expected")
        stats = torch.empty((T, H), dtype=torch.float32, device=self.device) if lse else None
        w = self._workspace("attend", size, s)
        _check(lib().esp_kv_attend(self.ptr, layer, kind, rows, T, off, sq, H, _view(q, T, H, self.head_dim, "q", self.device), scale,
                                   window, max_new, max_length, _view(out, T, H, self.head_dim, "out", self.device),
                                   None if stats is None else stats.data_ptr(), w.data_ptr(), w.numel(), s), "esp_kv_attend")
        if stats is None:
            return self._results("attend", q, out)[0], None
        return self._results("attend", q, out, stats)

    def _pages_work(self, stream: int) -> torch.Tensor:
        if self._pages_bytes is None:
            z = C.c_size_t(0)
            _check(lib().esp_kv_pages_workspace(self.ptr, self.sequences, C.byref(z)), "esp_kv_pages_workspace")
            self._pages_bytes = z.value
        return self._workspace("pages", self._pages_bytes, stream)

    @_on_stream
    def resize(self, lengths, *, s: int) -> None:
        """Sets every sequence's length (int32 [sequences]): pages are freed and the lowest free ones taken."""
        w = self._pages_work(s)
        _check(lib().esp_kv_resize(self.ptr, _ints(lengths, self.sequences, "lengths", self.device), w.data_ptr(), w.numel(), s),
               "esp_kv_resize")

    @_on_stream
    def fork(self, parents, children, *, s: int) -> None:
        """children[i] drops its pages and continues parents[i] (int32 [n] each)."""
        n = parents.numel()
        w = self._pages_work(s)
        _check(lib().esp_kv_fork(self.ptr, n, _ints(parents, n, "parents", self.device), _ints(children, n, "children", self.device),
                                 w.data_ptr(), w.numel(), s), "esp_kv_fork")

    @_on_stream
    def compact(self, limit: Optional[int] = None, *, s: int):
        """(table, refs, live) with no live page from `limit` on (None: from the number of live pages on).  The cache
        goes on with its old table, whose pages stay intact, until `install` is given the new one.  The pool keeps its
        size; `adopt` over clones of its first pages is a smaller one."""
        table, refs = torch.empty_like(self.table), torch.empty_like(self.refs)
        live = torch.empty((), dtype=torch.int32, device=self.device)
        w = self._pages_work(s)
        _check(lib().esp_kv_compact(self.ptr, -1 if limit is None else limit, table.data_ptr(), refs.data_ptr(), live.data_ptr(),
                                    w.data_ptr(), w.numel(), s), "esp_kv_compact")
        return table, refs, live

    @_on_stream
    def install(self, table, refs, *, s: int) -> None:
        """Takes the table and references of a compaction: copied into the cache's own tensors in stream order, so that
        captured graphs and calls already enqueued go on naming live memory.  Readers on other streams see the old or
        the new places, which hold the same until a later call writes pages: order them before that one."""
        _ints(table, self.table.numel(), "table", self.device)
        _ints(refs, self.pages, "refs", self.device)
        if table.shape != self.table.shape:
            raise ValueError("table: the cache's shape expected")
        self.table.copy_(table)
        self.refs.copy_(refs)

    @_on_stream
    def device_status(self, *, s: int) -> int:
        """The first error that the GPU recorded since the last call (waits for the stream).  After one, calls take new
        scratch: lengths that changed under a call may have left the old with parts that it waits for."""
        code = int(lib().esp_kv_device_status(self.ptr, s))
        if code != ESP_OK:
            self._work.clear()
        return code
