"""Python binding of the paged 8-bit key/value cache (include/esp_kv.h).

The functions carry the names of the C-ABI and only marshal arguments; `Rope`
and `PagedCache` own the tensors.  A step of an offline-inference job:

    cache.resize(lengths)                            # room for the new tokens
    q = cache.append(layer, k, v, offsets, rope=rope, q=q)
    out, lse = cache.attend(layer, q, offsets)

`fork`, `resize` and `compact` make a changed batch or memory budget real.
There is no CPU fallback.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional

import torch

from . import ESP_OK, EspError, _stream, lib as _base_lib

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
        _lib = L
    return _lib


def _check(code: int, where: str) -> None:
    if code != ESP_OK:
        raise EspError(code, where)


@contextlib.contextmanager
def _on(stream, device):
    """What the call allocates belongs to the stream it runs on."""
    if stream is None:
        with torch.cuda.device(device):
            yield _stream(None)
        return
    s = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device=device)
    with torch.cuda.stream(s):
        yield int(s.cuda_stream)


def _ints(t, n: Optional[int], what: str, device) -> int:
    """Address of a contiguous int32 device vector (of n values)."""
    if t.dtype != torch.int32 or t.device != device or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{what}: contiguous int32 tensor{'' if n is None else f' of {n} values'} on {device} expected")
    return t.data_ptr()


def _view(t, tokens: int, heads: int, dim: int, what: str, device) -> esp_kv_view:
    if t.dim() != 3 or tuple(t.shape) != (tokens, heads, dim) or t.device != device:
        raise ValueError(f"{what}: tensor [{tokens}, {heads}, {dim}] on {device} expected")
    if t.numel() and dim > 1 and t.stride(2) != 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return esp_kv_view(t.data_ptr(), t.stride(0), t.stride(1))


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
        self.c = esp_kv_rope(self.turns.data_ptr(), self.magnitude, self.rotary_dim, int(bool(interleaved)))
        self.ptr = C.addressof(self.c)


def rotate(rope: Rope, x: torch.Tensor, positions: torch.Tensor, inverse: bool = False, out: Optional[torch.Tensor] = None,
           stream=None) -> torch.Tensor:
    """x [tokens, heads, head_dim] turned by positions (int32 [tokens]); inverse: turned back, which is the gradient.
    out may be x."""
    if x.dim() != 3 or x.dtype not in _TYPES or not x.is_cuda:
        raise ValueError("x: bfloat16, float16 or float32 device tensor [tokens, heads, head_dim] expected")
    T, H, D = x.shape
    if D != rope.head_dim:
        raise ValueError(f"x: heads of {rope.head_dim} elements expected")
    with _on(stream, x.device) as s:
        if out is None:
            out = torch.empty((T, H, D), dtype=x.dtype, device=x.device)
        if out.dtype != x.dtype:
            raise ValueError("out: the type of x expected")
        _check(lib().esp_kv_rotate(rope.ptr, _TYPES[x.dtype], T, H, D, _view(x, T, H, D, "x", x.device),
                                   _ints(positions, T, "positions", x.device), int(bool(inverse)),
                                   _view(out, T, H, D, "out", x.device), s), "esp_kv_rotate")
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
        self.device = k.device
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.pages, self.layers, self.kv_heads, self.page_tokens, self.head_dim = P, L, H, T, D
        self.sequences, self.table_width = table.shape
        self._work = {}
        self._describe()

    def _describe(self) -> None:
        self.c = esp_kv_cache(self.pages, self.layers, self.kv_heads, self.page_tokens, self.head_dim, self.sequences,
                              self.table_width, self.k.data_ptr(), self.v.data_ptr(), self.scale.data_ptr(), self.table.data_ptr(),
                              self.lengths.data_ptr(), self.refs.data_ptr(), self.status.data_ptr())
        self.ptr = C.addressof(self.c)

    @property
    def page_bytes(self) -> int:
        """Bytes of one page: what a configuration's memory demand counts."""
        return 2 * self.layers * self.kv_heads * (self.page_tokens * self.head_dim + 4)

    def _workspace(self, kind: str, size, stream: int) -> torch.Tensor:
        """Scratch of this kind of call on this stream, kept and grown."""
        w = self._work.get((kind, stream))
        if w is None or w.numel() < size:
            w = torch.zeros(max(size, 256), dtype=torch.uint8, device=self.device)
            self._work[(kind, stream)] = w
        return w

    def _rows(self, offsets, seqs):
        if offsets.numel() < 1:
            raise ValueError("offsets: [rows + 1] expected")
        rows = offsets.numel() - 1
        if seqs is None and rows > self.sequences:
            raise ValueError("more rows than sequences")
        return rows, _ints(offsets, None, "offsets", self.device), None if seqs is None else _ints(seqs, rows, "seqs", self.device)

    def append(self, layer: int, k, v, offsets, rope: Optional[Rope] = None, q=None, seqs=None, stream=None):
        """Writes the new tokens k, v [tokens, kv_heads, head_dim], the last ones of their sequences, rows cut by
        offsets (int32 [rows + 1]); q [tokens, q_heads, head_dim] is turned too and returned."""
        if k.dim() != 3 or k.dtype not in (torch.bfloat16, torch.float16) or v.dtype != k.dtype or (q is not None and q.dtype != k.dtype):
            raise ValueError("k, v and q: bfloat16 or float16 [tokens, heads, head_dim] expected, of one type")
        if rope is not None and rope.head_dim != self.head_dim:
            raise ValueError("rope: made for another head_dim")
        if q is not None and rope is None:
            raise ValueError("q is given to be turned: rope expected")
        T, H, D = k.shape[0], self.kv_heads, self.head_dim
        rows, off, sq = self._rows(offsets, seqs)
        with _on(stream, self.device) as s:
            out, heads, vq, vo = None, 0, _NO_VIEW, _NO_VIEW
            if q is not None:
                heads = q.shape[1]
                if q.numel() and (q.data_ptr() % 16 or q.stride(0) % 8 or q.stride(1) % 8):
                    q = q.contiguous()
                out = torch.empty((T, heads, D), dtype=q.dtype, device=self.device)
                vq, vo = _view(q, T, heads, D, "q", self.device), _view(out, T, heads, D, "q", self.device)
            _check(lib().esp_kv_append(self.ptr, int(layer), _TYPES[k.dtype], rows, T, off, sq, _view(k, T, H, D, "k", self.device),
                                       _view(v, T, H, D, "v", self.device), None if rope is None else rope.ptr, heads, vq, vo, s),
                   "esp_kv_append")
        return out

    def gather(self, layer: int, starts, offsets, tokens: int, dtype=torch.bfloat16, seqs=None, stream=None):
        """Keys and values [tokens, kv_heads, head_dim] of row b's tokens from starts[b] on, as numbers; `tokens` is
        the last of offsets."""
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("dtype: bfloat16 or float16 expected")
        rows, off, sq = self._rows(offsets, seqs)
        with _on(stream, self.device) as s:
            k, v = (torch.empty((tokens, self.kv_heads, self.head_dim), dtype=dtype, device=self.device) for _ in range(2))
            _check(lib().esp_kv_gather(self.ptr, int(layer), _TYPES[dtype], rows, int(tokens), off, sq,
                                       _ints(starts, rows, "starts", self.device), k.data_ptr(), v.data_ptr(), s), "esp_kv_gather")
        return k, v

    def attend(self, layer: int, q, offsets, scale: Optional[float] = None, window: int = 0, max_new: Optional[int] = None,
               max_length: Optional[int] = None, out=None, lse: bool = True, seqs=None, stream=None):
        """(out, lse) of q [tokens, q_heads, head_dim] over the cache; scale defaults to head_dim ** -0.5.  max_new and
        max_length bound the rows' tokens and the sequences' lengths (default: what the shapes allow)."""
        if q.dim() != 3 or q.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("q: bfloat16 or float16 [tokens, q_heads, head_dim] expected")
        T, H, D = q.shape[0], q.shape[1], self.head_dim
        rows, off, sq = self._rows(offsets, seqs)
        scale = D ** -0.5 if scale is None else float(scale)
        max_new = T if max_new is None else int(max_new)
        max_length = self.table_width * self.page_tokens if max_length is None else int(max_length)
        n = C.c_size_t(0)
        _check(lib().esp_kv_attend_workspace(self.ptr, rows, T, H, max_new, max_length, C.byref(n)), "esp_kv_attend_workspace")
        with _on(stream, self.device) as s:
            if out is None:
                out = torch.empty((T, H, D), dtype=q.dtype, device=self.device)
            if out.dtype != q.dtype:
                raise ValueError("out: the type of q expected")
            stats = torch.empty((T, H), dtype=torch.float32, device=self.device) if lse else None
            w = self._workspace("attend", n.value, s)
            _check(lib().esp_kv_attend(self.ptr, int(layer), _TYPES[q.dtype], rows, T, off, sq, H, _view(q, T, H, D, "q", self.device),
                                       scale, int(window), max_new, max_length, _view(out, T, H, D, "out", self.device),
                                       None if stats is None else stats.data_ptr(), w.data_ptr(), w.numel(), s), "esp_kv_attend")
        return out, stats

    def _pages_work(self, n: int, stream: int) -> torch.Tensor:
        z = C.c_size_t(0)
        _check(lib().esp_kv_pages_workspace(self.ptr, n, C.byref(z)), "esp_kv_pages_workspace")
        return self._workspace("pages", z.value, stream)

    def resize(self, lengths, stream=None) -> None:
        """Sets every sequence's length (int32 [sequences]): pages are freed and the lowest free ones taken."""
        with _on(stream, self.device) as s:
            w = self._pages_work(0, s)
            _check(lib().esp_kv_resize(self.ptr, _ints(lengths, self.sequences, "lengths", self.device), w.data_ptr(), w.numel(), s),
                   "esp_kv_resize")

    def fork(self, parents, children, stream=None) -> None:
        """children[i] drops its pages and continues parents[i] (int32 [n] each)."""
        n = parents.numel()
        with _on(stream, self.device) as s:
            w = self._pages_work(n, s)
            _check(lib().esp_kv_fork(self.ptr, n, _ints(parents, n, "parents", self.device), _ints(children, n, "children", self.device),
                                     w.data_ptr(), w.numel(), s), "esp_kv_fork")

    def compact(self, limit: Optional[int] = None, stream=None):
        """(table, refs, live) with no live page from `limit` on (None: from the number of live pages on).  The cache
        goes on with its old table, whose pages stay intact, until `install` is given the new one."""
        with _on(stream, self.device) as s:
            table, refs = torch.empty_like(self.table), torch.empty_like(self.refs)
            live = torch.empty((), dtype=torch.int32, device=self.device)
            w = self._pages_work(0, s)
            _check(lib().esp_kv_compact(self.ptr, -1 if limit is None else int(limit), table.data_ptr(), refs.data_ptr(), live.data_ptr(),
                                        w.data_ptr(), w.numel(), s), "esp_kv_compact")
        return table, refs, live

    def install(self, table, refs) -> None:
        """Takes the table and references of a compaction."""
        _ints(table, self.table.numel(), "table", self.device)
        _ints(refs, self.pages, "refs", self.device)
        if table.shape != self.table.shape:
            raise ValueError("table: the cache's shape expected")
        self.table, self.refs = table, refs
        self._describe()

    def device_status(self, stream=None) -> int:
        """The first error that the GPU recorded since the last call (waits for the stream)."""
        with _on(stream, self.device) as s:
            return int(lib().esp_kv_device_status(self.ptr, s))
