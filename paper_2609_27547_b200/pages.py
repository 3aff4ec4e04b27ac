"""Paged prefixes (``include/ebrl_pages.h``): ctypes binding, argument marshalling only.

A pool is a uint8 CUDA tensor [n_pages, page_bytes]; a page holds the keys and values of ``page_tokens`` consecutive tokens of a sequence
for all layers, and one visibility bit per token.  A table is a CUDA int32 tensor [n, width] that names the pages of a call's sequences
(-1: no page).  Lengths and numbers of tokens are host data (lists, numpy arrays or CPU tensors): the library checks them before anything is
launched.  ``Book`` keeps, on the host, which page belongs to whom.
"""
from __future__ import annotations

import array
import ctypes as C
import functools
import math
from typing import NamedTuple, Optional, Sequence

import numpy as np
import torch

from .binding import OK, EbrlError, lib
from .prefix8 import _DTYPES, _HERE, Planes, _addresses, _elsewhere, _most, _on, _same_device, _stream
from .prefix8 import _host as _host_any


class _CLayout(C.Structure):
    _fields_ = [("kv_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32), ("dtype", C.c_int32)]


class Layout(NamedTuple):
    """``ebrl_pages_layout_t``; ``dtype`` is torch.bfloat16 or torch.float32."""
    kv_layers: int
    n_kv_heads: int
    head_dim: int
    page_tokens: int
    dtype: torch.dtype = torch.bfloat16

    @property
    def page_bytes(self) -> int:
        return _page(self)[1]


def _int32(v, what: str) -> int:
    """A plain integer that a call takes in 32 bits (ctypes would drop the others)."""
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError("%s = %d does not fit 32 bits" % (what, v))
    return v


_lib = None


def _load():
    global _lib
    if _lib is None:
        L = lib()
        p, i, l, f, u = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint64
        L.ebrl_pages_page_bytes.restype = u
        L.ebrl_pages_page_bytes.argtypes = [p]
        L.ebrl_pages_last_error.restype = C.c_char_p
        L.ebrl_pages_test_drop_copies.argtypes = [u]
        L.ebrl_pages_test_drop_copies.restype = None
        L.ebrl_pages_append.argtypes = [p, p, i, i, p, l, p, p, i, p, l, p, l, p, i, p]
        L.ebrl_pages_attend_workspace.restype = u
        L.ebrl_pages_attend_workspace.argtypes = [p, i, p, p, i, i, i, i, i]
        L.ebrl_pages_attend.argtypes = [p, p, i, i, p, l, p, p, i, p, l, i, p, l, p, f, i, i, i, p, u, i, p]
        L.ebrl_pages_copy.argtypes = [p, p, i, p, i, i, p, p, p, i, p]
        L.ebrl_pages_gather.argtypes = [p, p, i, i, p, l, p, p, p, l, p, i, p]
        L.ebrl_pages_book_create.argtypes = [i, i, i, p]
        L.ebrl_pages_book_clone.argtypes = [p, p]
        L.ebrl_pages_book_destroy.argtypes = [p]
        L.ebrl_pages_book_destroy.restype = None
        L.ebrl_pages_book_extend.argtypes = [p, i, p, p, p, p, p, p]
        L.ebrl_pages_book_fork.argtypes = [p, i, p, p]
        L.ebrl_pages_book_shorten.argtypes = [p, i, p, p]
        L.ebrl_pages_book_compact.argtypes = [p, i, p, p, p, p]
        L.ebrl_pages_book_table.argtypes = [p, i, p, p, l]
        L.ebrl_pages_book_len.argtypes = [p, i]
        L.ebrl_pages_book_used.argtypes = [p]
        _lib = L
    return _lib


@functools.lru_cache(maxsize=256)
def _page(layout: Layout):
    """(the C struct, a page's bytes, a reference that calls take; it holds the struct): kept, because a layout is a plain value."""
    if layout.dtype not in _DTYPES:
        raise TypeError("pages hold bf16 or fp32, not %s" % (layout.dtype,))
    c = _CLayout(*[_int32(v, f) for v, f in zip(layout, Layout._fields[:4])], _DTYPES[layout.dtype])
    at = C.byref(c)
    return c, int(_load().ebrl_pages_page_bytes(at)), at


def _host(v, what: str) -> torch.Tensor:
    """Host integers as a contiguous CPU int32 tensor."""
    if type(v) in (list, tuple, range) and len(v):      # (an array takes plain integers ten times as fast as a tensor does)
        try:
            return torch.frombuffer(array.array("i", v), dtype=torch.int32)
        except (TypeError, OverflowError) as e:
            raise ValueError("%s must be host integers of 32 bits (%s)" % (what, e)) from None
    return _host_any(v, what)


def _sum(v: torch.Tensor) -> int:
    return sum(v.tolist()) if v.numel() <= 64 else int(v.numpy().sum(dtype=np.int64))


def _check(st: int):
    if st != OK:
        raise EbrlError(st, (_load().ebrl_pages_last_error() or b"").decode())


def _covered(layout: Layout):
    """The layout's page, or the error that says why there is none."""
    page = _page(layout)
    if page[1] == 0:
        _load().ebrl_pages_page_bytes(page[2])     # says why
        raise EbrlError(1, (_load().ebrl_pages_last_error() or b"").decode())
    return page


def _pool(layout: Layout, pool: torch.Tensor, what: str = "pool"):
    page = _covered(layout)
    if pool.device.type != "cuda" or pool.dtype != torch.uint8 or pool.dim() != 2 or pool.shape[1] != page[1] or not pool.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA uint8 tensor [n_pages, %d]" % (what, page[1]))
    return page[2]


def _table(table: torch.Tensor, n: int):
    """(address, stride, width) of a table for n sequences."""
    if table.dtype != torch.int32 or table.dim() != 2 or table.shape[0] != n or (table.shape[1] > 1 and table.stride(1) != 1) or \
            (n > 1 and table.stride(0) < table.shape[1]):
        raise ValueError("table must be int32 [%d, pages] with contiguous rows" % n)
    return table.data_ptr(), (table.stride(0) if n > 1 else table.shape[1])


def _fits(layout: Layout, table: torch.Tensor, lens: torch.Tensor) -> int:
    """The longest length."""
    most = _most(lens)
    if most > table.shape[1] * layout.page_tokens:
        raise ValueError("a length needs more pages than the table has")
    return most


def _packed(layout: Layout, x: torch.Tensor, heads: Optional[int], what: str):
    if x.dim() != 3 or x.shape[2] != layout.head_dim or (heads is not None and x.shape[1] != heads):
        raise ValueError("%s must be [tokens, %s, %d], got %s" % (what, "heads" if heads is None else heads, layout.head_dim, tuple(x.shape)))
    if x.dtype != layout.dtype:
        raise TypeError("%s must be %s, not %s" % (what, layout.dtype, x.dtype))
    if x.numel() and (x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != layout.head_dim)):
        raise ValueError("the heads of %s must be contiguous" % what)


def _counts(new, lens):
    N, L = _host(new, "new"), _host(lens, "lens")
    if N.numel() != L.numel():
        raise ValueError("%d counts for %d lengths" % (N.numel(), L.numel()))
    return N, L


def _rows32(rows):
    """The distances of planes, in rows, which a call takes in 32 bits."""
    if max(rows, default=0) >= 2 ** 31:
        raise ValueError("planes are 2^31 rows or more apart")
    return rows


def new_pool(layout: Layout, n_pages: int, device="cuda") -> torch.Tensor:
    """A zeroed pool of ``n_pages`` pages."""
    return torch.zeros((int(n_pages), _covered(layout)[1]), dtype=torch.uint8, device=device)


def views(layout: Layout, pool: torch.Tensor):
    """(elements [n_pages, kv_layers, 2, heads, page_tokens, head_dim], mask words int32 [n_pages, page_tokens / 32]): views of the pool, on
    any device."""
    shape = (layout.kv_layers, 2, layout.n_kv_heads, layout.page_tokens, layout.head_dim)
    nb = math.prod(shape) * layout.dtype.itemsize
    return pool[:, :nb].view(layout.dtype).unflatten(1, shape), pool[:, nb:nb + layout.page_tokens // 8].view(torch.int32)


def append(layout: Layout, pool: torch.Tensor, table: torch.Tensor, k: torch.Tensor, v: torch.Tensor, new, lens, *, layer: int = 0,
           mask: Optional[torch.Tensor] = None, sm_quota: int = 0, stream: Optional[torch.cuda.Stream] = None):
    """``ebrl_pages_append``: writes the keys and values k, v [sum(new), kv_heads, head_dim] of each sequence's ``new`` last tokens, of one layer;
    ``lens`` are the lengths with them.  ``mask``: uint8 or bool [sum(new)], 0 hides a token."""
    layer, sm_quota = _int32(layer, "layer"), _int32(sm_quota, "sm_quota")
    cl = _pool(layout, pool)
    N, L = _counts(new, lens)
    n, total = N.numel(), _sum(N)
    _packed(layout, k, layout.n_kv_heads, "k")
    _packed(layout, v, layout.n_kv_heads, "v")
    if k.shape[0] < total or v.shape[0] < total:
        raise ValueError("%d new tokens, but k and v have %d and %d" % (total, k.shape[0], v.shape[0]))
    if mask is not None and (mask.dtype not in (torch.uint8, torch.bool) or mask.dim() != 1 or mask.numel() < total or (mask.numel() > 1 and mask.stride(0) != 1)):
        raise ValueError("mask must be contiguous uint8 or bool [>= %d]" % total)
    at, stride = _table(table, n)
    _fits(layout, table, L)
    _same_device(pool, table, k, v, mask)
    with _on(pool.device):
        st = _stream(pool.device, stream, pool, table, k, v, mask)
        if n:
            _check(_load().ebrl_pages_append(cl, pool.data_ptr(), pool.shape[0], n, at, stride, N.data_ptr(), L.data_ptr(), layer, k.data_ptr(), k.stride(0),
                                             v.data_ptr(), v.stride(0), None if mask is None else mask.data_ptr(), sm_quota, st))


def attend(layout: Layout, pool: torch.Tensor, table: torch.Tensor, q: torch.Tensor, new, lens, *, layer: int = 0, causal: bool = True, window: int = 0,
           scale: Optional[float] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, split_tokens: int = 0, sm_quota: int = 0,
           stream: Optional[torch.cuda.Stream] = None):
    """``ebrl_pages_attend``: (out, lse) of the queries q [>= sum(new), heads, head_dim], ``new`` of each sequence, over the sequences; lse fp32
    [.., heads].  ``scale``: default 1 / sqrt(head_dim).  Rows behind the last query are left as they were (zeros where ``out`` is made here)."""
    layer, window, split_tokens, sm_quota = _int32(layer, "layer"), _int32(window, "window"), _int32(split_tokens, "split_tokens"), _int32(sm_quota, "sm_quota")
    cl = _pool(layout, pool)
    N, L = _counts(new, lens)
    n, total = N.numel(), _sum(N)
    _packed(layout, q, None, "q")
    rows, heads, hd = q.shape
    if rows < total:
        raise ValueError("%d queries, but q has %d rows" % (total, rows))
    if out is not None:
        _packed(layout, out, heads, "out")
        if out.shape[0] < total:
            raise ValueError("out has %d rows for %d queries" % (out.shape[0], total))
    if lse is not None and (lse.dim() != 2 or lse.shape[0] < total or lse.shape[1] != heads or lse.dtype != torch.float32 or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous fp32 [>= %d, %d]" % (total, heads))
    at, stride = _table(table, n)
    most = _fits(layout, table, L)
    _same_device(pool, table, q, out, lse)
    dll = _load()
    with _on(pool.device):
        need = 0
        if total and (split_tokens > 0 or (split_tokens == 0 and most >= 512)):   # (left to itself the library cuts no shorter sequence)
            need = dll.ebrl_pages_attend_workspace(cl, n, N.data_ptr(), L.data_ptr(), heads, 1 if causal else 0, window, split_tokens, sm_quota)
        # what is allocated here belongs to the stream that writes it; results are used on the current one, too
        with torch.cuda.stream(stream) if _elsewhere(pool.device, stream) else _HERE:
            make = q.new_empty if rows == total else q.new_zeros
            if out is None:
                out = make((rows, heads, hd))
            if lse is None:
                lse = make((rows, heads), dtype=torch.float32)
            ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        st = _stream(pool.device, stream, pool, table, q, out, lse)
        if n and heads:
            _check(dll.ebrl_pages_attend(cl, pool.data_ptr(), pool.shape[0], n, at, stride, N.data_ptr(), L.data_ptr(), layer, q.data_ptr(), q.stride(0), heads,
                                         out.data_ptr(), out.stride(0), lse.data_ptr(), 1.0 / math.sqrt(hd) if scale is None else float(scale),
                                         1 if causal else 0, window, split_tokens, ws.data_ptr() if need else None, need, sm_quota, st))
    return out, lse


def copy(layout: Layout, src: torch.Tensor, dst: torch.Tensor, moves, *, sm_quota: int = 0, stream: Optional[torch.cuda.Stream] = None):
    """``ebrl_pages_copy``: pages of ``src`` to pages of ``dst`` (the same pool, or one that does not overlap it).  ``moves``: (from, to, tokens) as
    ``Book`` returns them, or (from, to); host data."""
    sm_quota = _int32(sm_quota, "sm_quota")
    cl = _pool(layout, src, "src")
    _pool(layout, dst, "dst")
    parts = [_host(m, "moves") for m in moves]
    if len(parts) not in (2, 3) or any(p.numel() != parts[0].numel() for p in parts):
        raise ValueError("moves must be (from, to) or (from, to, tokens), all of one length")
    _same_device(src, dst)
    n = parts[0].numel()
    with _on(src.device):
        st = _stream(src.device, stream, src, dst)
        if n:
            _check(_load().ebrl_pages_copy(cl, src.data_ptr(), src.shape[0], dst.data_ptr(), dst.shape[0], n, parts[0].data_ptr(), parts[1].data_ptr(),
                                           parts[2].data_ptr() if len(parts) == 3 else None, sm_quota, st))


def gather(layout: Layout, pool: torch.Tensor, table: torch.Tensor, lens, planes: Optional[Planes] = None, *, mask=None, sm_quota: int = 0,
           stream: Optional[torch.cuda.Stream] = None) -> Planes:
    """``ebrl_pages_gather``: sequences -> planes, the form that ``ActGen.submit`` and ``prefix8.quantize`` take.  ``planes``: one tensor [n,
    kv_layers, 2, P, heads * head_dim], or a sequence of tensors [kv_layers, 2, P_i, ..] (columns contiguous, planes a multiple of the row stride apart); default:
    new ones [kv_layers, 2, lens[i], ..].  ``mask``: uint8 [n, >= P] or a sequence of uint8 tensors / None: gets each token's visibility."""
    sm_quota = _int32(sm_quota, "sm_quota")
    cl = _pool(layout, pool)
    L = _host(lens, "lens")
    n, d = L.numel(), layout.n_kv_heads * layout.head_dim
    at, stride = _table(table, n)
    _fits(layout, table, L)
    given = L.tolist()
    if any(k < 0 for k in given):
        raise ValueError("a length is negative")
    with _on(pool.device):
        if planes is None:
            with torch.cuda.stream(stream) if _elsewhere(pool.device, stream) else _HERE:
                planes = [torch.empty((layout.kv_layers, 2, k, d), dtype=layout.dtype, device=pool.device) for k in given]
        views_ = [planes] if torch.is_tensor(planes) else list(planes)
        whole = torch.is_tensor(planes)
        if (planes.shape[0] if whole else len(views_)) != n:
            raise ValueError("planes for %d sequences are needed" % n)
        rows, rs = [], next((x.stride(-2) for x in views_ if x.dim() >= 2 and x.shape[-2] > 1), d)   # (one row has no distance to the next)
        for i, x in enumerate(views_):
            sh, sd = (x.shape[1:], x.stride()[1:]) if whole else (x.shape, x.stride())
            if x.dtype != layout.dtype:
                raise TypeError("planes must be %s, not %s" % (layout.dtype, x.dtype))
            if len(sh) != 4 or sh[0] != layout.kv_layers or sh[1] != 2 or sh[3] != d:
                raise ValueError("planes must be [%d, 2, P, %d], got %s" % (layout.kv_layers, d, tuple(sh)))
            if sh[2] < (_most(L) if whole else given[i]):
                raise ValueError("a length exceeds its planes")
            r, plane = sd[2] if sh[2] > 1 else rs, sd[1]
            if x.numel() and ((d > 1 and sd[3] != 1) or r != rs or r < d or plane % rs or plane < sh[2] * rs or (layout.kv_layers > 1 and sd[0] != 2 * plane)):
                raise ValueError("columns must be contiguous, planes share one row stride and lie a whole number of rows apart")
            rows.append(plane // rs)
        _rows32(rows)
        if whole and n > 1 and planes.numel() and planes.stride(0) < (layout.kv_layers * 2 - 1) * planes.stride(2) + (planes.shape[3] - 1) * rs + d:
            raise ValueError("the planes of the sequences overlap")
        if whole:
            ptrs = _addresses(planes.data_ptr(), planes.stride(0) * planes.element_size(), n)
            rows = (C.c_int32 * n).from_buffer(np.full(n, rows[0] if rows else 0, dtype=np.int32)) if n else None
        else:
            ptrs, rows = (C.c_void_p * n)(*[x.data_ptr() for x in views_]), (C.c_int32 * n)(*rows)
        mp, masks = None, []
        if mask is not None:
            masks = [mask] if torch.is_tensor(mask) else list(mask)
            if torch.is_tensor(mask):
                if mask.dim() != 2 or mask.shape[0] != n or mask.shape[1] < _most(L) or (mask.shape[1] > 1 and mask.stride(1) != 1) or (n > 1 and mask.stride(0) < mask.shape[1]):
                    raise ValueError("mask must be [n, >= P] with contiguous rows")
                mp = _addresses(mask.data_ptr(), mask.stride(0), n)
            else:
                if len(masks) != n or any(m is not None and (m.dim() != 1 or m.numel() < k or (m.numel() > 1 and m.stride(0) != 1)) for m, k in zip(masks, given)):
                    raise ValueError("masks must be n contiguous tensors [>= P_i] or None")
                mp = (C.c_void_p * n)(*[m.data_ptr() if m is not None else None for m in masks])
            if any(m is not None and m.dtype not in (torch.uint8, torch.bool) for m in masks):
                raise TypeError("masks must be uint8 or bool")
        _same_device(pool, table, *views_, *masks)
        st = _stream(pool.device, stream, pool, table, *views_, *masks)
        if n:
            _check(_load().ebrl_pages_gather(cl, pool.data_ptr(), pool.shape[0], n, at, stride, L.data_ptr(), ptrs, rows, rs, mp, sm_quota, st))
    return planes


def check(device=None):
    """``ebrl_pages_check``: waits for the device and raises if a kernel's bounded wait ran out on it since the last call."""
    with torch.cuda.device(device):
        _check(_load().ebrl_pages_check())


class Book:
    """``ebrl_pages_book_*``: which page belongs to which of ``max_sequences`` sequences.  ``extend`` and ``compact`` return moves
    (from, to, tokens) that ``copy`` has to make before anything that relies on them."""

    def __init__(self, n_pages: int, page_tokens: int, max_sequences: int, *, _of: Optional["Book"] = None):
        self._L, self._b = _load(), C.c_void_p()
        self.n_pages, self.page_tokens, self.max_sequences = _int32(n_pages, "n_pages"), _int32(page_tokens, "page_tokens"), _int32(max_sequences, "max_sequences")
        _check(self._L.ebrl_pages_book_clone(_of._b, C.byref(self._b)) if _of is not None else
               self._L.ebrl_pages_book_create(self.n_pages, self.page_tokens, self.max_sequences, C.byref(self._b)))

    def clone(self) -> "Book":
        return Book(self.n_pages, self.page_tokens, self.max_sequences, _of=self)

    def _call(self, fn, seqs, values, what):
        s, v = _host(seqs, "seqs"), _host(values, what)
        if s.numel() != v.numel():
            raise ValueError("%d sequences, %d %s" % (s.numel(), v.numel(), what))
        return s, v, fn

    def _moves(self, room: int):
        return torch.empty((3, max(1, room)), dtype=torch.int32), C.c_int32(0)

    def extend(self, seqs: Sequence[int], lens: Sequence[int]):
        s, v, fn = self._call(self._L.ebrl_pages_book_extend, seqs, lens, "lens")
        m, k = self._moves(s.numel())
        _check(fn(self._b, s.numel(), s.data_ptr(), v.data_ptr(), m[0].data_ptr(), m[1].data_ptr(), m[2].data_ptr(), C.byref(k)))
        return m[0, :k.value], m[1, :k.value], m[2, :k.value]

    def fork(self, seqs: Sequence[int], to: Sequence[int]):
        s, v, fn = self._call(self._L.ebrl_pages_book_fork, seqs, to, "targets")
        _check(fn(self._b, s.numel(), s.data_ptr(), v.data_ptr()))

    def shorten(self, seqs: Sequence[int], lens):
        """``lens``: an int or one per sequence; 0 frees them."""
        s = _host(seqs, "seqs")
        s, v, fn = self._call(self._L.ebrl_pages_book_shorten, s, [lens] * s.numel() if isinstance(lens, int) else lens, "lens")
        _check(fn(self._b, s.numel(), s.data_ptr(), v.data_ptr()))

    def compact(self, most: Optional[int] = None):
        room = min(self.used, self.n_pages - self.used)      # (there are no more moves than that)
        if most is not None:
            room = max(-1, min(room, int(most)))
        m, k = self._moves(max(0, room))
        _check(self._L.ebrl_pages_book_compact(self._b, room, m[0].data_ptr(), m[1].data_ptr(), m[2].data_ptr(), C.byref(k)))
        return m[0, :k.value], m[1, :k.value], m[2, :k.value]

    def table(self, seqs: Sequence[int], width: Optional[int] = None, device="cpu") -> torch.Tensor:
        """int32 [n, width] (default: as many columns as the longest of them needs)."""
        s = _host(seqs, "seqs")
        if width is None:
            width = max((-(-self.len(i) // self.page_tokens) for i in s.tolist()), default=0)
        out = torch.empty((s.numel(), int(width)), dtype=torch.int32, pin_memory=torch.device(device).type == "cuda")
        _check(self._L.ebrl_pages_book_table(self._b, s.numel(), s.data_ptr(), out.data_ptr(), int(width)))
        return out.to(device, non_blocking=True)

    def len(self, seq: int) -> int:
        seq = int(seq)
        return int(self._L.ebrl_pages_book_len(self._b, seq if 0 <= seq < 2 ** 31 else -1))

    @property
    def used(self) -> int:
        """Pages in use, each counted once."""
        return int(self._L.ebrl_pages_book_used(self._b))

    def __del__(self):
        b, self._b = getattr(self, "_b", None), None
        if b:
            self._L.ebrl_pages_book_destroy(b)
