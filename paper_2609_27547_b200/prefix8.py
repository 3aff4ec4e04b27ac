"""8-bit prefix caches (``include/ebrl_prefix8.h``): ctypes binding, argument marshalling only.

A pool is a uint8 CUDA tensor [n_slots, record_bytes]; a record holds an environment's keys and values as e4m3 codes with
an fp32 scale for each block of 32 tokens and head, and one visibility bit per token.  Lengths, slots and numbers of tokens to keep
are host data (lists, numpy arrays or CPU tensors): the library checks them before anything is launched.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
import math
from typing import NamedTuple, Optional, Sequence, Union

import numpy as np
import torch

from .binding import BF16, F32, OK, EbrlError, lib

BLOCK = 32
_DTYPES = {torch.bfloat16: BF16, torch.float32: F32}


class _CLayout(C.Structure):
    _fields_ = [("kv_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("capacity", C.c_int32)]


class Layout(NamedTuple):
    """``ebrl_prefix8_layout_t``."""
    kv_layers: int
    n_kv_heads: int
    head_dim: int
    capacity: int

    @property
    def rows(self) -> int:
        return -(-self.capacity // BLOCK) * BLOCK

    @property
    def record_bytes(self) -> int:
        return _record(self)[1]


_lib = None


def _load():
    global _lib
    if _lib is None:
        L = lib()
        p, i, l, f, u = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint64
        L.ebrl_prefix8_record_bytes.restype = u
        L.ebrl_prefix8_record_bytes.argtypes = [p]
        L.ebrl_prefix8_last_error.restype = C.c_char_p
        L.ebrl_prefix8_quantize.argtypes = [p, p, i, i, p, p, p, p, l, i, p, i, p]
        L.ebrl_prefix8_attend_workspace.restype = u
        L.ebrl_prefix8_attend_workspace.argtypes = [p, i, p, i, i, i, i]
        L.ebrl_prefix8_attend.argtypes = [p, p, i, i, p, p, i, p, i, i, i, l, l, p, l, l, p, f, i, p, u, i, p]
        L.ebrl_prefix8_weigh.argtypes = [p, p, i, i, p, p, i, p, i, i, i, l, l, p, l, l, l, f, p, l, i, i, p]
        L.ebrl_prefix8_evict.argtypes = [p, p, p, i, i, p, p, p, i, i, p, l, p, l, p, l, i, p]
        _lib = L
    return _lib


@functools.lru_cache(maxsize=256)
def _record(layout: Layout):
    """(the C struct, its record's bytes, a reference that calls take): kept, because a layout is a plain value.  The reference holds the
    struct, so that a call in progress is not touched when other layouts push this one out."""
    c = _CLayout(*[int(v) for v in layout])
    at = C.byref(c)
    return c, int(_load().ebrl_prefix8_record_bytes(at)), at


def _check(st: int):
    if st != OK:
        raise EbrlError(st, (_load().ebrl_prefix8_last_error() or b"").decode())


def _host(v, what: str) -> torch.Tensor:
    """Host integers as a contiguous CPU int32 tensor."""
    if type(v) is torch.Tensor:
        if v.dtype is torch.int32 and not v.is_cuda and v.dim() == 1 and v.is_contiguous():
            return v
    else:
        v = torch.as_tensor(v)
        if v.numel() == 0:
            v = v.to(torch.int32)
    if v.device.type != "cpu" or v.dim() != 1 or v.is_floating_point():
        raise ValueError("%s must be a one-dimensional sequence of host integers" % what)
    if v.dtype != torch.int32:
        if v.numel() and (int(v.max()) > 2 ** 31 - 1 or int(v.min()) < -2 ** 31):
            raise ValueError("%s does not fit 32 bits" % what)
        v = v.to(torch.int32)
    return v.contiguous()


def _most(v: torch.Tensor) -> int:
    """The largest of host integers, 0 of none."""
    return max(v.tolist(), default=0) if v.numel() <= 64 else int(v.numpy().max())


def _pool(layout: Layout, pool: torch.Tensor, what: str = "pool"):
    rec = _record(layout)
    if rec[1] == 0:
        _load().ebrl_prefix8_record_bytes(rec[2])     # says why
        raise EbrlError(1, (_load().ebrl_prefix8_last_error() or b"").decode())
    if pool.device.type != "cuda" or pool.dtype != torch.uint8 or pool.dim() != 2 or pool.shape[1] != rec[1] or not pool.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA uint8 tensor [n_slots, %d]" % (what, rec[1]))
    return rec[2]


@contextlib.contextmanager
def _moved(to: int, back: int):
    torch.cuda.set_device(to)
    try:
        yield
    finally:
        torch.cuda.set_device(back)


_HERE = contextlib.nullcontext()


def _on(device: torch.device):
    """Makes a device current for the call (nothing when it already is)."""
    now = torch._C._cuda_getDevice()      # (there is a CUDA tensor: the runtime is up)
    return _HERE if now == device.index else _moved(device.index, now)


def _same_device(pool, *tensors):
    d = pool.device
    for t in tensors:
        if t is not None and t.device != d:
            raise ValueError("every tensor must be on the pool's device, %s" % pool.device)


def _stream(device: torch.device, stream: Optional[torch.cuda.Stream], *tensors) -> int:
    """The stream's handle; tensors handed to another stream than the current one are marked as used there."""
    now = torch._C._cuda_getCurrentRawStream(device.index)
    if stream is None or stream.cuda_stream == now:
        return now
    if stream.device != device:
        raise ValueError("the stream belongs to another device")
    here = torch.cuda.current_stream(device)
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
            t.record_stream(here)
    return stream.cuda_stream


def _elsewhere(device: torch.device, stream: Optional[torch.cuda.Stream]) -> bool:
    """Whether the call runs on another stream than the current one."""
    return stream is not None and stream.cuda_stream != torch._C._cuda_getCurrentRawStream(device.index)


def _n_slots(lens: torch.Tensor, slots, pool: torch.Tensor):
    s = None if slots is None else _host(slots, "slots")
    if s is not None and s.numel() != lens.numel():
        raise ValueError("%d slots for %d lengths" % (s.numel(), lens.numel()))
    return s, (None if s is None else s.data_ptr())


def layout_for(cfg) -> Layout:
    """The layout of the records that a handle created with ``cfg`` (kv_dtype E4M3) takes."""
    return Layout(max(cfg.kv_layers, 1), cfg.n_heads, cfg.d // cfg.n_heads, cfg.max_prefix_len)


def _addresses(base: int, step: int, n: int):
    """n addresses, `step` bytes apart, as a C array."""
    if n <= 16:
        return (C.c_void_p * n)(*[base + i * step for i in range(n)])
    return (C.c_void_p * n).from_buffer(np.arange(n, dtype=np.int64) * step + base)


def new_pool(layout: Layout, n_slots: int, device="cuda") -> torch.Tensor:
    """A zeroed pool of ``n_slots`` records."""
    if layout.record_bytes == 0:
        raise EbrlError(1, (_load().ebrl_prefix8_last_error() or b"").decode())
    return torch.zeros((int(n_slots), layout.record_bytes), dtype=torch.uint8, device=device)


def views(layout: Layout, pool: torch.Tensor):
    """(codes uint8 [n, kv_layers, 2, heads, rows, head_dim], scales fp32 [n, kv_layers, 2, heads, rows / 32], mask words
    int32 [n, rows / 32]): views of the pool, on any device."""
    rows, nb, heads = layout.rows, layout.rows // BLOCK, layout.kv_layers * 2 * layout.n_kv_heads
    nc, ns = heads * rows * layout.head_dim, heads * nb * 4
    return (pool[:, :nc].unflatten(1, (layout.kv_layers, 2, layout.n_kv_heads, rows, layout.head_dim)),
            pool[:, nc:nc + ns].view(torch.float32).unflatten(1, (layout.kv_layers, 2, layout.n_kv_heads, nb)),
            pool[:, nc + ns:nc + ns + nb * 4].view(torch.int32))


Planes = Union[torch.Tensor, Sequence[torch.Tensor]]


def quantize(layout: Layout, pool: torch.Tensor, planes: Planes, lens=None, *, slots=None, mask=None, sm_quota: int = 0,
             stream: Optional[torch.cuda.Stream] = None):
    """``ebrl_prefix8_quantize``: planes -> records.  ``planes``: one tensor [n, kv_layers, 2, P, heads * head_dim], or a sequence of
    tensors [kv_layers, 2, P_i, heads * head_dim] (bf16 or fp32; columns contiguous, planes a multiple of the row stride
    apart).  ``lens``: default each P.  ``mask``: uint8 or bool [n, >= P] or a sequence of tensors [>= P_i] / None; 0 hides a token."""
    cl = _pool(layout, pool)
    whole = torch.is_tensor(planes)
    views_ = [planes] if whole else list(planes)
    n = planes.shape[0] if whole else len(views_)
    if n == 0:
        return
    d = layout.n_kv_heads * layout.head_dim
    dt, rows = views_[0].dtype, []
    rs = next((x.stride(-2) for x in views_ if x.dim() >= 2 and x.shape[-2] > 1), d)   # (one row has no distance to the next)
    if dt not in _DTYPES:
        raise TypeError("planes must be bf16 or fp32, not %s" % dt)
    for x in views_:
        sh, sd = (x.shape[1:], x.stride()[1:]) if whole else (x.shape, x.stride())
        if len(sh) != 4 or sh[0] != layout.kv_layers or sh[1] != 2 or sh[3] != d:
            raise ValueError("planes must be [kv_layers, 2, P, %d], got %s" % (d, tuple(sh)))
        if x.dtype != dt:
            raise TypeError("planes must have one dtype")
        P = sh[2]
        if d > 1 and sd[3] != 1:
            raise ValueError("columns must be contiguous")
        r = sd[2] if P > 1 else rs
        plane = sd[1]     # the distance of the planes, in whole rows
        if r != rs or r < d or plane % rs or plane < P * rs or (layout.kv_layers > 1 and sd[0] != 2 * plane):
            raise ValueError("planes must share one row stride and lie a whole number of rows apart")
        rows.append(plane // rs)
    if whole:
        limit = [P]
        ptrs = _addresses(planes.data_ptr(), planes.stride(0) * planes.element_size(), n)
        rows = (C.c_int32 * n)(*rows * n) if n <= 16 else (C.c_int32 * n).from_buffer(np.full(n, rows[0], dtype=np.int32))
    else:
        limit = [x.shape[2] for x in views_]
        ptrs = (C.c_void_p * n)(*[x.data_ptr() for x in views_])
        rows = (C.c_int32 * n)(*rows)
    _same_device(pool, *views_)
    L = torch.full((n,), P, dtype=torch.int32) if lens is None and whole else _host(limit if lens is None else lens, "lens")
    if L.numel() != n:
        raise ValueError("%d lengths for %d environments" % (L.numel(), n))
    given, most = (None, _most(L)) if whole else (L.tolist(), 0)
    if most > limit[0] if whole else any(a > b for a, b in zip(given, limit)):
        raise ValueError("a length exceeds its planes")
    mp, masks = None, []
    if mask is not None:
        masks = list(mask) if not torch.is_tensor(mask) else [mask]
        if torch.is_tensor(mask):
            if mask.dim() != 2 or mask.shape[0] != n or mask.shape[1] < (most if whole else max(given)) or (mask.shape[1] > 1 and mask.stride(1) != 1):
                raise ValueError("mask must be [n, >= P] with contiguous rows")
            mp = _addresses(mask.data_ptr(), mask.stride(0), n)
        else:
            if len(masks) != n or any(m is not None and (m.dim() != 1 or m.numel() < k or (m.numel() > 1 and m.stride(0) != 1)) for m, k in zip(masks, given or L.tolist())):
                raise ValueError("masks must be n contiguous tensors [>= P_i] or None")
            mp = (C.c_void_p * n)(*[m.data_ptr() if m is not None else None for m in masks])
        if any(m is not None and m.dtype not in (torch.uint8, torch.bool) for m in masks):
            raise TypeError("masks must be uint8 or bool")
        _same_device(pool, *masks)
    s, sp = _n_slots(L, slots, pool)
    with _on(pool.device):
        st = _stream(pool.device, stream, pool, *views_, *masks)
        _check(_load().ebrl_prefix8_quantize(cl, pool.data_ptr(), pool.shape[0], n, sp, ptrs, L.data_ptr(),
                                             rows, rs, _DTYPES[dt], mp, int(sm_quota), st))


def _queries(layout: Layout, pool: torch.Tensor, q: torch.Tensor, lens, what: str = "q"):
    if q.dim() != 4 or q.shape[3] != layout.head_dim or q.shape[0] != lens.numel():
        raise ValueError("%s must be [n, H, heads, %d] with n = %d" % (what, layout.head_dim, lens.numel()))
    if q.dtype not in _DTYPES:
        raise TypeError("%s must be bf16 or fp32, not %s" % (what, q.dtype))
    if q.stride(3) != 1 or (q.shape[2] > 1 and q.stride(2) != layout.head_dim):
        raise ValueError("the heads of %s must be contiguous" % what)


def attend(layout: Layout, pool: torch.Tensor, q: torch.Tensor, lens, *, layer: int = 0, scale: Optional[float] = None, slots=None,
           out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, split_tokens: int = 0, sm_quota: int = 0,
           stream: Optional[torch.cuda.Stream] = None):
    """``ebrl_prefix8_attend``: (out, lse) of the queries q [n, H, heads, head_dim] (bf16 or fp32; out has its dtype) over the
    environments' visible tokens; lse fp32 [n, H, heads].  ``scale``: default 1 / sqrt(head_dim)."""
    cl = _pool(layout, pool)
    L = _host(lens, "lens")
    _queries(layout, pool, q, L)
    n, H, heads, hd = q.shape
    if out is not None:
        _queries(layout, pool, out, L, "out")
        if out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out must have the shape and dtype of q")
    if lse is not None and (lse.shape != q.shape[:3] or lse.dtype != torch.float32 or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous fp32 [n, H, heads]")
    _same_device(pool, q, out, lse)
    s, sp = _n_slots(L, slots, pool)
    dll = _load()
    with _on(pool.device):
        # (left to itself and without a quota the library cuts no prefix of 4096 tokens or fewer into pieces, under a quota none of 256)
        need = 0
        if split_tokens > 0 or (split_tokens == 0 and layout.capacity > (256 if sm_quota else 4096)):
            need = dll.ebrl_prefix8_attend_workspace(cl, n, L.data_ptr(), H, heads, split_tokens, sm_quota)
        # what is allocated here belongs to the stream that writes it; results are used on the current one, too
        with torch.cuda.stream(stream) if _elsewhere(pool.device, stream) else _HERE:
            if out is None:
                out = torch.empty_like(q) if q.is_contiguous() else q.new_empty((n, H, heads, hd))
            if lse is None:
                lse = q.new_empty((n, H, heads), dtype=torch.float32)
            ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
        st = _stream(pool.device, stream, pool, q, out, lse)
        if n and H and heads:
            _check(dll.ebrl_prefix8_attend(cl, pool.data_ptr(), pool.shape[0], n, sp, L.data_ptr(), int(layer), q.data_ptr(), _DTYPES[q.dtype],
                                           H, heads, q.stride(0), q.stride(1), out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(),
                                           1.0 / math.sqrt(hd) if scale is None else float(scale), int(split_tokens),
                                           ws.data_ptr() if need else None, need, int(sm_quota), st))
    return out, lse


def _weights(layout: Layout, pool: torch.Tensor, w: torch.Tensor, what: str):
    if w.dtype != torch.float32 or w.dim() != 2 or w.shape[0] != pool.shape[0] or w.shape[1] < layout.capacity or (w.shape[1] > 1 and w.stride(1) != 1):
        raise ValueError("%s must be fp32 [n_slots, >= capacity] with contiguous rows" % what)
    return w.stride(0) if w.shape[0] > 1 else max(w.stride(0), w.shape[1])


def weigh(layout: Layout, pool: torch.Tensor, q: torch.Tensor, lse: torch.Tensor, lens, weight: torch.Tensor, *, layer: int = 0,
          scale: Optional[float] = None, slots=None, accumulate: bool = True, sm_quota: int = 0,
          stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """``ebrl_prefix8_weigh``: adds to (or, ``accumulate=False``, writes) the row of each environment's slot in ``weight``
    (fp32 [n_slots, >= capacity]) the weight its tokens got from the queries; ``lse`` as ``attend`` returned it."""
    cl = _pool(layout, pool)
    L = _host(lens, "lens")
    _queries(layout, pool, q, L)
    n, H, heads, hd = q.shape
    if lse.shape != q.shape[:3] or lse.dtype != torch.float32:
        raise ValueError("lse must be fp32 [n, H, heads]")
    ws = _weights(layout, pool, weight, "weight")
    _same_device(pool, q, lse, weight)
    s, sp = _n_slots(L, slots, pool)
    with _on(pool.device):
        st = _stream(pool.device, stream, pool, q, lse, weight)
        if n:
            _check(_load().ebrl_prefix8_weigh(cl, pool.data_ptr(), pool.shape[0], n, sp, L.data_ptr(), int(layer), q.data_ptr(), _DTYPES[q.dtype],
                                              H, heads, q.stride(0), q.stride(1), lse.data_ptr(), *lse.stride(), 1.0 / math.sqrt(hd) if scale is None else float(scale),
                                              weight.data_ptr(), ws, 1 if accumulate else 0, int(sm_quota), st))
    return weight


def evict(layout: Layout, src: torch.Tensor, dst: torch.Tensor, weight: torch.Tensor, lens, keep, *, slots=None, protect_first: int = 0,
          protect_last: int = 0, weight_out: Optional[torch.Tensor] = None, kept: Optional[torch.Tensor] = None, sm_quota: int = 0,
          stream: Optional[torch.cuda.Stream] = None):
    """``ebrl_prefix8_evict``: keeps each environment's ``keep`` (an int or one per environment) heaviest tokens, in order, from
    ``src`` to ``dst`` (the same pool: in place).  Returns (new lengths as a CPU int32 tensor, kept old indices int32 [n, ...])."""
    cl = _pool(layout, src, "src")
    _pool(layout, dst, "dst")
    if dst.shape != src.shape:
        raise ValueError("src and dst must have the same slots")
    L = _host(lens, "lens")
    n = L.numel()
    K = torch.full((n,), int(keep), dtype=torch.int32) if isinstance(keep, int) else _host(keep, "keep")
    if K.numel() != n:
        raise ValueError("%d numbers to keep for %d environments" % (K.numel(), n))
    new = torch.minimum(L, K)
    most = _most(new)
    ws = _weights(layout, src, weight, "weight")
    wo = 0 if weight_out is None else _weights(layout, src, weight_out, "weight_out")
    if kept is None:
        with torch.cuda.stream(stream) if _elsewhere(src.device, stream) else _HERE:
            kept = torch.empty((n, max(1, most)), dtype=torch.int32, device=src.device)
    elif kept.dtype != torch.int32 or kept.dim() != 2 or kept.shape[0] != n or (kept.shape[1] > 1 and kept.stride(1) != 1) or \
            kept.shape[1] < most or (n > 1 and kept.stride(0) < kept.shape[1]):
        raise ValueError("kept must be int32 [n, >= the largest new length] with contiguous rows")
    _same_device(src, dst, weight, weight_out, kept)
    s, sp = _n_slots(L, slots, src)
    with _on(src.device):
        st = _stream(src.device, stream, src, dst, weight, weight_out, kept)
        if n:
            _check(_load().ebrl_prefix8_evict(cl, src.data_ptr(), dst.data_ptr(), src.shape[0], n, sp, L.data_ptr(), K.data_ptr(), int(protect_first),
                                              int(protect_last), weight.data_ptr(), ws, None if weight_out is None else weight_out.data_ptr(), wo,
                                              kept.data_ptr(), kept.stride(0) if n > 1 else kept.shape[1], int(sm_quota), st))
    return new, kept
