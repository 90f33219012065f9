"""Thin ctypes binding of the paged-cache calls of libstarkv.so.

Every function mirrors the C entry point of the same name in
include/starkv_paged.h; its arguments have the meaning documented there.
``Cache`` ties a pool's tensors to the C struct, once.  The binding checks
types, shapes and devices, so that a wrong Python call fails here rather than
inside a kernel, and launches on the cache's device and the given (or
current) stream.  All compute happens in the library's HIP kernels.
"""

from __future__ import annotations

import ctypes
from array import array
from ctypes import POINTER, c_int32, c_int64, c_size_t, c_void_p

import torch

from . import starkv as sk
from .starkv import KVLayout, StarKVError

MAX_SEQS = 256
MAX_DRAFT_WORDS = 4
MAX_TOKENS = 1 << 26
SEQ_OK, SEQ_NO_PAGES, SEQ_RANGE = 0, 1, 2


class Paged(ctypes.Structure):
    _fields_ = [("n_layers", c_int32), ("H", c_int32), ("G", c_int32), ("d", c_int32),
                ("dtype", c_int32), ("page_tokens", c_int32), ("n_pages", c_int32),
                ("n_slots", c_int32), ("max_pages", c_int32), ("reserved", c_int32),
                ("layer_stride", c_int64), ("page_stride", c_int64), ("group_stride", c_int64),
                ("token_stride", c_int64), ("k", c_void_p), ("v", c_void_p),
                ("table", c_void_p), ("len", c_void_p), ("refs", c_void_p)]


_P, _L = POINTER(Paged), POINTER(KVLayout)

# name -> (restype, argtypes)
SIGNATURES = {
    "starkv_pages_init": (c_int32, [_P, c_void_p]),
    "starkv_pages_workspace_bytes": (c_size_t, [_P, c_int32, c_int32]),
    "starkv_pages_grow": (c_int32, [_P, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_size_t,
                                    c_void_p]),
    "starkv_pages_write": (c_int32, [_P, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, _L,
                                     c_void_p]),
    "starkv_pages_write_grown": (c_int32, [_P, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, _L,
                                           c_void_p, c_void_p]),
    "starkv_pages_fork": (c_int32, [_P, c_void_p, c_void_p, c_int32, c_void_p]),
    "starkv_pages_free": (c_int32, [_P, c_void_p, c_int32, c_int32, c_int32, c_void_p]),
    "starkv_pages_compact": (c_int32, [_P, c_void_p, c_int32, c_void_p, c_void_p, c_int64, c_int32,
                                       c_void_p, c_int32, c_void_p, c_void_p, c_size_t,
                                       c_void_p]),
    "starkv_pages_compact_grown": (c_int32, [_P, c_void_p, c_int32, c_void_p, c_void_p, c_int64,
                                             c_int32, c_void_p, c_int32, c_void_p, c_void_p,
                                             c_void_p, c_size_t, c_void_p]),
    "starkv_attend_workspace_bytes": (c_size_t, [_P, c_void_p, c_int32, c_int32]),
    "starkv_attend_tree": (c_int32, [_P, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_int32,
                                     c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "starkv_attend_window": (c_int32, [_P, c_void_p, c_int32, c_void_p, c_void_p, c_int32, c_int32,
                                       c_int32, c_void_p, c_void_p, c_void_p, c_size_t,
                                       c_void_p]),
}

_lib = None


def lib():
    """The loaded library with the paged calls declared."""
    global _lib
    if _lib is None:
        L = sk.lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _tensor(t, dtype, what, device=None):
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{what}: {t.dtype}, {dtype} required")
    if device is not None and t.device != device:
        raise ValueError(f"{what} is on {t.device}, the cache on {device}")


class Cache:
    """A pool's tensors and the struct that every call takes.

    k, v:   [n_layers, n_pages, G, page_tokens, d], bfloat16 or float32, any
            strides (the same for both) with a unit last one
    table:  [n_slots, max_pages] int32;  length: [n_slots] int32;
    refs:   [n_pages] int32; all three contiguous
    H:      query heads
    """

    def __init__(self, k, v, table, length, refs, H: int):
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.stride(4) != 1:
            raise ValueError("k and v: [n_layers, n_pages, G, page_tokens, d] of the same strides, "
                             "the last one 1")
        if k.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"k: {k.dtype}, bfloat16 or float32 required")
        _tensor(k, k.dtype, "k")
        _tensor(v, k.dtype, "v", k.device)
        for t, n, what in ((table, 2, "table"), (length, 1, "length"), (refs, 1, "refs")):
            _tensor(t, torch.int32, what, k.device)
            if t.dim() != n or not t.is_contiguous():
                raise ValueError(f"{what} must be contiguous, of {n} dimension(s)")
        if length.shape[0] != table.shape[0] or refs.shape[0] != k.shape[1]:
            raise ValueError("length: one per row of table; refs: one per page")
        self.k, self.v, self.table, self.length, self.refs = k, v, table, length, refs
        self.device, self.dtype = k.device, k.dtype
        nl, n_pages, G, P, d = k.shape
        sl, sp, sg, st, _ = k.stride()
        self.n_layers, self.H, self.G, self.d, self.page_tokens = nl, H, G, d, P
        self.cap = table.shape[1] * P
        self.c = Paged(nl, H, G, d, sk.F32 if k.dtype == torch.float32 else sk.BF16, P, n_pages,
                       table.shape[0], table.shape[1], 0, sl, sp, sg, st, k.data_ptr(),
                       v.data_ptr(), table.data_ptr(), length.data_ptr(), refs.data_ptr())
        self.ref = ctypes.byref(self.c)

    def layers(self, first: int, count: int = 1) -> "Cache":
        """The same pages, `count` of the layers, to write and attend layer by
        layer.  (grow and compact take the whole cache: they copy rows of every
        layer that they are given, and change the one table.)"""
        k = self.k[first:first + count]
        if count < 1 or k.shape[0] != count:     # a slice of fewer would pass for the whole
            raise ValueError(f"layers [{first}, {first + count}) of {self.n_layers}")
        return Cache(k, self.v[first:first + count], self.table, self.length, self.refs, self.H)


def new_cache(n_layers: int, n_pages: int, page_tokens: int, G: int, d: int, n_slots: int,
              max_pages: int, H: int, dtype=torch.bfloat16, device="cuda") -> Cache:
    """A pool of its own tensors, made empty."""
    k = torch.empty(n_layers, n_pages, G, page_tokens, d, dtype=dtype, device=device)
    i32 = dict(dtype=torch.int32, device=device)
    c = Cache(k, torch.empty_like(k), torch.empty(n_slots, max_pages, **i32),
              torch.empty(n_slots, **i32), torch.empty(n_pages, **i32), H)
    pages_init(c)
    return c


def rows_layout(t) -> KVLayout:
    """Layout of new K or V rows shaped [n_layers, rows, G, d]."""
    if t.dim() != 4 or t.stride(3) != 1:
        raise ValueError("rows: [n_layers, rows, G, d] with a unit last stride")
    return KVLayout(t.stride(0), t.stride(2), t.stride(1))


# ------------------------------------------------------------------ marshalling

def _ints(x):
    """A host list as int32; _run passes its address."""
    return array("i", x)


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _run(name, cache, stream, *args):
    fn = getattr(_lib or lib(), name)
    index = cache.device.index
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(index)
    else:
        stream = getattr(stream, "cuda_stream", stream)
    at = [x.buffer_info()[0] if type(x) is array else x for x in args]   # args keeps the arrays
    if torch._C._cuda_getDevice() == index:
        code = fn(cache.ref, *at, stream)
    else:
        with torch.cuda.device(index):
            code = fn(cache.ref, *at, stream)
    if code != 0:
        raise StarKVError(name, code)


def _buffer(t, nbytes, what, device):
    """A workspace or output buffer of at least nbytes."""
    if t is None:
        if nbytes:
            raise ValueError(f"{what}: {nbytes} bytes required")
        return
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{what} must be a tensor on {device}")
    if not t.is_contiguous() or t.numel() * t.element_size() < nbytes:
        raise ValueError(f"{what}: {nbytes} contiguous bytes required")


def _bytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def _int32(t, n, what, device):
    _tensor(t, torch.int32, what, device)
    if not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{what}: {n} contiguous int32 required")


# ------------------------------------------------------------------ pages

def pages_init(cache: Cache, stream=None):
    _run("starkv_pages_init", cache, stream)


def pages_workspace_bytes(cache: Cache, n: int, most: int | None = None) -> int:
    """For n sequences, at most `most` tokens added or moved in each (default:
    what a table row holds)."""
    return int(lib().starkv_pages_workspace_bytes(cache.ref, n, cache.cap if most is None else most))


def pages_grow(cache: Cache, slots, add, status, ws, stream=None):
    n = len(slots)
    if len(add) != n:
        raise ValueError("add: one number per slot")
    _int32(status, n, "status", cache.device)
    _buffer(ws, 0, "ws", cache.device)
    _run("starkv_pages_grow", cache, stream, _ints(slots), n, _ints(add), _ptr(status), _ptr(ws),
         _bytes(ws))


def pages_write(cache: Cache, slots, rows, k, v, layout: KVLayout, stream=None, grown=None):
    """k, v: K and V of the sequences' new tokens, `layout` over (layer, group,
    row): rows_layout of a [n_layers, rows, G, d] tensor, or contiguous_layout
    of a compacted cache's [n_layers, G, rows, d].  grown: the status of the
    pages_grow of the same slots that made the tokens (starkv_pages_write_grown):
    a sequence that it left unchanged stays so."""
    n, tot = len(slots), sum(rows)
    if len(rows) != n:
        raise ValueError("rows: one number per slot")
    last = ((cache.n_layers - 1) * layout.layer_stride + (cache.G - 1) * layout.group_stride
            + (tot - 1) * layout.token_stride + cache.d)
    for t, what in ((k, "k"), (v, "v")):
        _tensor(t, cache.dtype, what, cache.device)
        have = t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
        if tot and have < last:
            raise ValueError(f"{what}: {have} elements < {last} required")
    args = (_ints(slots), n, _ints(rows), _ptr(k), _ptr(v), ctypes.byref(layout))
    if grown is None:
        _run("starkv_pages_write", cache, stream, *args)
    else:
        _int32(grown, n, "grown", cache.device)
        _run("starkv_pages_write_grown", cache, stream, *args, _ptr(grown))


def pages_fork(cache: Cache, src, dst, stream=None):
    if len(src) != len(dst):
        raise ValueError("src and dst: one slot each per fork")
    _run("starkv_pages_fork", cache, stream, _ints(src), _ints(dst), len(src))


def pages_free(cache: Cache, slots, keep_first: int = 0, keep_last: int = 0, stream=None):
    _run("starkv_pages_free", cache, stream, _ints(slots), len(slots), keep_first, keep_last)


def pages_compact(cache: Cache, slots, idx, status, ws, tail: int = 0, span=None, counts=None,
                  stream=None, grown=None):
    """idx: [n_layers, n, B] int32, or [1, n, B] where all layers keep the same
    tokens.  grown: as for pages_write (starkv_pages_compact_grown); it may be
    `status` itself."""
    n = len(slots)
    if idx.dim() != 3 or idx.shape[0] not in (1, cache.n_layers) or idx.shape[1] != n:
        raise ValueError(f"idx: [{cache.n_layers} or 1, {n}, B] required, got {tuple(idx.shape)}")
    _int32(idx, 0, "idx", cache.device)
    _int32(status, n, "status", cache.device)
    if counts is not None:
        _int32(counts, n, "counts", cache.device)
    if span is not None and len(span) != n:
        raise ValueError("span: one number per slot")
    B = idx.shape[2]
    _buffer(ws, 0, "ws", cache.device)
    args = (_ints(slots), n, _ints(span) if span is not None else None, _ptr(idx),
            n * B if idx.shape[0] > 1 else 0, B, _ptr(counts), tail)
    out = (_ptr(status), _ptr(ws), _bytes(ws))
    if grown is None:
        _run("starkv_pages_compact", cache, stream, *args, *out)
    else:
        _int32(grown, n, "grown", cache.device)
        _run("starkv_pages_compact_grown", cache, stream, *args, _ptr(grown), *out)


# ------------------------------------------------------------------ attention

def attend_workspace_bytes(cache: Cache, rows, max_len: int) -> int:
    rows = _ints(rows)
    return int(lib().starkv_attend_workspace_bytes(cache.ref, rows.buffer_info()[0], len(rows),
                                                   max_len))


def _attend_args(cache, slots, rows, q, out, lse, ws):
    n, tot = len(slots), sum(rows)
    if len(rows) != n:
        raise ValueError("rows: one number per slot")
    need = cache.n_layers * tot * cache.H * cache.d
    for t, what in ((q, "q"), (out, "out")):
        _tensor(t, cache.dtype, what, cache.device)
        if not t.is_contiguous() or t.numel() < need:
            raise ValueError(f"{what}: {need} contiguous elements required")
    if lse is not None:
        _tensor(lse, torch.float32, "lse", cache.device)
        if not lse.is_contiguous() or lse.numel() < need // cache.d:
            raise ValueError(f"lse: {need // cache.d} contiguous elements required")
    _buffer(ws, 0, "ws", cache.device)
    return n, tot


def attend_tree(cache: Cache, slots, rows, q, mask, out, ws, lse=None, max_len: int | None = None,
                stream=None):
    """mask: [sum(rows), words] int64 or uint64, bit j of a row's words for
    drafted token j."""
    n, tot = _attend_args(cache, slots, rows, q, out, lse, ws)
    if mask.dim() != 2 or mask.shape[0] < tot or not mask.is_contiguous():
        raise ValueError(f"mask: contiguous [{tot}, words] required")
    if mask.dtype != torch.int64:
        _tensor(mask, torch.uint64, "mask")
    _tensor(mask, mask.dtype, "mask", cache.device)
    _run("starkv_attend_tree", cache, stream, _ints(slots), n, _ints(rows), _ptr(q), _ptr(mask),
         mask.shape[1], cache.cap if max_len is None else max_len, _ptr(out), _ptr(lse), _ptr(ws),
         _bytes(ws))


def attend_window(cache: Cache, slots, rows, q, window: int, sinks: int, out, ws, lse=None,
                  max_len: int | None = None, stream=None):
    n, _ = _attend_args(cache, slots, rows, q, out, lse, ws)
    _run("starkv_attend_window", cache, stream, _ints(slots), n, _ints(rows), _ptr(q), window, sinks,
         cache.cap if max_len is None else max_len, _ptr(out), _ptr(lse), _ptr(ws), _bytes(ws))
