"""Binding of the paged key-value cache and its attention (include/lora_kv.h).

Marshalling only, with the C functions' names.  ``Cache``, ``Seqs`` and ``Book``
describe torch tensors to the library and keep them alive; the calls take
device buffers and streams as the rest of the package does.  int32 arrays and
workspaces that are given as tensors are checked for type, length and device before
anything is enqueued (``ValueError``).
"""
from __future__ import annotations

import ctypes as C

import numpy as np

from . import lora as _lora

EXPORTS = ("lora_kv_append", "lora_attn_create", "lora_attn_destroy", "lora_attn_decode", "lora_attn_prompt",
           "lora_kv_workspace_bytes", "lora_kv_grow", "lora_kv_grow_step", "lora_kv_fork", "lora_kv_fork_step",
           "lora_kv_free", "lora_kv_trim", "lora_kv_copy", "lora_kv_compact")


class _Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p),
                ("layer_stride", C.c_int64), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("row_stride", C.c_int64),
                ("dtype", C.c_int32), ("n_layers", C.c_int32), ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32),
                ("page_rows", C.c_int32), ("head_dim", C.c_int32)]


class _Seqs(C.Structure):
    _fields_ = [("tables", C.c_void_p), ("lens", C.c_void_p), ("n_seqs", C.c_int32), ("ld_table", C.c_int32),
                ("max_len", C.c_int32)]


class _Book(C.Structure):
    _fields_ = [("tables", C.c_void_p), ("lens", C.c_void_p), ("refs", C.c_void_p), ("n_seqs", C.c_int32),
                ("ld_table", C.c_int32), ("n_pages", C.c_int32), ("page_rows", C.c_int32)]


def _int32(t, dims, name):
    if str(t.dtype) != "torch.int32" or t.dim() != dims or (t.numel() and t.stride(-1) != 1):
        raise ValueError(f"{name}: an int32 tensor of {dims} dimension(s), dense in the last, is needed")
    return t


def _gpu(t) -> int:
    return t.get_device() if t.is_cuda else -1


def _table(t, lens):
    _int32(t, 2, "tables")
    _int32(lens, 1, "lens")
    if lens.shape[0] != t.shape[0] or not t.is_contiguous():
        raise ValueError("tables must be contiguous, [n_seqs, ld], with one length per row")
    if t.device != lens.device:
        raise ValueError("tables and lens must be on one device")


class Cache:
    """Keys and values of every layer: 16-bit tensors [n_layers, n_pages,
    n_kv_heads, page_rows, head_dim] of equal strides, dense in the last."""

    def __init__(self, k, v):
        if k.dim() != 5 or k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v: two tensors [n_layers, n_pages, n_kv_heads, page_rows, head_dim] of one type")
        if k.numel() and (k.stride() != v.stride() or k.stride(4) != 1):
            raise ValueError("k and v need equal strides and a dense last dimension")
        if k.device != v.device:
            raise ValueError("k and v must be on one device")
        dtype = {"torch.float16": _lora.LORA_F16, "torch.bfloat16": _lora.LORA_BF16}.get(str(k.dtype))
        if dtype is None:
            raise ValueError("k and v must be float16 or bfloat16")
        self.k, self.v, self.device, self.gpu = k, v, k.device, _gpu(k)
        n = [int(x) for x in k.shape]
        self._c = _Cache(k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1), k.stride(2), k.stride(3), dtype,
                         n[0], n[1], n[2], n[3], n[4])
        self.c = C.byref(self._c)


class Seqs:
    """The sequences of a step: int32 device tensors tables [n_seqs, ld] and
    lens [n_seqs]; ``max_len`` bounds every length the launches read."""

    def __init__(self, tables, lens, max_len: int):
        _table(tables, lens)
        self.tables, self.lens, self.device, self.gpu = tables, lens, lens.device, _gpu(lens)
        self.n_seqs = int(lens.shape[0])
        self._c = _Seqs(tables.data_ptr(), lens.data_ptr(), self.n_seqs, int(tables.shape[1]), int(max_len))
        self.c = C.byref(self._c)


class Book:
    """Tables, lengths and reference counts (int32 device tensors)."""

    def __init__(self, tables, lens, refs, page_rows: int):
        _table(tables, lens)
        _int32(refs, 1, "refs")
        if refs.device != lens.device:
            raise ValueError("refs and lens must be on one device")
        self.tables, self.lens, self.refs, self.device, self.gpu = tables, lens, refs, lens.device, _gpu(lens)
        self.n_seqs = int(lens.shape[0])
        self._c = _Book(tables.data_ptr(), lens.data_ptr(), refs.data_ptr(), self.n_seqs, int(tables.shape[1]),
                        int(refs.shape[0]), int(page_rows))
        self.c = C.byref(self._c)


_bound = None


def _lib():
    global _bound
    if _bound is not None:
        return _bound
    lib = _lora.load()
    vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    cache, seqs, book = C.POINTER(_Cache), C.POINTER(_Seqs), C.POINTER(_Book)
    i32p = C.POINTER(i32)
    sig = {
        "lora_kv_append": [cache, i32, seqs, vp, i32, vp, i64, vp, i64, vp],
        "lora_attn_create": [C.POINTER(vp), C.c_int, vp],
        "lora_attn_destroy": [vp],
        "lora_attn_decode": [vp, cache, i32, seqs, i32, vp, i64, vp, i64, f32, i32, i32, vp],
        "lora_attn_prompt": [vp, cache, i32, seqs, vp, i32, i32, vp, i64, vp, i64, f32, i32, i32, vp],
        "lora_kv_workspace_bytes": [book, C.POINTER(sz)],
        "lora_kv_grow": [book, vp, vp, vp, sz, vp],
        "lora_kv_grow_step": [book, vp, i32, vp, vp, vp, sz, vp],
        "lora_kv_fork": [cache, book, i32, i32p, i32p, vp, vp, sz, vp],
        "lora_kv_fork_step": [cache, book, i32, i32p, i32p, vp, vp, vp, sz, vp],
        "lora_kv_free": [book, i32, i32p, vp],
        "lora_kv_trim": [book, i32, i32, vp],
        "lora_kv_copy": [cache, i32, i32p, i32p, vp],
        "lora_kv_compact": [cache, book, vp, vp, vp, vp, sz, vp],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = C.c_int
    _bound = lib
    return lib


_stream = _lora._stream
_check = _lora._check


def _addr(p) -> int:
    try:                                   # (a call of a few rows costs the host what this costs it)
        return p.data_ptr()
    except AttributeError:
        return 0 if p is None else int(p)


def _words(name: str, t, n: int, of) -> int:
    """The address of an int32 array of at least n entries on the device of ``of``'s."""
    if t is None:
        return 0
    try:
        p = t.data_ptr()
    except AttributeError:
        return int(t)
    if t.dtype != of.lens.dtype or t.numel() < n or t.device != of.device or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous int32 tensor of {n} or more on {of.device} is needed, not {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return p


def _space(t, n: int, of) -> int:
    """The address of a workspace of at least n bytes."""
    p = _addr(t)
    if hasattr(t, "data_ptr") and (t.numel() * t.element_size() < n or t.device != of.device or not t.is_contiguous()):
        raise ValueError(f"ws: a contiguous tensor of {n} bytes or more on {of.device} is needed")
    return p


def _on_gpu(of) -> None:
    if of.gpu < 0:
        raise ValueError(f"tables and lens are on {of.device}: device tensors are needed")


def _together(cache: Cache, of) -> None:
    if cache.gpu != of.gpu or of.gpu < 0:
        _on_gpu(of)
        raise ValueError(f"the cache is on {cache.device}, the sequences on {of.device}")


def _ids(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(C.c_int32))


def lora_kv_append(cache: Cache, layer: int, seqs: Seqs, seg_offset, n_rows: int, k_new, ldk: int, v_new, ldv: int,
                   stream=None) -> None:
    """``seg_offset`` None: one row per sequence."""
    _together(cache, seqs)
    off = 0 if seg_offset is None else _words("seg_offset", seg_offset, seqs.n_seqs + 1, seqs)
    _check(_lib().lora_kv_append(cache.c, layer, seqs.c, off, n_rows, _addr(k_new), ldk, _addr(v_new),
                                 ldv, _stream(stream)))


def lora_attn_create(device: int, stream=None) -> int:
    out = C.c_void_p()
    _check(_lib().lora_attn_create(C.byref(out), device, _stream(stream)))
    return int(out.value or 0)


def lora_attn_destroy(attn: int) -> None:
    _check(_lib().lora_attn_destroy(attn))


def lora_attn_decode(attn: int, cache: Cache, layer: int, seqs: Seqs, n_heads: int, q, ldq: int, out, ldo: int,
                     scale: float, window: int = 0, n_sinks: int = 0, stream=None) -> None:
    _together(cache, seqs)
    _check(_lib().lora_attn_decode(attn, cache.c, layer, seqs.c, n_heads, _addr(q), ldq, _addr(out), ldo, scale,
                                   window, n_sinks, _stream(stream)))


def lora_attn_prompt(attn: int, cache: Cache, layer: int, seqs: Seqs, seg_offset, n_rows: int, n_heads: int, q,
                     ldq: int, out, ldo: int, scale: float, window: int = 0, n_sinks: int = 0, stream=None) -> None:
    _together(cache, seqs)
    off = _words("seg_offset", seg_offset, seqs.n_seqs + 1, seqs)
    _check(_lib().lora_attn_prompt(attn, cache.c, layer, seqs.c, off, n_rows, n_heads, _addr(q), ldq,
                                   _addr(out), ldo, scale, window, n_sinks, _stream(stream)))


def lora_kv_workspace_bytes(book: Book) -> int:
    out = C.c_size_t()
    _check(_lib().lora_kv_workspace_bytes(book.c, C.byref(out)))
    return int(out.value)


def lora_kv_grow(book: Book, add, info, ws, ws_bytes: int, stream=None) -> None:
    _on_gpu(book)
    _check(_lib().lora_kv_grow(book.c, _words("add", add, book.n_seqs, book), _words("info", info, 2, book),
                               _space(ws, ws_bytes, book), ws_bytes, _stream(stream)))


def lora_kv_grow_step(book: Book, add, max_len: int, step_lens, info, ws, ws_bytes: int, stream=None) -> None:
    """Grow, with the lengths that the step's calls use (``Seqs``) in ``step_lens``."""
    _on_gpu(book)
    n = book.n_seqs
    _check(_lib().lora_kv_grow_step(book.c, _words("add", add, n, book), max_len,
                                    _words("step_lens", step_lens, n, book), _words("info", info, 2, book),
                                    _space(ws, ws_bytes, book), ws_bytes, _stream(stream)))


def _pairs(parents, children):
    p, pp = _ids(parents)
    c, cp = _ids(children)
    if p.size != c.size:
        raise ValueError("parents and children differ in number")
    return p, pp, c, cp


def lora_kv_fork(cache: Cache, book: Book, parents, children, info, ws, ws_bytes: int, stream=None) -> None:
    _together(cache, book)
    p, pp, c, cp = _pairs(parents, children)
    _check(_lib().lora_kv_fork(cache.c, book.c, p.size, pp, cp, _words("info", info, 2, book),
                               _space(ws, ws_bytes, book), ws_bytes, _stream(stream)))


def lora_kv_fork_step(cache: Cache, book: Book, parents, children, step_lens, info, ws, ws_bytes: int,
                      stream=None) -> None:
    _together(cache, book)
    p, pp, c, cp = _pairs(parents, children)
    _check(_lib().lora_kv_fork_step(cache.c, book.c, p.size, pp, cp,
                                    _words("step_lens", step_lens, book.n_seqs, book), _words("info", info, 2, book),
                                    _space(ws, ws_bytes, book), ws_bytes, _stream(stream)))


def lora_kv_free(book: Book, seqs, stream=None) -> None:
    _on_gpu(book)
    s, sp = _ids(seqs)
    _check(_lib().lora_kv_free(book.c, s.size, sp, _stream(stream)))


def lora_kv_trim(book: Book, window: int, n_sinks: int = 0, stream=None) -> None:
    _on_gpu(book)
    _check(_lib().lora_kv_trim(book.c, window, n_sinks, _stream(stream)))


def lora_kv_copy(cache: Cache, src, dst, stream=None) -> None:
    if cache.gpu < 0:
        raise ValueError(f"the cache is on {cache.device}: device tensors are needed")
    s, sp = _ids(src)
    d, dp = _ids(dst)
    if s.size != d.size:
        raise ValueError("src and dst differ in number")
    _check(_lib().lora_kv_copy(cache.c, s.size, sp, dp, _stream(stream)))


def lora_kv_compact(cache: Cache, book: Book, tables_out, refs_out, info, ws, ws_bytes: int, stream=None) -> None:
    _together(cache, book)
    _check(_lib().lora_kv_compact(cache.c, book.c, _words("tables_out", tables_out, book.tables.numel(), book),
                                  _words("refs_out", refs_out, book.refs.numel(), book), _words("info", info, 2, book),
                                  _space(ws, ws_bytes, book), ws_bytes, _stream(stream)))
