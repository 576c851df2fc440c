"""Binding of the choice of the next tokens (include/lora_sample.h).

Marshalling only, with the C functions' names.  ``Params`` describes the rows' parameters
(device tensors) to the library and keeps them alive.
"""
from __future__ import annotations

import ctypes as C

from . import lora as _lora
from .mx import LORA_F32, _addr  # noqa: F401

EXPORTS = ("lora_sample_workspace_bytes", "lora_sample")


class _Params(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p)]


class Params:
    """Device tensors [n_rows], float32 (top_k int32), or None for 1, all, 1 and 0."""

    def __init__(self, temperature=None, top_k=None, top_p=None, min_p=None):
        n = {}
        for name, t in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p)):
            want = "torch.int32" if name == "top_k" else "torch.float32"
            if t is not None and (str(t.dtype) != want or t.dim() != 1 or not t.is_contiguous()):
                raise ValueError(f"{name}: a contiguous tensor of {want} and one dimension is needed")
            if t is not None:
                n[name] = int(t.shape[0])
        self.temperature, self.top_k, self.top_p, self.min_p = temperature, top_k, top_p, min_p
        self.n_rows = min(n.values()) if n else None        # rows that every tensor has
        self._c = _Params(_addr(temperature), _addr(top_k), _addr(top_p), _addr(min_p))
        self.c = C.byref(self._c)


_bound = None


def _lib():
    global _bound
    if _bound is not None:
        return _bound
    lib = _lora.load()
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    lib.lora_sample_workspace_bytes.argtypes = [i32, i32, i32, C.POINTER(sz)]
    lib.lora_sample.argtypes = [vp, i64, i32, i32, i32, C.POINTER(_Params), vp, vp, vp, vp, sz, vp]
    for name in EXPORTS:
        getattr(lib, name).restype = C.c_int
    _bound = lib
    return lib


_stream, _check = _lora._stream, _lora._check


def lora_sample_workspace_bytes(n_rows: int, n_vocab: int, dtype: int) -> int:
    out = C.c_size_t()
    _check(_lib().lora_sample_workspace_bytes(n_rows, n_vocab, dtype, C.byref(out)))
    return int(out.value)


def lora_sample(logits, ld: int, dtype: int, n_rows: int, n_vocab: int, params, u, tokens, probs, ws, ws_bytes: int,
                stream=None) -> None:
    if params is not None and params.n_rows is not None and params.n_rows < n_rows:
        raise ValueError(f"params: {params.n_rows} rows of {n_rows}")
    _check(_lib().lora_sample(_addr(logits), ld, dtype, n_rows, n_vocab, params.c if params is not None else None,
                              _addr(u), _addr(tokens), _addr(probs), _addr(ws), ws_bytes, _stream(stream)))
