"""Binding of the choice of the next tokens (include/lora_sample.h).

Marshalling only, with the C functions' names.  ``Params`` describes the rows' parameters
(device tensors) to the library and keeps them alive.  Arrays and workspaces that are given as
tensors are checked for type, length and device before anything is enqueued (``ValueError``).
"""
from __future__ import annotations

import ctypes as C

from . import lora as _lora
from .mx import LORA_F32, _addr, _at, _space  # noqa: F401

EXPORTS = ("lora_sample_workspace_bytes", "lora_sample")


class _Params(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p)]


class Params:
    """Device tensors [n_rows], float32 (top_k int32), or None for 1, all, 1 and 0."""

    def __init__(self, temperature=None, top_k=None, top_p=None, min_p=None):
        n, on = {}, set()
        for name, t in (("temperature", temperature), ("top_k", top_k), ("top_p", top_p), ("min_p", min_p)):
            want = "torch.int32" if name == "top_k" else "torch.float32"
            if t is not None and (str(t.dtype) != want or t.dim() != 1 or not t.is_contiguous()):
                raise ValueError(f"{name}: a contiguous tensor of {want} and one dimension is needed")
            if t is not None:
                n[name] = int(t.shape[0])
                on.add(t.device)
        if len(on) > 1:
            raise ValueError(f"the parameters are on {sorted(map(str, on))}: one device is needed")
        self.device = on.pop() if on else None
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


def _array(name: str, t, n: int, dtype: str, device) -> int:
    """The address of an array of at least n entries."""
    try:
        p = t.data_ptr()
    except AttributeError:
        return 0 if t is None else int(t)
    if str(t.dtype) != dtype or t.numel() < n or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor of {n} or more on {device} is needed, not {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return p


def lora_sample_workspace_bytes(n_rows: int, n_vocab: int, dtype: int) -> int:
    out = C.c_size_t()
    _check(_lib().lora_sample_workspace_bytes(n_rows, n_vocab, dtype, C.byref(out)))
    return int(out.value)


def lora_sample(logits, ld: int, dtype: int, n_rows: int, n_vocab: int, params, u, tokens, probs, ws, ws_bytes: int,
                stream=None) -> None:
    if params is not None and params.n_rows is not None and params.n_rows < n_rows:
        raise ValueError(f"params: {params.n_rows} rows of {n_rows}")
    on = next((t.device for t in (tokens, u, logits, probs, ws, params) if getattr(t, "device", None) is not None), None)
    if on is not None and on.type != "cuda":
        raise ValueError(f"tensors on {on}: device tensors are needed")
    if params is not None and params.device is not None and on != params.device:
        raise ValueError(f"the parameters are on {params.device}, the rows on {on}")
    _check(_lib().lora_sample(_at(-1 if on is None else on.index, "logits", logits)[0], ld, dtype, n_rows, n_vocab, params.c if params is not None else None,
                              _array("u", u, n_rows, "torch.float32", on), _array("tokens", tokens, n_rows, "torch.int32", on),
                              _array("probs", probs, n_rows, "torch.float32", on), _space(ws, ws_bytes, on), ws_bytes,
                              _stream(stream)))
