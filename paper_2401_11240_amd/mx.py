"""Binding of rows in blocks, the norm and the product (include/lora_mx.h).

Marshalling only, with the C functions' names.  ``Rows`` describes torch tensors of codes and
scales to the library and keeps them alive; the calls take device buffers and streams as the
rest of the package does.  Rows, and tensors beside them, that are not on one GPU, and workspaces given as
tensors that are too short or on another device, are refused before anything is enqueued (``ValueError``).
"""
from __future__ import annotations

import ctypes as C

from . import lora as _lora

LORA_F32 = 2
LORA_E4M3 = 0
LORA_E2M1 = 1

EXPORTS = ("lora_norm", "lora_mx_quantize", "lora_mx_dequantize", "lora_mx_workspace_bytes", "lora_mx_apply")


class _Rows(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("ld_codes", C.c_int64), ("ld_scales", C.c_int64),
                ("n_rows", C.c_int32), ("h", C.c_int32), ("format", C.c_int32)]


def code_bytes(h: int, fmt: int) -> int:
    """Bytes of a row's codes."""
    return -(-h // 32) * (32 if fmt == LORA_E4M3 else 16)


def scale_bytes(h: int) -> int:
    """Bytes from one row's scales to the next's, where they are as near as they may be."""
    return -(-h // 128) * 4


class Rows:
    """Rows of h elements in blocks: uint8 device tensors codes [n_rows, at least
    ``code_bytes``] and scales [n_rows, at least a byte for each block], dense in the last
    dimension.  (The product reads the last row's scales to the end of a 4-byte word: torch's own
    allocations have it, memory of another origin must.)"""

    def __init__(self, codes, scales, fmt: int, h: int):
        for name, t in (("codes", codes), ("scales", scales)):
            if str(t.dtype) != "torch.uint8" or t.dim() != 2 or (t.numel() and t.stride(1) != 1):
                raise ValueError(f"{name}: a uint8 tensor of 2 dimensions, dense in the last, is needed")
        if codes.shape[0] != scales.shape[0] or codes.device != scales.device:
            raise ValueError("codes and scales must have the same rows, on one device")
        if codes.shape[1] < code_bytes(h, fmt) or scales.shape[1] < -(-h // 32):
            raise ValueError(f"a row of {h} elements takes {code_bytes(h, fmt)} bytes and {-(-h // 32)} scales, not "
                             f"{codes.shape[1]} and {scales.shape[1]}")
        self.codes, self.scales, self.fmt, self.h, self.device = codes, scales, fmt, h, codes.device
        self.gpu = codes.get_device() if codes.is_cuda else -1
        self.n_rows = int(codes.shape[0])
        # (torch gives the stride of a single row any value)
        ldc, lds = ((codes.stride(0), scales.stride(0)) if self.n_rows > 1 else
                    (code_bytes(h, fmt), scale_bytes(h)))
        self._c = _Rows(codes.data_ptr(), scales.data_ptr(), ldc, lds, self.n_rows, h, fmt)
        self.c = C.byref(self._c)


def empty_rows(n_rows: int, h: int, fmt: int, device) -> Rows:
    """Rows to be written."""
    import torch
    return Rows(torch.empty((n_rows, code_bytes(h, fmt)), dtype=torch.uint8, device=device),
                torch.empty((n_rows, scale_bytes(h)), dtype=torch.uint8, device=device), fmt, h)


_bound = None


def _lib():
    global _bound
    if _bound is not None:
        return _bound
    lib = _lora.load()
    vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
    rows = C.POINTER(_Rows)
    sig = {
        "lora_norm": [vp, i64, vp, i64, vp, f32, i32, i32, i32, vp, i64, vp, i64, rows, vp],
        "lora_mx_quantize": [vp, i64, i32, rows, vp],
        "lora_mx_dequantize": [rows, vp, i64, i32, vp],
        "lora_mx_workspace_bytes": [rows, rows, C.POINTER(sz)],
        "lora_mx_apply": [rows, rows, vp, i64, i32, vp, sz, vp],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = C.c_int
    _bound = lib
    return lib


_stream, _check = _lora._stream, _lora._check


def _addr(p) -> int:
    try:                                   # (a call of a few rows costs the host what this costs it)
        return p.data_ptr()
    except AttributeError:
        return 0 if p is None else int(p)


def _at(gpu: int, names: str, *tensors) -> list:
    """The addresses of tensors on that GPU (or those that are given), in one call: each costs the host what a
    launch of few rows is about to wait for."""
    out = []
    for t in tensors:
        if t is None:
            out.append(None)
            continue
        try:
            p = t.data_ptr()
        except AttributeError:
            out.append(int(t))
            continue
        if t.get_device() != gpu or gpu < 0:
            raise ValueError(f"{names.split()[len(out)]} is on {t.device}: a tensor on cuda:{max(gpu, 0)} is needed")
        out.append(p)
    return out


def _on_gpu(*rows: Rows) -> None:
    gpu = rows[0].gpu
    for r in rows:
        if r.gpu != gpu or gpu < 0:
            raise ValueError(f"rows in blocks on {rows[0].device} and {r.device}: device tensors of one GPU are needed")


def _space(t, n: int, device) -> int:
    """The address of a workspace of at least n bytes."""
    try:
        p = t.data_ptr()
    except AttributeError:
        return 0 if t is None else int(t)
    if t.numel() * t.element_size() < n or (device is not None and t.device != device) or not t.is_contiguous():
        raise ValueError(f"ws: a contiguous tensor of {n} bytes or more on {device} is needed")
    return p


def lora_norm(x, ldx: int, residual, ldr: int, weight, eps: float, n_rows: int, h: int, dtype: int, total, ldt: int,
              y, ldy: int, q: Rows = None, stream=None) -> None:
    if q is not None:
        _on_gpu(q)
        gpu = q.gpu
    else:                                  # (outputs are never all missing: one of them says where)
        on = next((t for t in (y, total, x, weight, residual) if hasattr(t, "get_device")), None)
        gpu = -1 if on is None else on.get_device()
    px, pr, pw, pt, py = _at(gpu, "x residual weight total y", x, residual, weight, total, y)
    _check(_lib().lora_norm(px, ldx, pr, ldr, pw, eps, n_rows, h, dtype, pt, ldt, py, ldy, None if q is None else q.c,
                            _stream(stream)))


def lora_mx_quantize(x, ldx: int, dtype: int, q: Rows, stream=None) -> None:
    _on_gpu(q)
    _check(_lib().lora_mx_quantize(_at(q.gpu, "x", x)[0], ldx, dtype, q.c, _stream(stream)))


def lora_mx_dequantize(q: Rows, y, ldy: int, dtype: int, stream=None) -> None:
    _on_gpu(q)
    _check(_lib().lora_mx_dequantize(q.c, _at(q.gpu, "y", y)[0], ldy, dtype, _stream(stream)))


def lora_mx_workspace_bytes(x: Rows, w: Rows) -> int:
    out = C.c_size_t()
    _check(_lib().lora_mx_workspace_bytes(x.c, w.c, C.byref(out)))
    return int(out.value)


def lora_mx_apply(x: Rows, w: Rows, y, ldy: int, dtype: int, ws, ws_bytes: int, stream=None) -> None:
    _on_gpu(x, w)
    _check(_lib().lora_mx_apply(x.c, w.c, _at(x.gpu, "y", y)[0], ldy, dtype, _space(ws, ws_bytes, x.device), ws_bytes, _stream(stream)))
