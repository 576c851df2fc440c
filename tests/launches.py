"""Which kernels a call launches, without a GPU: the library's host code against a stand-in runtime
(tests/sanitize/launches.cpp) that writes launches down and runs none."""
import ctypes as C
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor
from typing import NamedTuple

import pytest

from paper_2401_11240_amd import build as B
from paper_2401_11240_amd import mx as MX
from paper_2401_11240_amd import sample as SA

SOURCES = ("lora_api", "lora_kv", "lora_mx", "lora_mx_gemm", "lora_sample")
CLANGXX = "/opt/rocm/llvm/bin/clang++"
GB = 1 << 30


class Launch(NamedTuple):
    kernel: str            # with its template arguments
    grid: tuple
    threads: int


def build(folder) -> C.CDLL:
    """The host code and the stand-in as a library in `folder`."""
    if not all(os.path.exists(c) for c in (B.hipcc(), CLANGXX)):
        pytest.skip("ROCm compilers missing")
    here = os.path.dirname(os.path.abspath(__file__))
    srcs = [os.path.join(B.CSRC, s + ".hip") for s in SOURCES] + [os.path.join(here, "sanitize", "launches.cpp")]

    def compiled(src):
        out = os.path.join(folder, os.path.basename(src) + ".o")
        res = subprocess.run([B.hipcc(), "-x", "hip", f"--offload-arch={B.ARCH}", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-c",
                              f"-I{B.INCLUDE}", f"-I{B.CSRC}", src, "-o", out], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-4000:]
        return out

    with ThreadPoolExecutor(4) as pool:
        objs = list(pool.map(compiled, srcs))
    # (the device code, which is not there)
    names = subprocess.run(["nm", "-u"] + objs, capture_output=True, text=True, check=True).stdout.split()
    absent = [f"-Wl,--defsym={n}=0" for n in sorted(set(names)) if n.startswith("__hip_fatbin")]
    lib = os.path.join(folder, "launches.so")
    res = subprocess.run([CLANGXX, "-shared", "-Wl,-Bsymbolic", "-L/opt/rocm/lib", "-Wl,-rpath,/opt/rocm/lib"] + objs + absent +
                         ["-lamdhip64", "-o", lib], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    lib = C.CDLL(lib)
    for bound in (MX, SA):                 # (the signatures are the library's)
        real = bound._lib()
        for name in bound.EXPORTS:
            getattr(lib, name).argtypes = getattr(real, name).argtypes
    lib.lora_last_error.restype = lib.launches_log.restype = lib.launches_kernels.restype = C.c_char_p
    return lib


class Calls:
    """Calls on made-up addresses: the launches of each."""

    def __init__(self, folder):
        self.lib = build(str(folder))

    def kernels(self):
        return set(self.lib.launches_kernels().decode().splitlines())

    def _launched(self, rc):
        lines = [ln.split("\t") for ln in self.lib.launches_log().decode().splitlines()]
        assert rc == 0 or not lines
        if rc:
            raise ValueError(f"{rc}: {self.lib.lora_last_error().decode()}")
        return [Launch(n, (int(x), int(y), int(z)), int(t)) for n, x, y, z, t in lines]

    @staticmethod
    def _rows(at, n, h, fmt):
        return MX._Rows((2 * at + 1) << 48, (2 * at + 2) << 48, MX.code_bytes(h, fmt), MX.scale_bytes(h), n, h, fmt)

    def product(self, rows, h, h_out, fmt, dtype):
        """(launches, workspace bytes)"""
        x, w, need = self._rows(0, rows, h, fmt), self._rows(1, h_out, h, MX.LORA_E2M1), C.c_size_t()
        self._launched(self.lib.lora_mx_workspace_bytes(C.byref(x), C.byref(w), C.byref(need)))
        return self._launched(self.lib.lora_mx_apply(C.byref(x), C.byref(w), 9 << 48, h_out, dtype, 13 << 48, need.value, None)), need.value

    def norm(self, rows, h, dtype):
        return self._launched(self.lib.lora_norm(1 << 48, h, None, h, None, 1e-5, rows, h, dtype, None, h, 2 << 48, h, None, None))
