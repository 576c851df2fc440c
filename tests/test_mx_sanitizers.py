"""The host code of the calls on rows in blocks, of the norm and of the choice of tokens built with
AddressSanitizer and UndefinedBehaviorSanitizer, against a stand-in HIP runtime
(tests/sanitize/mx_calls.cpp).  CPU only: nothing is launched on a GPU (the device
code is compiled as usual and never run)."""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest


def test_mx_calls_on_a_stand_in_runtime(tmp_path):
    base = pytest.importorskip("test_host_sanitizers")     # its compiler lines and paths
    if not all(os.path.exists(c) for c in (base.HIPCC, base.CLANGXX)):
        pytest.skip("ROCm compilers missing")
    srcs = [os.path.join(base.CSRC, s + ".hip") for s in ("lora_api", "lora_kv", "lora_mx", "lora_mx_gemm", "lora_sample")]
    srcs.append(os.path.join(base.SAN, "mx_calls.cpp"))
    with ThreadPoolExecutor(4) as pool:
        objs = list(pool.map(lambda s: base.hip_object(s, str(tmp_path / (os.path.basename(s) + ".o"))), srcs))
    base.link_and_run(objs, str(tmp_path / "mx_calls"))
