"""The host code of the key-value cache and attention calls built with
AddressSanitizer and UndefinedBehaviorSanitizer, against a stand-in HIP runtime
(tests/sanitize/kv_calls.cpp).  CPU only: nothing is launched on a GPU (the device
code is compiled as usual and never run)."""
import os

import pytest


def test_kv_calls_on_a_stand_in_runtime(tmp_path):
    base = pytest.importorskip("test_host_sanitizers")     # its compiler lines and paths
    if not all(os.path.exists(c) for c in (base.HIPCC, base.CLANGXX)):
        pytest.skip("ROCm compilers missing")
    objs = [base.hip_object(os.path.join(base.CSRC, src), str(tmp_path / (src + ".o")))
            for src in ("lora_api.hip", "lora_kv.hip", "lora_attn.hip")]
    objs.append(base.hip_object(os.path.join(base.SAN, "kv_calls.cpp"), str(tmp_path / "kv_calls.o")))
    base.link_and_run(objs, str(tmp_path / "kv_calls"))
