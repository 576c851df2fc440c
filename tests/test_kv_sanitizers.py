"""The host code of the key-value cache and attention calls built with
AddressSanitizer and UndefinedBehaviorSanitizer, against a stand-in HIP runtime
(tests/sanitize/kv_calls.cpp).  CPU only: nothing is launched on a GPU (the device
code is compiled as usual and never run)."""
import os

from test_host_sanitizers import CSRC, SAN, hip_object, link_and_run, pytestmark  # noqa: F401


def test_kv_calls_on_a_stand_in_runtime(tmp_path):
    objs = [hip_object(os.path.join(CSRC, src), str(tmp_path / (src + ".o")))
            for src in ("lora_api.hip", "lora_kv.hip", "lora_attn.hip")]
    objs.append(hip_object(os.path.join(SAN, "kv_calls.cpp"), str(tmp_path / "kv_calls.o")))
    link_and_run(objs, str(tmp_path / "kv_calls"))
