"""The page book's calls with up to 2^31 - 1 sequences, their host code under the
sanitizers against a stand-in HIP runtime (tests/sanitize/kv_grids.cpp).  CPU only."""
import os

import pytest


def test_books_of_very_many_sequences(tmp_path):
    base = pytest.importorskip("test_host_sanitizers")     # its compiler lines and paths
    if not all(os.path.exists(c) for c in (base.HIPCC, base.CLANGXX)):
        pytest.skip("ROCm compilers missing")
    objs = [base.hip_object(os.path.join(base.CSRC, src), str(tmp_path / (src + ".o")))
            for src in ("lora_api.hip", "lora_kv.hip", "lora_attn.hip")]
    objs.append(base.hip_object(os.path.join(base.SAN, "kv_grids.cpp"), str(tmp_path / "kv_grids.o")))
    base.link_and_run(objs, str(tmp_path / "kv_grids"))
