"""lora_sample beside addresses: parameters and workspaces on the host are refused before anything is enqueued."""
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2401_11240_amd import build as B  # noqa: E402
from paper_2401_11240_amd import lora as L  # noqa: E402
from paper_2401_11240_amd import sample as SA  # noqa: E402

GB = 1 << 30


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(B.lib_path()):
        B.build()
    L.load()


@pytest.mark.parametrize("which", ["temperature", "top_k", "top_p", "min_p", "ws"])
def test_host_tensors_beside_addresses(which):
    """(The logits, u, the tokens and probs as addresses, which say nothing of a device.)"""
    params, ws = None, 5 * GB
    if which == "ws":
        ws = torch.zeros(64, dtype=torch.uint8)
    else:
        params = SA.Params(**{which: torch.ones(3, dtype=torch.int32 if which == "top_k" else torch.float32)})
    with pytest.raises(ValueError):
        SA.lora_sample(GB, 64, L.LORA_F16, 3, 64, params, 2 * GB, 3 * GB, 4 * GB, ws, 64)
