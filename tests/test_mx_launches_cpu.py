"""Which kernels the norm and the product launch, for which sizes, on a stand-in runtime: no GPU is needed."""
import pytest

from launches import Calls

from paper_2401_11240_amd import lora as L
from paper_2401_11240_amd import mx as MX


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    L.load()
    return Calls(tmp_path_factory.mktemp("launches"))


MOST = 1 << 22             # tiles of a launch


@pytest.mark.parametrize("fmt", [MX.LORA_E4M3, MX.LORA_E2M1])
@pytest.mark.parametrize("rows,h,h_out", [((1 << 28) + 64, 32, 8), (600000, 8192, 28672), (64, 64, 1 << 29), (1, 8, 1 << 30), (0x7fffffff, 32, 2048),
                                          (33, 64, 0x7ffffff8), (1 << 21, 32, 1 << 21)])
def test_products_of_more_tiles_than_a_launch_has(calls, rows, h, h_out, fmt):
    """Go to several launches, whose tiles cover y (the first number is of tiles of 64 x 64; one launch may do with larger ones)."""
    assert -(-rows // 64) * -(-h_out // 64) > MOST
    launched, need = calls.product(rows, h, h_out, fmt, L.LORA_BF16)
    assert need == 16 and len({ln.kernel for ln in launched}) == 1
    assert all(ln.kernel.startswith("lora_mx_tile_kernel<") and ln.grid[1:] == (1, 1) for ln in launched)
    tn, tt = (int(v) for v in launched[0].kernel.split("<")[1].split(",")[1:3])
    tiles = -(-rows // tt) * -(-h_out // tn)
    assert sum(ln.grid[0] for ln in launched) >= tiles and tiles / MOST <= len(launched) <= 4 * tiles / MOST + 1
    assert all(ln.grid[0] <= MOST + 8 for ln in launched)


@pytest.mark.parametrize("rows,h,h_out", [(1 << 21, 8, (1 << 21) + 8), (0x7fffffff, 8, 2056)])
def test_products_of_more_than_2_to_42_elements_are_refused(calls, rows, h, h_out):
    with pytest.raises(ValueError, match="2\\^42"):
        calls.product(rows, h, h_out, MX.LORA_E4M3, L.LORA_F16)
