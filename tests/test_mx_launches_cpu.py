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


COLUMNS = 1 << 48          # a buffer of 5 rows, 4096 bytes apart


def mx_rows(codes, scales, ld, n=5, h=256, fmt=MX.LORA_E4M3):
    return MX._Rows(COLUMNS + codes, COLUMNS + scales, ld, ld, n, h, fmt)


@pytest.mark.parametrize("codes,scales,meet", [(0, 256, False), (16, 272, False), (256, 248, False), (0, 252, True), (0, 4088, False),
                                               (0, 4092, True), (0, -8, False), (0, -4, True), (3840, 4096 - 256 - 8, False), (3856, 0, True),
                                               (4096, 256, False), (4096, 256 + 2 * 4096, False), (4096, 252 + 2 * 4096, True), (0, 0, True)])
def test_codes_and_scales_in_columns_of_one_buffer(calls, codes, scales, meet):
    """256 bytes of codes and 8 of scales a row: refused only where a row's bytes are another's."""
    q = mx_rows(codes + 4096, scales + 4096, 4096)

    def call():
        return calls._launched(calls.lib.lora_mx_quantize(9 << 48, 256, L.LORA_F16, q, None))
    if meet:
        with pytest.raises(ValueError, match="overlap"):
            call()
    else:
        assert len(call()) == 1


@pytest.mark.parametrize("rows,ldy,y,meet", [(5, 2048, 512, False), (5, 2048, 496, True), (5, 2048, 4096 - 512, False), (5, 2048, 4096 - 496, True),
                                             (5, 2048, 16384 + 512, False), (5, 2056, 512, True), (5, 256, 5 * 4096, False), (1, 256, 512, False),
                                             (1, 2048, 496, True), (1, 8, 512, False)])
def test_a_norm_beside_its_rows(calls, rows, ldy, y, meet):
    """Rows of 256 16-bit elements, 2048 apart: y in other columns, in rows of another distance, one row."""
    def call():
        return calls._launched(calls.lib.lora_norm(COLUMNS, 2048, None, 0, None, 1e-5, rows, 256, L.LORA_F16, None, 0, COLUMNS + y, max(ldy, 256), None, None))
    if meet:
        with pytest.raises(ValueError, match="overlap"):
            call()
    else:
        assert len(call()) == 1


def test_one_row_between_others(calls):
    """u, tokens and probs between two rows of logits."""
    launched = calls._launched(calls.lib.lora_sample(COLUMNS, 2048, L.LORA_F16, 5, 256, None, COLUMNS + 512, COLUMNS + 532, COLUMNS + 4096 - 20, 9 << 48, 16, None))
    assert len(launched) == 1
    for tokens, probs in ((COLUMNS + 508, COLUMNS + 600), (COLUMNS + 600, COLUMNS + 4096 - 16), (COLUMNS + 528, COLUMNS + 600), (COLUMNS + 600, COLUMNS + 612)):
        with pytest.raises(ValueError, match="overlap"):
            calls._launched(calls.lib.lora_sample(COLUMNS, 2048, L.LORA_F16, 5, 256, None, COLUMNS + 512, tokens, probs, 9 << 48, 16, None))


def test_every_kernel_is_reached(calls):
    """No form of the norm, the blocks, the product or the sampling kernels is compiled that no call launches."""
    reached = set()

    def take(launched):
        reached.update(ln.kernel for ln in launched)
    for dtype in (L.LORA_F16, L.LORA_BF16, MX.LORA_F32):
        for fmt in (MX.LORA_E4M3, MX.LORA_E2M1):
            for rows in (1, 1 << 18):
                q = calls._rows(0, rows, 1024, fmt)
                take(calls._launched(calls.lib.lora_mx_quantize(9 << 48, 1024, dtype, q, None)))
                take(calls._launched(calls.lib.lora_mx_dequantize(q, 9 << 48, 1024, dtype, None)))
            for rows in (1, 4, 5, 16, 17, 32, 33, 64, 128, 256, 512, 2048, 8437):
                for h in (64, 512, 4096, 8192):
                    for h_out in (64, 1024, 4104, 8192, 28672):
                        take(calls.product(rows, h, h_out, fmt, dtype)[0])
        if dtype != MX.LORA_F32:
            for rows in (1, 1023, 1024):
                for chunks in [2 ** i + d for i in range(14) for d in (0, 1)] + [767, 768, 769, 3 * 256, 8192]:
                    if chunks <= 8192:
                        take(calls.norm(rows, 8 * chunks, dtype))
        for rows, vocab in ((1, 100), (64, 128000)):
            take(calls._launched(calls.lib.lora_sample(1 << 48, vocab, dtype, rows, vocab, None, 2 << 48, 3 << 48, None, 4 << 48, 1 << 40, None)))
    mine = {k for k in calls.kernels() if k.startswith(("lora_norm", "lora_mx", "lora_sample"))}
    assert reached == mine, sorted(mine - reached)
