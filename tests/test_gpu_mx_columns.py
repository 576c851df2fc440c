"""Rows that are columns of one buffer: a row's codes with its scales behind them, a norm's outputs beside its rows, against the
same calls on buffers of their own, bit for bit."""
import numpy as np
import pytest

import mx_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_mx import DEV, TYPE, apply, dtypes16, formats, random_rows, rows_of, stream  # noqa: E402

from paper_2401_11240_amd import mx as MX  # noqa: E402


def packed(n, h, fmt, gap=16):
    """Codes, scales and a gap in rows of one buffer."""
    c, s = MX.code_bytes(h, fmt), MX.scale_bytes(h)
    ld = (c + s + gap + 15) // 16 * 16
    buf = torch.full((n, ld), 0xAB, dtype=torch.uint8, device=DEV)
    return buf, MX.Rows(buf[:, :c], buf[:, c:c + s], fmt, h)


@formats
@pytest.mark.parametrize("rows,h", [(1, 264), (5, 264), (70, 1024), (300, 4104)])
def test_scales_behind_their_codes(rows, h, fmt):
    rng = np.random.default_rng([40, rows, h, fmt])
    x = torch.from_numpy(rng.standard_normal((rows, h))).to(DEV).half()
    n = R.blocks(h)
    buf, q = packed(rows, h, fmt)
    dense, w = rows_of(rows, h, fmt), random_rows(rng, 264, h, R.E2M1)
    y, want = torch.empty_like(x), torch.empty_like(x)
    for run in (lambda r: MX.lora_mx_quantize(x, h, R.F16, r, stream()),
                lambda r: MX.lora_norm(x, h, None, h, None, 1e-5, rows, h, R.F16, None, h, y, h, r, stream())):
        buf.fill_(0xAB)
        run(q)
        run(dense)
        assert torch.equal(q.codes, dense.codes) and torch.equal(q.scales[:, :n], dense.scales[:, :n])
        assert (buf[:, q.codes.shape[1] + n:] == 0xAB).all()
    MX.lora_mx_dequantize(q, y, h, R.F16, stream())
    MX.lora_mx_dequantize(dense, want, h, R.F16, stream())
    assert torch.equal(y, want)
    assert torch.equal(apply(q, w, R.F32), apply(dense, w, R.F32))
    wide, ws = packed(264, h, R.E2M1)
    ws.codes.copy_(w.codes)
    ws.scales.copy_(w.scales)
    assert torch.equal(apply(q, ws, R.F32), apply(dense, w, R.F32))


@dtypes16
@pytest.mark.parametrize("rows,h", [(1, 72), (7, 72), (1030, 512), (9, 4104)])
def test_a_norm_beside_its_rows(rows, h, dtype):
    """x, residual, total and y in four columns of one buffer."""
    rng = np.random.default_rng([41, rows, h, dtype])
    buf = torch.full((rows, 4 * h + 8), 7.0, dtype=TYPE[dtype], device=DEV)
    x, r, t, y = (buf[:, i * h:(i + 1) * h] for i in range(4))
    for m in (x, r):
        m.copy_(torch.from_numpy(rng.standard_normal((rows, h))).to(DEV))
    xs, rs = x.contiguous(), r.contiguous()
    ts, ys = torch.empty_like(xs), torch.empty_like(xs)
    ld = 4 * h + 8
    MX.lora_norm(x, ld, r, ld, None, 1e-5, rows, h, dtype, t, ld, y, ld, None, stream())
    MX.lora_norm(xs, h, rs, h, None, 1e-5, rows, h, dtype, ts, h, ys, h, None, stream())
    assert torch.equal(t, ts) and torch.equal(y, ys) and torch.equal(x, xs) and torch.equal(r, rs) and (buf[:, 4 * h:] == 7).all()


@formats
@pytest.mark.parametrize("rows,h", [(1, 8), (3, 40), (1, 4104), (70, 264), (260, 1064)])
def test_bytes_behind_the_last_scale_count_for_nothing(rows, h, fmt):
    """Scales that end with their last block: the rest of the word may hold anything."""
    rng = np.random.default_rng([42, rows, h, fmt])
    n, ld = R.blocks(h), MX.scale_bytes(h)
    x, w = random_rows(rng, rows, h, fmt), random_rows(rng, 264, h, R.E2M1)
    want = apply(x, w, R.F32)

    def ending(q, fill):
        flat = torch.full((q.n_rows * ld + 64,), fill, dtype=torch.uint8, device=DEV)
        s = flat.as_strided((q.n_rows, n), (ld, 1))
        s.copy_(q.scales[:, :n])
        return MX.Rows(q.codes, s, q.fmt, h)
    for fill in (0, 1, 127, 255):
        assert torch.equal(apply(ending(x, fill), ending(w, fill), R.F32), want)
