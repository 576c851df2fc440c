"""How often the norm's outputs are not the exact values rounded once: 16-bit rows and 8-bit codes against 64 bits.

The norm's one error beyond its outputs' rounding that counts here is that of the mean square.  Squares of eight neighbours are
summed in float32, the h / 8 sums in binary64.  A rounding to float32 is off by 2^-24 / sqrt(3) of its result in the root mean
square, at most, so eight of them by sqrt(8 / 3) 2^-24 of the sum.  The errors of the h / 8 sums are independent, and the spread of
sums of eight squares of normal values makes them sqrt(1 + 2 / 8) larger than of equal ones: the mean is off by
1.83 2^-24 / sqrt(h / 8), its root by half of that.  With h = 4096 that is SIGMA = 2.4e-9 of y in the root mean square, 0.8 SIGMA in
the mean magnitude.

A value is rounded to the wrong side of a border between two where the border lies within that error.  `per_octave` borders to a
factor of two are per_octave / ln 2 to a factor of e, so 0.8 SIGMA n per_octave / ln 2 of n values are expected to be off (a row
has one error for all of its values, but there are thousands of rows).  Four times that and three more are allowed.  Were y a
float32 value rounded again, one of 2^13 (16-bit floats) or 2^16 (bfloat16) would end half way and half of those go the wrong way:
1024 and 128 where 195 and 27 are allowed."""
import math

import numpy as np
import pytest

import mx_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_mx import DEV, TYPE, dtypes16, rows_of, stream  # noqa: E402

from paper_2401_11240_amd import mx as MX  # noqa: E402

ROWS, H = 4096, 4096
EPS = float(np.float32(1e-5))


SIGMA = 0.5 * math.sqrt(8 / 3) * math.sqrt(1 + 2 / 8) * 2.0 ** -24 / math.sqrt(H / 8)


def limit(n, per_octave):
    return 4 * 0.8 * SIGMA * n * per_octave / math.log(2) + 3


def normed(dtype, seed):
    """x, weight, the kernel's y and blocks, and the exact y in float64."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((ROWS, H), generator=gen, device=DEV).to(TYPE[dtype])
    g = (1 + 0.2 * torch.randn(H, generator=gen, device=DEV)).to(TYPE[dtype])
    y, q = torch.empty_like(x), rows_of(ROWS, H, R.E4M3)
    MX.lora_norm(x, H, None, H, g, EPS, ROWS, H, dtype, None, H, y, H, q, stream())
    s = x.double()
    return y, q, s * g.double() / (s.square().mean(1, keepdim=True) + EPS).sqrt()


def rounded(v, dtype):
    """float64 values, not zero, rounded once to 16 bits: ties to even."""
    unit = torch.exp2(torch.floor(torch.log2(v.abs())) - (10 if dtype == R.F16 else 7))
    if dtype == R.F16:
        unit = unit.clamp(min=2.0 ** -24)
    return torch.round(v / unit) * unit


@dtypes16
def test_16_bit_rows_are_the_exact_values_rounded_once(dtype):
    y, _, exact = normed(dtype, 70)
    some = exact.abs() > 2.0 ** -20
    off = y[some].double() != rounded(exact[some], dtype)
    assert int(off.sum()) <= limit(ROWS * H, 1024 if dtype == R.F16 else 128)


@dtypes16
def test_values_that_float32_puts_half_way(dtype):
    """Of the exact values those that float32 rounds to half way between two 16-bit values, from below and from above, by more
    than a quarter of a step of float32: six times SIGMA at its largest there (SIGMA 2^25 = 0.081 half steps)."""
    assert 6 * SIGMA * 2 ** 25 < 0.5
    y, _, exact = normed(dtype, 71)
    low = 1 << (12 if dtype == R.F16 else 15)
    f = exact.float()
    half_way = ((f.view(torch.int32) & (2 * low - 1)) == low) & (exact.abs() > 2.0 ** -13)
    rest = ((exact - f.double()) / torch.exp2(torch.floor(torch.log2(exact.abs().clamp(min=2.0 ** -30))) - 24))   # in half steps
    for side in (half_way & (rest > 0.5), half_way & (rest < -0.5)):
        assert int(side.sum()) > (300 if dtype == R.F16 else 30)
        assert torch.equal(y[side].double(), rounded(exact[side], dtype))


@dtypes16
def test_8_bit_codes_are_those_of_the_exact_values(dtype):
    _, q, exact = normed(dtype, 72)
    codes, scales, e = q.codes.cpu().numpy(), q.scales.cpu().numpy(), exact.cpu().numpy()
    off = 0
    for r in range(0, ROWS, 512):
        want, s = R.quantize(e[r:r + 512], R.E4M3)
        assert np.array_equal(scales[r:r + 512, :s.shape[1]], s)
        off += int((codes[r:r + 512] != want).sum())
    assert off <= limit(ROWS * H, 8)
