"""Every form of the product (mx_forms.py) against its definition in 64 bits, computed by the GPU's float64 product of the stored
values, and on whole numbers whose sums are exact."""
import numpy as np
import pytest

import mx_reference as R
from mx_forms import FORMS

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_mx import DEV, FLOOR, HALF, apply, rows_of  # noqa: E402

BYTES = torch.arange(256, device=DEV)


def table(fmt):
    """The values of a byte's codes: [256, 1], or of its two 4-bit codes [256, 2]."""
    grid = torch.from_numpy(np.append(R.GRID[fmt], 0.0) if fmt == R.E4M3 else R.GRID[fmt]).to(DEV)
    both = torch.cat([grid, -grid])
    return both[BYTES][:, None] if fmt == R.E4M3 else torch.stack([both[BYTES % 16], both[BYTES // 16]], 1)


def values(q):
    """float64 [rows, h] on the GPU, and the largest magnitude of every eight elements, none below the format's smallest normal
    one."""
    n = R.blocks(q.h)
    v = torch.empty((q.n_rows, 32 * n), dtype=torch.float64, device=DEV)
    eight = torch.empty((q.n_rows, 4 * n), dtype=torch.float64, device=DEV)
    # (some rows at a time: torch gathers from a table of two columns with a wave for each index, and from 2^26 indices on its
    # grid passes what a launch takes: it is refused, or leaves most of the result unwritten)
    step = max(1, (1 << 24) // (32 * n))
    for r in range(0, q.n_rows, step):
        codes, unit = q.codes[r:r + step, :n * (32 if q.fmt == R.E4M3 else 16)], torch.exp2(q.scales[r:r + step, :n].double() - 127)
        part = table(q.fmt)[codes.int()].view(-1, n, 32) * unit[..., None]
        v[r:r + step] = part.view(-1, 32 * n)
        eight[r:r + step] = part.abs().view(-1, n, 4, 8).amax(3).maximum(unit[..., None] * (2.0 ** -6 if q.fmt == R.E4M3 else 1)).view(-1, 4 * n)
    return v, eight


def random_rows(gen, n, h, fmt, spread):
    """Random codes (no NaN) and scales around 1, zero codes past h, NaN scales behind the last block."""
    q = rows_of(n, h, fmt, fill=0xFF)
    c = torch.randint(0, 254 if fmt == R.E4M3 else 16, (n, R.blocks(h) * 32), generator=gen, device=DEV)
    if fmt == R.E4M3:
        c = torch.where(c >= 127, c + 1, c)
    c[:, h:] = 0
    store(q, c)
    q.scales[:, :R.blocks(h)] = torch.randint(127 - spread, 128 + spread, (n, R.blocks(h)), generator=gen, device=DEV).byte()
    return q


def store(q, codes):
    q.codes.copy_((codes if q.fmt == R.E4M3 else codes[:, 0::2] | (codes[:, 1::2] << 4)).byte())


@pytest.mark.parametrize("dtype", [R.BF16, R.F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: f.name)
def test_form_against_64_bits(form, dtype):
    gen = torch.Generator(device=DEV).manual_seed(hash((50, *form[:4], dtype)) & 0x7fffffff)
    x, w = random_rows(gen, form.rows, form.h, form.fmt, 3), random_rows(gen, form.h_out, form.h, R.E2M1, 3)
    y = apply(x, w, dtype).double()
    (vx, ex), (vw, ew) = values(x), values(w)
    want, size = vx @ vw.t(), vx.abs() @ vw.abs().t()
    # products are exact in float32; at most h + 16 additions, each off by half a step of a partial sum (and one for each
    # further range of K)
    bound = (form.h + 16 + form.ranges) * 2.0 ** -24 * size
    if form.fmt == R.E4M3:
        # of eight consecutive products the matrix instruction cuts off what is below 2^-13 of the power of two under the
        # largest: less than that from each of the other seven
        bound += 7 * 2.0 ** -13 * (ex @ ew.t())
    assert bool(((y - want).abs() <= bound + HALF[dtype] * (want.abs() + bound) + FLOOR[dtype]).all())


@pytest.mark.parametrize("form", FORMS, ids=lambda f: f.name)
def test_form_on_whole_numbers_is_exact(form):
    """Codes of small whole numbers, x and W each in scales of 1 and 2 by blocks: every sum is a whole number below 2^24, so any
    misplaced element or scale shows."""
    gen = torch.Generator(device=DEV).manual_seed(hash((51, *form[:4])) & 0x7fffffff)

    def whole(n, fmt, most):
        q = rows_of(n, form.h, fmt, fill=0xFF)
        v = torch.randint(-most, most + 1, (n, R.blocks(form.h) * 32), generator=gen, device=DEV)
        v[:, form.h:] = 0
        code = torch.tensor([0, 0x38, 0x40, 0x44, 0x48] if fmt == R.E4M3 else [0, 2, 4, 5, 6], device=DEV)[v.abs()]
        store(q, code | torch.where(v < 0, 128 if fmt == R.E4M3 else 8, 0))
        q.scales[:, :R.blocks(form.h)] = torch.randint(127, 129, (n, R.blocks(form.h)), generator=gen, device=DEV).byte()
        return q

    x, w = whole(form.rows, form.fmt, 2), whole(form.h_out, R.E2M1, 4)
    y = apply(x, w, R.F32, 0)
    assert 16424 * 2 * 2 * 4 * 2 < 1 << 24
    assert torch.equal(y.double(), values(x)[0] @ values(w)[0].t())
