"""Products of more tiles than one launch has: every row and column of y, against a product of one launch."""
import numpy as np
import pytest

import mx_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_mx import DEV, apply, random_rows, stream  # noqa: E402

from paper_2401_11240_amd import mx as MX  # noqa: E402

PERIOD = (1 << 20) + 7     # rows after which the operand of many rows repeats


def repeated(q, n):
    """q's rows again and again, n rows."""
    out = MX.empty_rows(n, q.h, q.fmt, DEV)
    for to, src in ((out.codes, q.codes), (out.scales, q.scales)):
        for r in range(0, n, q.n_rows):
            to[r:r + q.n_rows] = src[:min(q.n_rows, n - r)]
    return out


def product(x, w):
    n = MX.lora_mx_workspace_bytes(x, w)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    y = torch.full((x.n_rows, w.n_rows), -1, dtype=torch.bfloat16, device=DEV)
    MX.lora_mx_apply(x, w, y, w.n_rows, R.BF16, ws, n, stream())
    return y


def test_more_rows_than_a_launch_has():
    rng = np.random.default_rng(30)
    x, w = random_rows(rng, PERIOD, 32, R.E2M1), random_rows(rng, 8, 32, R.E2M1)
    want = apply(x, w, R.BF16, 0)
    rows = (1 << 28) + 64
    y = product(repeated(x, rows), w)
    for r in range(0, rows, PERIOD):
        assert torch.equal(y[r:r + PERIOD], want[:rows - r]), r


def test_more_columns_than_a_launch_has():
    rng = np.random.default_rng(31)
    x, w = random_rows(rng, 8, 32, R.E2M1), random_rows(rng, PERIOD + 1, 32, R.E2M1)      # (a multiple of 8)
    want = apply(x, w, R.BF16, 0)
    cols = (1 << 29) + 64
    y = product(x, repeated(w, cols))
    for n in range(0, cols, w.n_rows):
        assert torch.equal(y[:, n:n + w.n_rows], want[:, :cols - n]), n
