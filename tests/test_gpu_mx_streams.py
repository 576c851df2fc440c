"""Products whose K is split, on two streams at once: their sums lie in workspaces of their own."""
import numpy as np
import pytest

import mx_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from test_gpu_mx import DEV, apply, check_product, random_rows  # noqa: E402

from paper_2401_11240_amd import mx as MX  # noqa: E402


def test_split_products_on_two_streams_at_once():
    rng = np.random.default_rng(60)
    jobs = []
    for rows, h, h_out in ((48, 2048, 1032), (200, 2080, 1032)):
        x, w = random_rows(rng, rows, h, R.E4M3), random_rows(rng, h_out, h, R.E2M1)
        n = MX.lora_mx_workspace_bytes(x, w)
        assert n >= 2 * 4 * rows * h_out                  # sums of two ranges and more, which the call leaves in the workspace
        want = apply(x, w, R.F32, 0)
        check_product(x, w, want, R.F32)
        jobs.append((x, w, torch.empty(n, dtype=torch.uint8, device=DEV), want, torch.cuda.Stream()))
    ys = [[torch.empty((j[0].n_rows, j[1].n_rows), device=DEV) for _ in range(100)] for j in jobs]
    torch.cuda.synchronize()
    for i in range(100):
        for (x, w, ws, _, st), y in zip(jobs, ys):
            MX.lora_mx_apply(x, w, y[i], w.n_rows, R.F32, ws, ws.numel(), st)
    torch.cuda.synchronize()
    for (_, _, _, want, _), y in zip(jobs, ys):
        assert all(torch.equal(a, want) for a in y)
