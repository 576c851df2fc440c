"""Attention at the ends of the number range: scores far beyond those of a trained model
and weights far below the largest, for single tokens and prompts in both types."""
import numpy as np
import pytest

import kv_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2401_11240_amd import kv as KV  # noqa: E402
from test_gpu_kv import DEV, DTYPES, Case, stream  # noqa: E402


@pytest.fixture(scope="module")
def attn():
    a = KV.lora_attn_create(0, stream())
    yield a
    torch.cuda.synchronize()
    KV.lora_attn_destroy(a)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 64), (4, 2, 128), (4, 1, 256), (72, 1, 64), (68, 4, 128), (64, 64, 80)])
def test_scores_of_any_size(attn, dtype, sign, heads, kv_heads, dim):
    # q is 2^15 everywhere, key j a_j everywhere: scores of up to dim * 2^15 * 2^15 sqrt(dim) apart by thousands,
    # exact in float32, so that each row's output is the value of its largest score, bit for bit
    n = 300
    a = sign * 128 * np.random.default_rng(dim).permutation(np.arange(1, 257))        # eight bits and less
    a = np.concatenate([a, a[:n - 256]])[:n]
    for kind in ("prompt", "decode"):
        c = Case(dtype, heads, kv_heads, dim, 16, [n], [n if kind == "prompt" else 1], seed=3)
        first = 0 if kind == "prompt" else n - 1
        k = torch.zeros(c.kd[0].shape, dtype=torch.float32)
        v = np.zeros((n, kv_heads, dim))
        for j in range(n):
            k[c.table[0, j // 16], :, j % 16] = float(a[j])
            v[j] = c.v[c.table[0, j // 16], :, j % 16]
        # (a key stands twice where the list starts again: the same value there)
        for j in range(256, n):
            v[j] = v[j - 256]
            c.vd[0][int(c.table[0, j // 16]), :, j % 16] = torch.from_numpy(v[j]).to(DTYPES[dtype]).to(DEV)
        c.kd[0].copy_(k)
        c.qd.fill_(2.0 ** 15)
        getattr(c, kind)(attn)
        got = c.got()
        for r in range(got.shape[0]):
            best = int(np.argmax(a[:first + r + 1]))
            want = v[best][np.arange(heads) // (heads // kv_heads)]
            assert np.array_equal(got[r], want), (kind, r)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [2, 72])
def test_scores_that_come_up_from_far_below(attn, dtype, heads):
    # the first 100 tokens score about -2^30, the others as usual: the early ones leave nothing behind
    for kind in ("prompt", "decode"):
        c = Case(dtype, heads, 1, 64, 16, [400], [280 if kind == "prompt" else 1], seed=5)
        k = c.kd[0].float().cpu()
        for j in range(100):
            k[c.table[0, j // 16], :, j % 16] = -30720.0
        c.kd[0].copy_(k)
        c.k = c.kd[0].double().cpu().numpy()
        c.qd.fill_(2.0 ** -6)
        for d in range(8):                       # the first dimensions decide
            c.qd[:, d::64] = 2.0 ** 15
        for j in range(100, 400):
            c.kd[0][int(c.table[0, j // 16]), :, j % 16, :8] = 0.0
        c.k = c.kd[0].double().cpu().numpy()
        c.q = c.qd[:, :heads * 64].double().cpu().numpy().reshape(-1, heads, 64)
        getattr(c, kind)(attn)
        got = c.got()
        lo = 400 - got.shape[0]
        for r in range(got.shape[0]):            # rows before token 100 are left out: all their scores are alike
            if lo + r < 100:
                continue
            ref, m, reach = R.attention(c.q[r:r + 1], c.k, c.v, c.table[0], lo + r + 1, lo + r, c.scale, 0, 0)
            # (the reach is that of the tokens that have weight)
            near = c.k.copy()
            near[near <= -30000.0] = 0.0
            _, _, reach = R.attention(c.q[r:r + 1], near, c.v, c.table[0], lo + r + 1, lo + r, c.scale, 0, 0)
            tol = R.allowance(ref, m, reach, 64, 400, dtype == "bf16")
            assert (np.abs(got[r:r + 1] - ref) <= tol).all(), (kind, r)


@pytest.mark.parametrize("kind,heads,lens", [("prompt", 2, [131072]), ("prompt", 72, [131072]), ("prompt", 2, [20000, 9000]),
                                             ("decode", 2, [1024] * 1024), ("decode", 16, [131072, 5])])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_long_tail_of_weights_far_below_the_largest(attn, dtype, kind, heads, lens):
    # the first token has weight 1 and value 0, the others 2^-26.4 and values of 1 to 2: they are the output.
    # A weight of 2^-26.4, times 2^7, is off by half of binary16's smallest, 2^-25 of 2^-19.4: 2^-5.6 of it, all
    # alike, in the output and (hardly) in the sum; bfloat16 rounds it by 2^-9.  Then the output's own rounding.
    rows = [{72: 120}.get(heads, 40) if kind == "prompt" else 1 for _ in lens]
    c = Case(dtype, heads, 1, 64, 256, lens, [min(r, n) for r, n in zip(rows, lens)], seed=37)
    k = torch.zeros(c.kd[0].shape, dtype=torch.float32)
    for s in range(len(lens)):
        k[c.table[s, 0], :, 0, 0] = 15.0
    c.kd[0].copy_(k)
    v = torch.where(torch.isnan(c.vd[0]), c.vd[0], 1 + c.vd[0].abs().clamp(max=1))
    for s in range(len(lens)):
        v[int(c.table[s, 0]), :, 0] = 0
    c.vd[0].copy_(v)
    c.qd.zero_()
    for h in range(heads):
        c.qd[:, h * 64] = 9.75                   # 15 * 9.75 / 8 = 18.28 = 26.4 powers of two
    getattr(c, kind)(attn)
    got = c.got()
    vv = c.vd[0].double().cpu().numpy()
    w = np.exp(-15 * 9.75 / 8)
    at = 0
    for s, n in enumerate(lens):
        tokens = vv[c.table[s, :-(-n // 256)], 0].reshape(-1, 64)[:n]
        sums = np.cumsum(tokens, axis=0)
        for r in range(c.rows[s]):
            j = n - c.rows[s] + r                # sees tokens 0 .. j
            want = w * sums[j] / (1 + w * j)
            tol = (2.0 ** -5.6 if dtype == "f16" else 2.0 ** -8) * 1.1 * want + 2.0 ** -25
            assert (np.abs(got[at] - want) <= tol).all(), (s, r, got[at, 0, :4], want[:4])
            at += 1
