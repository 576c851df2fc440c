"""Blocks, norm and the choice of a token by their definitions, in numpy and Python
integers: what the tests compare lora_mx.h and lora_sample.h with."""
import numpy as np

F16, BF16, F32 = 0, 1, 2
E4M3, E2M1 = 0, 1
EMAX = {E4M3: 8, E2M1: 2}

GRID = {
    # magnitudes by code, without the sign
    E4M3: np.array([(c & 7) / 8 * 2.0 ** -6 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)]),
    E2M1: np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6]),
}


def blocks(h):
    return -(-h // 32)


def nearest_code(a, fmt):
    """Codes of the grid values nearest to magnitudes a, ties to the even code, held to the largest."""
    g = GRID[fmt]
    a = np.minimum(a, g[-1])
    hi = np.clip(np.searchsorted(g, a), 1, len(g) - 1)
    down, up = a - g[hi - 1], g[hi] - a
    return np.where((down > up) | ((down == up) & (hi % 2 == 0)), hi, hi - 1).astype(np.uint8)


def quantize(v, fmt):
    """float64 [rows, h] -> codes [rows, bytes], scales [rows, blocks], as they are stored."""
    rows, h = v.shape
    n = blocks(h)
    b = np.zeros((rows, n * 32))
    b[:, :h] = v
    b = b.reshape(rows, n, 32)
    bad = ~np.isfinite(b).all(2)
    m = np.abs(np.where(bad[..., None], 0, b)).max(2)
    top = np.frexp(m)[1] - 1                                   # floor(log2 m)
    scale = np.where(m > 0, np.maximum(0, top - EMAX[fmt] + 127), 0)
    with np.errstate(invalid="ignore"):
        s = b / np.ldexp(1.0, scale - 127)[..., None]
    code = nearest_code(np.abs(np.where(bad[..., None], 0, s)), fmt)
    code |= (np.signbit(b) & ~bad[..., None]).astype(np.uint8) << (7 if fmt == E4M3 else 3)
    scale = np.where(bad, 255, scale).astype(np.uint8)
    code = code.reshape(rows, -1)
    if fmt == E2M1:
        code = code[:, 0::2] | (code[:, 1::2] << 4)
    return code, scale


def values(codes, scales, fmt, h):
    """Stored blocks as float64 [rows, h]."""
    rows, n = codes.shape[0], blocks(h)
    if fmt == E4M3:
        mag = np.append(GRID[fmt], np.nan)[codes & 127]
        v = np.where(codes & 128, -mag, mag)
    else:
        c = np.stack([codes & 15, codes >> 4], 2).reshape(rows, -1)
        v = np.where(c & 8, -GRID[fmt][c & 7], GRID[fmt][c & 7])
    s = scales[:, :n].astype(np.int64)
    unit = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    return (v[:, :n * 32].reshape(rows, n, 32) * unit[..., None]).reshape(rows, -1)[:, :h]


def norm(x, residual, weight, eps):
    """float64 in: (sum, normalised rows)."""
    s = x if residual is None else x + residual
    y = s / np.sqrt((s * s).mean(1, keepdims=True) + eps)
    return s, y if weight is None else y * weight


ONE = 1 << 43


def sample(z, temperature, top_k, top_p, min_p, u):
    """One row: (token, weight of the token, sum of the weights), sums in Python integers."""
    z = np.asarray(z, np.float64)
    z = np.where(np.isnan(z), -np.inf, z) + 0.0
    order = np.lexsort((np.arange(len(z)), -z))
    order = order[z[order] > -np.inf]
    if len(order) == 0:
        return -1, 0, 1
    top = z[order[0]]
    if not temperature >= 2.0 ** -100:
        return int(order[0]), 1, 1
    temperature = min(temperature, 2.0 ** 100)
    with np.errstate(invalid="ignore", over="ignore", under="ignore"):
        d = np.where(z == top, 0.0, (z - top) / np.float64(temperature))
        w = np.rint(np.exp(np.where(np.isnan(d), -np.inf, d)) * ONE).astype(np.int64)
    if 0 < top_k < len(z):
        order = order[:top_k]
    if not top_p >= 1 and not np.isnan(top_p):
        total = int(w[order].sum())
        before = np.concatenate([[0], np.cumsum(w[order])[:-1]]).astype(np.float64)
        n = int((before < float(top_p) * float(total)).sum()) if top_p > 0 else 1
        order = order[:max(1, n)]
    if min_p > 0:
        order = order[w[order].astype(np.float64) >= float(min(min_p, 1)) * ONE]
    left = np.sort(order)
    cum = np.cumsum(w[left])
    total = int(cum[-1])
    uu = 1.0 if u >= 1 else float(u) if u > 0 else 0.0
    target = min(int(np.floor(uu * float(total))), total - 1)
    i = int((cum <= target).sum())
    return int(left[i]), int(w[left[i]]), total
