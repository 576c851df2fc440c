"""The choice of the next token (include/lora_sample.h) against its definition in whole numbers
(mx_reference.py): tokens equal, probabilities within one rounding."""
import numpy as np
import pytest

import mx_reference as R

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():   # collected on CPU-only hosts, never run there
    pytest.skip("no GPU", allow_module_level=True)

from paper_2401_11240_amd import sample as SA  # noqa: E402

DEV = torch.device("cuda:0")
TYPE = {R.F16: torch.float16, R.BF16: torch.bfloat16, R.F32: torch.float32}
NAMES = {R.F16: "f16", R.BF16: "bf16", R.F32: "f32"}
dtypes = pytest.mark.parametrize("dtype", [R.F16, R.BF16, R.F32], ids=NAMES.get)


def stream():
    return torch.cuda.current_stream(DEV)


def device(a, t):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, t)).to(DEV)


def choose(z, params, u, dtype, st=None):
    """z a device matrix (a view of wider rows, perhaps)."""
    rows, v = z.shape
    n = SA.lora_sample_workspace_bytes(rows, v, dtype)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    tokens = torch.full((rows + 2,), -7, dtype=torch.int32, device=DEV)
    probs = torch.full((rows + 2,), -7.0, device=DEV)
    u = device(u, np.float32)
    SA.lora_sample(z, z.stride(0) if rows > 1 else v, dtype, rows, v, params, u, tokens, probs, ws, n, st or stream())
    torch.cuda.synchronize()
    assert (tokens[rows:] == -7).all() and (probs[rows:] == -7).all() and (ws[n:] == 0xFF).all()
    return tokens[:rows].cpu().numpy(), probs[:rows].cpu().numpy()


def check(z, t, k, p, m, u, dtype):
    rows = z.shape[0]
    params = SA.Params(device(t, np.float32), device(k, np.int32), device(p, np.float32), device(m, np.float32))
    tokens, probs = choose(z, params, u, dtype)
    zz = z.double().cpu().numpy()
    at = lambda a, r, none: none if a is None else np.float32(a[r]) if none != 0 or a is not k else a[r]  # noqa: E731
    for r in range(rows):
        want, own, total = R.sample(zz[r], at(t, r, 1.0), 0 if k is None else int(k[r]), at(p, r, 1.0),
                                    0.0 if m is None else np.float32(m[r]), np.float32(u[r]))
        assert tokens[r] == want, (r, tokens[r], want, [None if a is None else a[r] for a in (t, k, p, m)], u[r])
        # the ratio of two whole numbers, each rounded to binary64, in binary64 and then in float32
        assert abs(probs[r] - own / total) <= own / total * (2.0 ** -24 + 2.0 ** -50), (r, probs[r], own / total)
    return tokens


def logits(rng, rows, v, dtype, pad=0, scale=2.0):
    z = rng.standard_normal((rows, v)) * scale
    for r in range(rows):
        at = rng.integers(0, v, min(v, 12))
        z[r, at] += rng.uniform(0, 14, len(at)) * rng.random()
    whole = torch.full((rows, v + pad), 1000.0, device=DEV).to(TYPE[dtype])
    whole[:, :v] = torch.from_numpy(z).to(DEV).to(TYPE[dtype])
    return whole[:, :v]


def mixed(rng, rows, v):
    t = np.where(rng.random(rows) < 0.1, 0, rng.uniform(0.2, 2, rows)).astype(np.float32)
    k = np.where(rng.random(rows) < 0.5, 0, rng.integers(1, max(2, min(v, 400)), rows)).astype(np.int32)
    p = np.where(rng.random(rows) < 0.3, 1, rng.uniform(0.02, 1, rows)).astype(np.float32)
    m = np.where(rng.random(rows) < 0.5, 0, rng.uniform(0, 0.4, rows)).astype(np.float32)
    return t, k, p, m


@dtypes
@pytest.mark.parametrize("rows,v,pad", [(1, 1, 0), (3, 2, 3), (40, 17, 0), (9, 257, 1), (33, 1000, 0), (24, 4096, 8), (8, 32000, 0),
                                        (5, 50257, 0), (6, 65537, 3), (4, 131072, 16), (2, 524288, 0), (300, 700, 0)])
def test_tokens_of_mixed_requests(rows, v, pad, dtype):
    rng = np.random.default_rng([1, rows, v, dtype])
    z = logits(rng, rows, v, dtype, pad)
    check(z, *mixed(rng, rows, v), rng.random(rows).astype(np.float32), dtype)


@dtypes
@pytest.mark.parametrize("what", ["temperature", "top_k", "top_p", "min_p", "none", "no arrays"])
@pytest.mark.parametrize("v", [300, 40001])
def test_each_parameter_alone(v, what, dtype):
    rows = 12
    rng = np.random.default_rng([2, v, dtype])
    z = logits(rng, rows, v, dtype)
    t, k, p, m = mixed(rng, rows, v)
    one = {"temperature": (t, None, None, None), "top_k": (None, k, None, None), "top_p": (None, None, p, None),
           "min_p": (None, None, None, m), "none": (t * 0 + 1, k * 0, p * 0 + 1, m * 0), "no arrays": (None,) * 4}[what]
    check(z, *one, rng.random(rows).astype(np.float32), dtype)


@dtypes
@pytest.mark.parametrize("v", [1, 64, 5000, 70000])
def test_equal_logits_go_to_the_lowest_indices(v, dtype):
    """All equal, and few distinct values: the thresholds cut through equal ones."""
    rng = np.random.default_rng([3, v])
    rows = 24
    z = torch.zeros((rows, v), device=DEV, dtype=TYPE[dtype])
    z[8:] = torch.from_numpy(rng.integers(-3, 3, (rows - 8, v)) * 0.5).to(DEV).to(TYPE[dtype])
    z[5, ::2] = -0.0
    k = np.array([0, 1, 2, 63, 64, 1000, 4999, 69999] * 3, np.int32)
    p = np.array([1, 0.5, 0.25, 1, 0.9, 0.999, 0.01, 0.3] * 3, np.float32)
    u = np.array([0, 0.5, 0.999999, 0.25] * 6, np.float32)
    check(z, np.ones(rows, np.float32), k, p, np.zeros(rows, np.float32), u, dtype)
    check(z, np.full(rows, 0.7, np.float32), k, p, np.full(rows, 0.3, np.float32), u, dtype)


@dtypes
@pytest.mark.parametrize("scale", [0.02, 0.3, 3.0])
@pytest.mark.parametrize("v", [5000, 40000])
def test_filters_that_end_among_many(v, scale, dtype):
    """Few, hundreds and thousands of logits before and at the places where top_k and top_p end."""
    rng = np.random.default_rng([4, v, int(100 * scale), dtype])
    k = np.array([0, 2, 64, 255, 256, 257, 511, 512, 513, 1000, 2500, 4000] * 3, np.int32)
    p = np.repeat(np.array([1, 0.9, 0.03], np.float32), 12)
    m = np.where(np.arange(36) % 5 == 0, 0.6, 0).astype(np.float32)
    z = torch.from_numpy(rng.standard_normal((36, v)) * scale).to(DEV).to(TYPE[dtype])
    check(z, np.ones(36, np.float32), k, p, m, rng.random(36).astype(np.float32), dtype)


@dtypes
@pytest.mark.parametrize("likely", [300, 1500, 2900])
@pytest.mark.parametrize("v", [7000, 20000, 60000])
def test_likely_logits_that_are_neighbours(v, likely, dtype):
    """All that the filters leave lies in a short piece of the row, at its start, inside and at its end."""
    rng = np.random.default_rng([5, v, likely, dtype])
    z = rng.standard_normal((18, v)) * 0.5 - 20
    for r in range(18):
        first = (0, (v - likely) // 3, v - likely)[r % 3]
        z[r, first:first + likely] += 20
    z = torch.from_numpy(z).to(DEV).to(TYPE[dtype])
    k = np.repeat(np.array([0, 280, 1000], np.int32), 6)
    p = np.array([1, 1, 1, 0.9, 0.9, 0.4] * 3, np.float32)
    m = np.where(np.arange(18) % 4 == 3, 0.2, 0).astype(np.float32)
    check(z, np.ones(18, np.float32), k, p, m, rng.random(18).astype(np.float32), dtype)


@dtypes
@pytest.mark.parametrize("v", [9, 3000, 90000])
def test_masked_infinite_and_nan_logits(v, dtype):
    rng = np.random.default_rng([4, v])
    rows = 12
    z = logits(rng, rows, v, dtype)
    z[0] = float("-inf")
    z[1] = float("nan")
    z[2, 1:] = float("-inf")
    z[3, :-1] = float("nan")
    z[4, 2], z[4, 5] = float("inf"), float("inf")
    z[5, rng.random(v) < 0.5] = float("-inf")
    z[6, rng.random(v) < 0.5] = float("nan")
    z[7] = torch.finfo(TYPE[dtype]).min
    z[8] = torch.finfo(TYPE[dtype]).min
    z[8, v // 2] = torch.finfo(TYPE[dtype]).max
    z[9, rng.random(v) < 0.9] = torch.finfo(TYPE[dtype]).min
    z[10] = float("-inf")
    z[10, v - 2:] = 3.0
    z[11] = float("inf")
    u = rng.random(rows).astype(np.float32)
    for t, k, p, m in ((1, 0, 1, 0), (0.5, 5, 0.8, 0.1), (0, 0, 1, 0), (1.5, 1, 1, 0), (1, 0, 0.5, 0), (1, v - 1, 0.99, 0)):
        full = lambda x, d: np.full(rows, x, d)  # noqa: E731
        tokens = check(z, full(t, np.float32), full(k, np.int32), full(p, np.float32), full(m, np.float32), u, dtype)
        assert tokens[0] == -1 and tokens[1] == -1


@dtypes
def test_parameters_outside_their_ranges(dtype):
    v, nan, inf = 777, np.nan, np.inf
    rng = np.random.default_rng(5)
    t = [1, -1, nan, 0, 1e-30, inf, 1e30, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1e-45]
    k = [-5, 0, 0, 3, 0, 0, 0, v, v + 1, 2 ** 31 - 1, -2 ** 31, 0, 0, 0, 0, 0, 0, 0, 0]
    p = [1, 1, 1, 1, 1, 1, 0.5, 1, 1, 1, 2, 0, -1, nan, inf, 1, 1, 1, 1]
    m = [0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1, 2, nan, 0]
    rows = len(t)
    z = logits(rng, rows, v, dtype, pad=5)
    for u in (np.zeros(rows), np.full(rows, 1 - 2.0 ** -24), np.full(rows, 0.37), np.full(rows, 1.0), np.full(rows, 7.0),
              np.full(rows, -1.0), np.full(rows, nan)):
        check(z, np.array(t, np.float32), np.array(k, np.int32), np.array(p, np.float32), np.array(m, np.float32),
              u.astype(np.float32), dtype)


@pytest.mark.parametrize("dtype", [R.BF16, R.F32], ids=NAMES.get)
@pytest.mark.parametrize("v", [900, 70000])
def test_temperatures_at_the_ends_of_their_range(v, dtype):
    """Logits as far apart as the temperature, up to the type's whole range and down to its subnormal
    numbers; past the ends of 2^-100 .. 2^100 the temperature does not matter any more."""
    rng = np.random.default_rng([8, v])
    t, scale = zip(*[(2.0 ** 100, 1e30), (1e38, 1e30), (np.inf, 1e30), (2.0 ** 100, 1e38), (1e30, 3e37), (1.1e30, 2e30),
                     (2.0 ** -100, 1e-30), (7.8e-31, 1e-30), (1e-30, 1e-30), (1e-30, 1e-38), (1e-38, 1e-38), (1, 1e-40)])
    rows = len(t)
    z = torch.from_numpy(rng.standard_normal((rows, v)) * np.array(scale)[:, None]).to(DEV).to(TYPE[dtype])
    for k, p, m in ((0, 1, 0), (0, 0.7, 0), (0, 1, 0.2), (40, 0.9, 0.05), (v - 1, 0.9, 0.01)):
        full = lambda x, d: np.full(rows, x, d)  # noqa: E731
        check(z, np.array(t, np.float32), full(k, np.int32), full(p, np.float32), full(m, np.float32),
              rng.random(rows).astype(np.float32), dtype)


def test_frequencies_follow_the_probabilities():
    """u in even steps meets every token as often as its share: counts are off by at most 1 on
    either side of its stretch, and by the rounding of u."""
    rng = np.random.default_rng(6)
    v, n = 50, 4096
    row = torch.from_numpy(rng.standard_normal((1, v)) * 1.5).to(DEV).float()
    z = row.expand(n, v).contiguous()
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tokens, probs = choose(z, None, u, R.F32)
    soft = torch.softmax(row.double(), 1)[0].cpu().numpy()
    counts = np.bincount(tokens, minlength=v)
    assert (np.abs(counts - soft * n) <= 1 + 1e-3).all()
    assert np.abs(probs - soft[tokens]).max() <= 2.0 ** -23
    assert (np.diff(tokens) >= 0).all()


def test_recorded_with_new_logits_and_parameters():
    rng = np.random.default_rng(7)
    rows, v = 20, 9000
    z = logits(rng, rows, v, R.BF16)
    t, k, p, m = (device(a, d) for a, d in zip(mixed(rng, rows, v), (np.float32, np.int32, np.float32, np.float32)))
    u = device(rng.random(rows), np.float32)
    params = SA.Params(t, k, p, m)
    tokens = torch.empty(rows, dtype=torch.int32, device=DEV)
    n = SA.lora_sample_workspace_bytes(rows, v, R.BF16)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    st = torch.cuda.Stream()
    st.wait_stream(stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        SA.lora_sample(z, v, R.BF16, rows, v, params, u, tokens, None, ws, n, st)
    for i in range(4):
        z.copy_(logits(rng, rows, v, R.BF16))
        new = mixed(rng, rows, v)
        for dst, a, d in zip((t, k, p, m), new, (np.float32, np.int32, np.float32, np.float32)):
            dst.copy_(device(a, d))
        uu = rng.random(rows).astype(np.float32)
        u.copy_(device(uu, np.float32))
        tokens.fill_(-9)
        g.replay()
        torch.cuda.synchronize()
        got = tokens.cpu().numpy()
        assert np.array_equal(got, choose(z, params, uu, R.BF16)[0])
        assert np.array_equal(got, check(z, *new, uu, R.BF16))


def test_no_rows():
    z = torch.zeros((0, 100), device=DEV)
    tokens, probs = choose(z, None, np.zeros(0), R.F32)
    assert tokens.size == 0


@pytest.mark.parametrize("v", [700, 40000])
def test_rows_more_than_4_gib_apart(v):
    rng = np.random.default_rng([9, v])
    ld = (1 << 32) + 3
    z = torch.empty(ld + v, dtype=torch.float16, device=DEV).as_strided((2, v), (ld, 1))
    z.copy_(logits(rng, 2, v, R.F16))
    check(z, *mixed(rng, 2, v), rng.random(2).astype(np.float32), R.F16)


def test_more_rows_than_a_launch_has():
    """Rows past 2^20 go to launches of their own."""
    rows, v = (1 << 20) + 37, 9
    rng = np.random.default_rng(10)
    gen = torch.Generator(device=DEV).manual_seed(10)
    z = torch.randn((rows, v), generator=gen, device=DEV).half()
    t, k, p, m = mixed(rng, rows, v)
    u = rng.random(rows).astype(np.float32)
    params = SA.Params(device(t, np.float32), device(k, np.int32), device(p, np.float32), device(m, np.float32))
    tokens, probs = choose(z, params, u, R.F16)
    at = np.concatenate([np.arange(300), np.arange((1 << 20) - 50, rows)])
    zz = z[torch.from_numpy(at).to(DEV)].double().cpu().numpy()
    for i, r in enumerate(at):
        want, own, total = R.sample(zz[i], t[r], int(k[r]), p[r], m[r], u[r])
        assert tokens[r] == want, r
        assert abs(probs[r] - own / total) <= own / total * (2.0 ** -24 + 2.0 ** -50), r


def test_logits_on_the_host_are_refused():
    z, u = torch.zeros((2, 64)), torch.zeros(2, device=DEV)
    tokens, ws = torch.zeros(2, dtype=torch.int32, device=DEV), torch.empty(64, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        SA.lora_sample(z, 64, R.F32, 2, 64, None, u, tokens, None, ws, 64, stream())


@pytest.mark.parametrize("rows,v", [(3, 24576), (3, 24577), (64, 24577), (65, 24577), (65, 49152), (65, 49153), (128, 49153), (129, 49153)])
def test_sizes_at_the_borders_between_one_launch_and_several(rows, v):
    rng = np.random.default_rng([10, rows, v])
    z = logits(rng, rows, v, R.BF16, pad=1)
    check(z, *mixed(rng, rows, v), rng.random(rows).astype(np.float32), R.BF16)


def test_two_recordings_of_several_launches_share_a_workspace():
    """Rows of slices and rows of one workgroup, replayed in turn with other inputs and eager calls between."""
    rng = np.random.default_rng(11)
    st = torch.cuda.Stream()
    st.wait_stream(stream())
    shapes = ((6, 50000), (9, 30000))
    n = max(SA.lora_sample_workspace_bytes(rows, v, R.F32) for rows, v in shapes)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    made = []
    for rows, v in shapes:
        z, u = logits(rng, rows, v, R.F32), device(rng.random(rows), np.float32)
        arrays = [device(a, d) for a, d in zip(mixed(rng, rows, v), (np.float32, np.int32, np.float32, np.float32))]
        params, tokens = SA.Params(*arrays), torch.empty(rows, dtype=torch.int32, device=DEV)
        probs = torch.empty(rows, device=DEV)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            SA.lora_sample(z, v, R.F32, rows, v, params, u, tokens, probs, ws, n, st)
        made.append((rows, v, z, u, arrays, params, tokens, probs, g))
    for i in range(6):
        rows, v, z, u, arrays, params, tokens, probs, g = made[i % 2]
        z.copy_(logits(rng, rows, v, R.F32, scale=(2.0, 0.02, 0.5)[i // 2]))
        new = mixed(rng, rows, v)
        for dst, a, d in zip(arrays, new, (np.float32, np.int32, np.float32, np.float32)):
            dst.copy_(device(a, d))
        uu = rng.random(rows).astype(np.float32)
        u.copy_(device(uu, np.float32))
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        torch.cuda.synchronize()
        got, own = tokens.cpu().numpy(), probs.cpu().numpy()
        eager = choose(z, params, uu, R.F32)
        assert np.array_equal(got, eager[0]) and np.array_equal(own, eager[1])
        assert np.array_equal(got, check(z, *new, uu, R.F32))
