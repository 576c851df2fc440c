"""Rows in blocks, their product, the norm and the choice of the next token on the host: headers
and bindings agree, the library exports what the headers declare, and bad arguments are refused
before any GPU work (device pointers here are made-up addresses that no call may touch)."""
import ctypes as C
import os
import re

import pytest

from paper_2401_11240_amd import build as B
from paper_2401_11240_amd import lora as L
from paper_2401_11240_amd import mx as MX
from paper_2401_11240_amd import sample as SA

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GB = 1 << 30           # made-up addresses lie whole GiB apart
OK, ARG, SHAPE, ALIGN, OVERLAP, WS = 0, L.LORA_E_ARG, L.LORA_E_SHAPE, L.LORA_E_ALIGN, L.LORA_E_OVERLAP, L.LORA_E_WORKSPACE
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(B.lib_path()):
        B.build()
    L.load()


@pytest.mark.parametrize("header,exports", [("lora_mx.h", MX.EXPORTS), ("lora_sample.h", SA.EXPORTS)])
def test_header_binding_and_library_agree(header, exports):
    text = open(os.path.join(ROOT, "include", header)).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"^\s*int\s+(lora_\w+)\s*\(", text, flags=re.M)))
    assert names == sorted(exports)
    for n in names:
        assert hasattr(L.load(), n), n


def code(rc):
    if rc != 0:
        assert L.lora_last_error()
    return rc


def rows(**kw):
    f = dict(codes=GB, scales=2 * GB, ld_codes=128, ld_scales=4, n_rows=5, h=128, format=MX.LORA_E4M3)
    f.update(kw)
    return MX._Rows(**f)


def weight(**kw):
    return rows(**dict(dict(codes=3 * GB, scales=4 * GB, ld_codes=64, n_rows=16, format=MX.LORA_E2M1), **kw))


BAD_ROWS = [(dict(format=2), ARG), (dict(format=-1), ARG), (dict(n_rows=-1), ARG), (dict(h=0), SHAPE), (dict(h=-8), SHAPE),
            (dict(h=124), SHAPE), (dict(ld_codes=120), SHAPE), (dict(ld_codes=112), SHAPE), (dict(ld_codes=2 * BIG), SHAPE),
            (dict(h=136), SHAPE), (dict(ld_scales=3), SHAPE), (dict(ld_scales=6), SHAPE), (dict(ld_scales=0), SHAPE),
            (dict(ld_scales=2 * BIG), SHAPE), (dict(codes=0), ARG), (dict(scales=0), ARG), (dict(codes=GB + 8), ALIGN),
            (dict(scales=2 * GB + 2), ALIGN)]


def quantize(q, x=5 * GB, ld=128, dtype=L.LORA_F16):
    return MX._lib().lora_mx_quantize(x, ld, dtype, q and C.byref(q), None)


def dequantize(q, y=5 * GB, ld=128, dtype=L.LORA_F16):
    return MX._lib().lora_mx_dequantize(q and C.byref(q), y, ld, dtype, None)


def norm(q=None, x=5 * GB, ldx=128, res=6 * GB, ldr=128, w=7 * GB, eps=1e-5, n=5, h=128, dtype=L.LORA_BF16, total=8 * GB,
         ldt=128, y=9 * GB, ldy=128):
    return MX._lib().lora_norm(x, ldx, res, ldr, w, eps, n, h, dtype, total, ldt, y, ldy, q and C.byref(q), None)


def apply(x, w, y=10 * GB, ldy=16, dtype=L.LORA_F16, ws=11 * GB, ws_bytes=1 << 20):
    return MX._lib().lora_mx_apply(x and C.byref(x), w and C.byref(w), y, ldy, dtype, ws, ws_bytes, None)


def space(x, w):
    n = C.c_size_t()
    return MX._lib().lora_mx_workspace_bytes(x and C.byref(x), w and C.byref(w), C.byref(n))


@pytest.mark.parametrize("bad,want", BAD_ROWS)
def test_bad_rows(bad, want):
    q = rows(**bad)
    h = q.h if want != SHAPE else 128
    assert code(quantize(q)) == want
    assert code(dequantize(q)) == want
    if q.n_rows == 5 and q.h == h:
        assert code(norm(q)) == want
    assert code(space(q, weight(h=q.h))) == want
    assert code(apply(q, weight(h=q.h))) == want


@pytest.mark.parametrize("bad,want", [b for b in BAD_ROWS if "ld_codes" not in b[0]])
def test_bad_weights(bad, want):
    w = weight(**{k: v + 2 * GB if k in ("codes", "scales") and v else v for k, v in bad.items()})
    assert code(space(rows(h=w.h), w)) in (want, SHAPE)
    assert code(apply(rows(), w)) == want


def test_bad_values():
    for call, name in ((quantize, "x"), (dequantize, "y")):
        assert code(call(None)) == ARG
        for dtype in (3, -1):
            assert code(call(rows(), dtype=dtype)) == ARG
        assert code(call(rows(), 0)) == ARG
        assert code(call(rows(), 5 * GB + 8)) == ALIGN
        assert code(call(rows(), ld=120)) == SHAPE
        assert code(call(rows(), ld=132)) == SHAPE
        assert code(call(rows(), ld=2 * BIG)) == SHAPE
        # the last of 5 rows of 128 float32, and one byte of the codes' or scales'
        assert code(call(rows(), GB - 4 * (4 * 128 + 128) + 16, dtype=MX.LORA_F32)) == OVERLAP
        assert code(call(rows(), GB + 4 * 128 + 112)) == OVERLAP
        assert code(call(rows(), 2 * GB)) == OVERLAP
        assert code(call(rows(scales=GB + 16))) == OVERLAP
        assert call(rows(n_rows=0, codes=0, scales=0), 0) == OK


BAD_NORM = [(dict(dtype=2), ARG), (dict(dtype=-1), ARG), (dict(n=-1), ARG), (dict(h=0), SHAPE), (dict(h=12), SHAPE),
            (dict(h=65544, ldx=65544), SHAPE), (dict(eps=0.0), ARG), (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG),
            (dict(eps=float("inf")), ARG), (dict(y=0), ARG), (dict(x=0), ARG), (dict(x=5 * GB + 8), ALIGN),
            (dict(ldx=120), SHAPE), (dict(ldx=132), SHAPE), (dict(ldx=2 * BIG), SHAPE), (dict(res=6 * GB + 2), ALIGN),
            (dict(ldr=64), SHAPE), (dict(w=7 * GB + 4), ALIGN), (dict(total=8 * GB + 8), ALIGN), (dict(ldt=126), SHAPE),
            (dict(y=9 * GB + 8), ALIGN), (dict(ldy=0), SHAPE),
            (dict(y=5 * GB + 16), OVERLAP), (dict(y=5 * GB, ldy=136), OVERLAP), (dict(total=6 * GB + 256), OVERLAP),
            (dict(y=7 * GB), OVERLAP), (dict(total=9 * GB), OVERLAP), (dict(total=5 * GB, y=5 * GB), OVERLAP),
            (dict(x=5 * GB, res=5 * GB + 256, total=5 * GB), OVERLAP)]


@pytest.mark.parametrize("bad,want", BAD_NORM)
def test_bad_norms(bad, want):
    assert code(norm(**bad)) == want


def test_bad_norms_in_blocks():
    assert code(norm(rows(n_rows=4))) == SHAPE
    assert code(norm(rows(h=120))) == SHAPE
    assert code(norm(rows(codes=5 * GB))) == OVERLAP
    assert code(norm(rows(scales=9 * GB + 4))) == OVERLAP
    assert code(norm(rows(scales=GB + 4))) == OVERLAP
    assert code(norm(rows(codes=7 * GB))) == OVERLAP
    assert norm(rows(n_rows=0), n=0, x=0, res=0, total=0, w=0, y=0) == OK
    assert norm(n=0, x=0, res=0, total=0, y=9 * GB) == OK


BAD_PRODUCT = [(dict(dtype=3), ARG), (dict(y=0), ARG), (dict(y=10 * GB + 8), ALIGN), (dict(ldy=8), SHAPE), (dict(ldy=20), SHAPE),
               (dict(ldy=2 * BIG), SHAPE), (dict(ws=0), WS), (dict(ws_bytes=0), WS), (dict(ws=11 * GB + 8), ALIGN),
               (dict(y=GB), OVERLAP), (dict(y=2 * GB), OVERLAP), (dict(y=3 * GB + 16), OVERLAP), (dict(y=4 * GB), OVERLAP),
               (dict(ws=GB), OVERLAP), (dict(ws=4 * GB), OVERLAP), (dict(ws=10 * GB), OVERLAP)]


@pytest.mark.parametrize("bad,want", BAD_PRODUCT)
def test_bad_products(bad, want):
    assert code(apply(rows(), weight(), **bad)) == want


def test_rows_and_weights_that_do_not_fit():
    assert code(apply(None, weight())) == ARG
    assert code(apply(rows(), None)) == ARG
    assert code(apply(rows(), weight(format=MX.LORA_E4M3, ld_codes=128))) == ARG
    assert code(apply(rows(h=120), weight())) == SHAPE
    for n in (0, 4, 12):
        assert code(apply(rows(), weight(n_rows=n))) == SHAPE
    big = 1 << 24                          # 256 rows span 4 GiB
    assert code(apply(rows(ld_codes=big), weight())) == SHAPE
    assert code(apply(rows(), weight(ld_scales=big))) == SHAPE
    many = dict(codes=64 * GB, scales=32 * GB, n_rows=0x7fffffff)
    assert code(apply(rows(**many), weight(n_rows=1 << 20), y=1 << 42, ldy=1 << 20)) == SHAPE
    assert apply(rows(n_rows=0, codes=0, scales=0), weight(), y=0) == OK
    assert code(MX._lib().lora_mx_workspace_bytes(C.byref(rows()), C.byref(weight()), None)) == ARG


@pytest.mark.parametrize("n,h,h_out", [(1, 4096, 4096), (64, 8192, 28672), (40, 28672, 8192), (2048, 8192, 8192), (256, 65536, 128)])
def test_product_workspaces(n, h, h_out):
    """None to speak of, or whole sums of 2 to 8 ranges; a byte less is refused."""
    x = rows(n_rows=n, h=h, ld_codes=h, ld_scales=h // 32)
    w = weight(n_rows=h_out, h=h, ld_codes=h // 2, ld_scales=h // 32)
    b = C.c_size_t()
    assert MX._lib().lora_mx_workspace_bytes(C.byref(x), C.byref(w), C.byref(b)) == OK
    assert b.value == 16 or b.value in [4 * s * n * h_out for s in range(2, 9)]
    assert code(apply(x, w, y=64 * GB, ldy=h_out, ws=32 * GB, ws_bytes=b.value - 1)) == WS


def sample(logits=GB, ld=1000, dtype=L.LORA_BF16, n=3, v=1000, par=None, u=2 * GB, tokens=3 * GB, probs=4 * GB, ws=5 * GB,
           ws_bytes=1 << 24):
    return SA._lib().lora_sample(logits, ld, dtype, n, v, par and C.byref(par), u, tokens, probs, ws, ws_bytes, None)


def params(**kw):
    return SA._Params(**dict(dict(temperature=6 * GB, top_k=7 * GB, top_p=8 * GB, min_p=9 * GB), **kw))


BAD_SAMPLE = [(dict(n=-1), ARG), (dict(v=0), SHAPE), (dict(v=(1 << 19) + 1, ld=1 << 20), SHAPE), (dict(dtype=3), ARG),
              (dict(dtype=-1), ARG), (dict(ld=999), SHAPE), (dict(ld=2 * BIG), SHAPE), (dict(logits=0), ARG), (dict(u=0), ARG),
              (dict(tokens=0), ARG), (dict(logits=GB + 1), ALIGN), (dict(logits=GB + 2, dtype=MX.LORA_F32), ALIGN),
              (dict(u=2 * GB + 2), ALIGN), (dict(tokens=3 * GB + 1), ALIGN), (dict(probs=4 * GB + 2), ALIGN), (dict(ws=0), WS),
              (dict(ws_bytes=15), WS), (dict(ws=5 * GB + 8), ALIGN), (dict(tokens=GB), OVERLAP),
              (dict(tokens=GB + 2 * 2999 - 2), OVERLAP), (dict(probs=2 * GB + 8), OVERLAP), (dict(tokens=4 * GB), OVERLAP),
              (dict(ws=GB), OVERLAP), (dict(ws=3 * GB), OVERLAP)]


@pytest.mark.parametrize("bad,want", BAD_SAMPLE)
def test_bad_samples(bad, want):
    assert code(sample(**bad)) == want
    assert code(sample(par=params(), **bad)) == want


def test_bad_parameters_and_workspaces():
    for k in ("temperature", "top_k", "top_p", "min_p"):
        assert code(sample(par=params(**{k: 12 * GB + 2}))) == ALIGN
        for out in (3 * GB, 4 * GB + 8, 5 * GB + 12):
            assert code(sample(par=params(**{k: out}))) == OVERLAP
    assert sample(n=0, logits=0, u=0, tokens=0, probs=0) == OK
    b = C.c_size_t()
    for n, v in ((0, 1), (1, 1), (1, 50257), (7, 128000), (64, 1 << 19), (100000, 32000)):
        assert SA._lib().lora_sample_workspace_bytes(n, v, L.LORA_F16, C.byref(b)) == OK and b.value >= 16
        assert b.value % 16 == 0
        assert code(sample(n=n, v=v, ld=v, logits=64 * GB, ws_bytes=b.value - 1)) == WS
    assert code(SA._lib().lora_sample_workspace_bytes(1, 10, L.LORA_F16, None)) == ARG


def test_descriptions_are_checked():
    torch = pytest.importorskip("torch")
    u8 = dict(dtype=torch.uint8)
    c, s = torch.zeros((3, 160), **u8), torch.zeros((3, 8), **u8)
    MX.Rows(c, s, MX.LORA_E4M3, 136)
    for bad in ((c.float(), s), (c, s.int()), (c[0], s), (c.t(), s), (c[:2], s), (c[:, :128], s), (c, s[:, :4]),
                (torch.zeros((160, 3), **u8).t(), s)):
        with pytest.raises(ValueError):
            MX.Rows(*bad, MX.LORA_E4M3, 136)
    f, i = torch.ones(3), torch.ones(3, dtype=torch.int32)
    SA.Params(f, i, f, f)
    for bad in ((i,), (None, f), (f.double(),), (None, i.long()), (torch.ones((3, 1)),), (torch.ones(6)[::2],)):
        with pytest.raises(ValueError):
            SA.Params(*bad)


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x, w = MX.empty_rows(2, 64, MX.LORA_E4M3, "cpu"), MX.empty_rows(8, 64, MX.LORA_E2M1, "cpu")
    y = torch.zeros((2, 64), dtype=torch.float16)
    for call in (lambda: MX.lora_norm(y, 64, None, 0, None, 1e-5, 2, 64, L.LORA_F16, None, 0, y, 64, x),
                 lambda: MX.lora_mx_quantize(y, 64, L.LORA_F16, x), lambda: MX.lora_mx_dequantize(x, y, 64, L.LORA_F16),
                 lambda: MX.lora_mx_apply(x, w, y, 8, L.LORA_F16, None, 16)):
        with pytest.raises(ValueError):
            call()
    f, i = torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        SA.lora_sample(y, 64, L.LORA_F16, 2, 64, None, f, i, None, ws, 16)
    with pytest.raises(ValueError):            # parameters of fewer rows
        SA.lora_sample(GB, 64, L.LORA_F16, 3, 64, SA.Params(f), 2 * GB, 3 * GB, 0, 4 * GB, 16)


@pytest.mark.parametrize("which", ["x", "residual", "weight", "total", "y"])
def test_a_norm_of_host_tensors_is_refused(which):
    torch = pytest.importorskip("torch")
    a = dict(x=GB, residual=2 * GB, weight=3 * GB, total=4 * GB, y=5 * GB)
    a[which] = torch.zeros((2, 64), dtype=torch.float16)
    with pytest.raises(ValueError):
        MX.lora_norm(a["x"], 64, a["residual"], 64, a["weight"], 1e-5, 2, 64, L.LORA_F16, a["total"], 64, a["y"], 64)
