"""Paged key-value cache on the host: header and binding agree, the library
exports what the header declares, and bad arguments are refused before any GPU
work (device pointers here are made-up addresses that no call may touch)."""
import ctypes as C
import os
import re

import pytest

from paper_2401_11240_amd import build as B
from paper_2401_11240_amd import kv as KV
from paper_2401_11240_amd import lora as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20            # a 16-byte aligned address


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(B.lib_path()):
        B.build()
    L.load()


def test_header_binding_and_library_agree():
    text = open(os.path.join(ROOT, "include", "lora_kv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"^\s*int\s+(lora_\w+)\s*\(", text, flags=re.M)))
    assert names == sorted(KV.EXPORTS)
    for n in names:
        assert hasattr(L.load(), n), n


def cache(**kw):
    f = dict(k=P, v=P + (1 << 30), layer_stride=1 << 20, page_stride=4096, head_stride=2048, row_stride=128,
             dtype=L.LORA_BF16, n_layers=2, n_pages=10, n_kv_heads=2, page_rows=16, head_dim=128)
    f.update(kw)
    return KV._Cache(**f)


def seqs(**kw):
    f = dict(tables=P, lens=P, n_seqs=3, ld_table=4, max_len=64)
    f.update(kw)
    return KV._Seqs(**f)


def book(**kw):
    f = dict(tables=P, lens=P, refs=P, n_seqs=3, ld_table=4, n_pages=10, page_rows=16)
    f.update(kw)
    return KV._Book(**f)


def code(rc):
    if rc != 0:
        assert L.lora_last_error()
    return rc


BAD_CACHE = [(dict(dtype=2), L.LORA_E_ARG), (dict(n_layers=0), L.LORA_E_ARG), (dict(n_pages=-1), L.LORA_E_ARG),
             (dict(n_kv_heads=0), L.LORA_E_ARG), (dict(head_dim=12), L.LORA_E_SHAPE), (dict(head_dim=264), L.LORA_E_SHAPE),
             (dict(head_dim=0), L.LORA_E_SHAPE), (dict(page_rows=8), L.LORA_E_SHAPE), (dict(page_rows=48), L.LORA_E_SHAPE),
             (dict(page_rows=1 << 17), L.LORA_E_SHAPE), (dict(row_stride=132), L.LORA_E_SHAPE),
             (dict(row_stride=64), L.LORA_E_SHAPE), (dict(head_stride=-8), L.LORA_E_SHAPE),
             (dict(page_stride=1 << 62), L.LORA_E_SHAPE), (dict(row_stride=1 << 27), L.LORA_E_SHAPE),
             (dict(k=0), L.LORA_E_ARG), (dict(v=P + 8), L.LORA_E_ALIGN)]


def decode(c, s, attn=P, layer=0, heads=4, q=P, ldq=512, out=P + (1 << 21), ldo=512, scale=0.1, window=0, sinks=0):
    return KV._lib().lora_attn_decode(attn, c and C.byref(c), layer, s and C.byref(s), heads, q, ldq, out, ldo, scale,
                                      window, sinks, None)


def prompt(c, s, attn=P, off=P, rows=9, heads=4, q=P, ldq=512, out=P + (1 << 21), ldo=512, scale=0.1, window=0,
           sinks=0):
    return KV._lib().lora_attn_prompt(attn, C.byref(c), 0, C.byref(s), off, rows, heads, q, ldq, out, ldo, scale, window,
                                      sinks, None)


def append(c, s, layer=0, off=None, rows=3, k=P, ldk=256, v=P, ldv=256):
    return KV._lib().lora_kv_append(C.byref(c), layer, C.byref(s), off, rows, k, ldk, v, ldv, None)


@pytest.mark.parametrize("bad,want", BAD_CACHE)
def test_bad_caches(bad, want):
    c = cache(**bad)
    i = (C.c_int32 * 1)(0)
    j = (C.c_int32 * 1)(1)
    assert code(decode(c, seqs())) == want
    assert code(prompt(c, seqs())) == want
    assert code(append(c, seqs())) == want
    assert code(KV._lib().lora_kv_copy(C.byref(c), 1, i, j, None)) == want
    assert code(KV._lib().lora_kv_fork(C.byref(c), C.byref(book()), 1, i, j, None, P, 1 << 20, None)) == want
    assert code(KV._lib().lora_kv_compact(C.byref(c), C.byref(book()), P, P, None, P, 1 << 20, None)) == want


BAD_SEQS = [(dict(n_seqs=-1), L.LORA_E_ARG), (dict(lens=0), L.LORA_E_ARG), (dict(tables=0), L.LORA_E_ARG),
            (dict(max_len=65), L.LORA_E_SHAPE), (dict(max_len=-1), L.LORA_E_ARG), (dict(ld_table=-1), L.LORA_E_ARG),
            (dict(lens=P + 2), L.LORA_E_ALIGN)]


@pytest.mark.parametrize("bad,want", BAD_SEQS)
def test_bad_sequences(bad, want):
    assert code(decode(cache(), seqs(**bad))) == want
    assert code(prompt(cache(), seqs(**bad))) == want
    assert code(append(cache(), seqs(**bad))) == want


BAD_ATTN = [(dict(attn=None), L.LORA_E_ARG), (dict(heads=0), L.LORA_E_SHAPE), (dict(heads=5), L.LORA_E_SHAPE),
            (dict(heads=1 << 20, ldq=1 << 27, ldo=1 << 27), L.LORA_E_SHAPE),
            (dict(q=None), L.LORA_E_ARG), (dict(out=None), L.LORA_E_ARG), (dict(q=P + 8), L.LORA_E_ALIGN),
            (dict(out=P + (1 << 21) + 2), L.LORA_E_ALIGN), (dict(ldq=504), L.LORA_E_SHAPE), (dict(ldo=516), L.LORA_E_SHAPE),
            (dict(scale=0.0), L.LORA_E_ARG), (dict(scale=-1.0), L.LORA_E_ARG), (dict(scale=float("nan")), L.LORA_E_ARG),
            (dict(scale=float("inf")), L.LORA_E_ARG), (dict(window=-1), L.LORA_E_ARG), (dict(sinks=-1), L.LORA_E_ARG),
            (dict(out=P + 1024), L.LORA_E_OVERLAP), (dict(out=P), L.LORA_E_OVERLAP)]


@pytest.mark.parametrize("bad,want", BAD_ATTN)
def test_bad_attention_arguments(bad, want):
    assert code(decode(cache(), seqs(), **bad)) == want
    assert code(prompt(cache(), seqs(), **bad)) == want


def test_other_bad_arguments():
    assert code(decode(None, seqs())) == L.LORA_E_ARG
    assert code(decode(cache(), None)) == L.LORA_E_ARG
    assert code(decode(cache(), seqs(), layer=2)) == L.LORA_E_INDEX
    assert code(decode(cache(), seqs(), layer=-1)) == L.LORA_E_INDEX
    assert code(prompt(cache(), seqs(), off=None)) == L.LORA_E_ARG
    assert code(prompt(cache(), seqs(), off=P + 2)) == L.LORA_E_ALIGN
    assert code(prompt(cache(), seqs(), rows=-1)) == L.LORA_E_ARG
    assert code(append(cache(), seqs(), rows=2)) == L.LORA_E_SHAPE
    assert code(append(cache(), seqs(), off=P, rows=-2)) == L.LORA_E_ARG
    assert code(append(cache(), seqs(), layer=5)) == L.LORA_E_INDEX
    assert code(append(cache(), seqs(), k=None)) == L.LORA_E_ARG
    assert code(append(cache(), seqs(), v=P + 4)) == L.LORA_E_ALIGN
    assert code(append(cache(), seqs(), ldk=248)) == L.LORA_E_SHAPE
    assert code(append(cache(), seqs(), ldv=260)) == L.LORA_E_SHAPE
    lib = KV._lib()
    assert code(lib.lora_attn_create(None, 0, None)) == L.LORA_E_ARG
    out = C.c_void_p(5)
    assert code(lib.lora_attn_create(C.byref(out), -1, None)) == L.LORA_E_ARG and not out.value
    assert code(lib.lora_attn_destroy(None)) == L.LORA_E_ARG


def arr(*v):
    return (C.c_int32 * max(1, len(v)))(*v)


def test_bad_book_arguments():
    lib = KV._lib()
    n = C.c_size_t()
    ref = C.byref
    for bad, want in [(dict(page_rows=17), L.LORA_E_SHAPE), (dict(n_pages=-1), L.LORA_E_ARG), (dict(refs=0), L.LORA_E_ARG),
                      (dict(tables=0), L.LORA_E_ARG), (dict(lens=P + 1), L.LORA_E_ALIGN)]:
        b = book(**bad)
        assert code(lib.lora_kv_workspace_bytes(ref(b), ref(n))) == want
        assert code(lib.lora_kv_grow(ref(b), P, None, P, 1 << 20, None)) == want
        assert code(lib.lora_kv_free(ref(b), 1, arr(0), None)) == want
        assert code(lib.lora_kv_trim(ref(b), 5, 0, None)) == want
    b, c = book(), cache()
    assert lib.lora_kv_workspace_bytes(ref(b), ref(n)) == 0 and n.value > 0
    assert code(lib.lora_kv_workspace_bytes(None, ref(n))) == L.LORA_E_ARG
    assert code(lib.lora_kv_workspace_bytes(ref(b), None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_grow(ref(b), None, None, P, 1 << 20, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_grow(ref(b), P, None, None, 1 << 20, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_grow(ref(b), P, None, P + 8, 1 << 20, None)) == L.LORA_E_ALIGN
    assert code(lib.lora_kv_grow(ref(b), P, None, P, n.value - 1, None)) == L.LORA_E_WORKSPACE
    assert code(lib.lora_kv_grow(ref(b), P + 2, None, P, 1 << 20, None)) == L.LORA_E_ALIGN
    assert code(lib.lora_kv_grow(ref(b), P, P + 1, P, 1 << 20, None)) == L.LORA_E_ALIGN
    fork = lambda ps, cs, bb=b, cc=c: code(lib.lora_kv_fork(ref(cc), ref(bb), len(ps), arr(*ps), arr(*cs), None, P,
                                                            1 << 20, None))
    assert fork([0], [3]) == L.LORA_E_INDEX
    assert fork([-1], [1]) == L.LORA_E_INDEX
    assert fork([0, 0], [1, 1]) == L.LORA_E_ARG
    assert fork([0, 1], [1, 2]) == L.LORA_E_ARG
    assert fork([0], [1], bb=book(page_rows=32)) == L.LORA_E_SHAPE
    assert fork([0], [1], bb=book(n_pages=11)) == L.LORA_E_SHAPE
    assert code(lib.lora_kv_fork(ref(c), ref(b), -1, None, None, None, P, 1 << 20, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_fork(ref(c), ref(b), 1, None, arr(1), None, P, 1 << 20, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_fork(ref(c), ref(b), 1, arr(0), arr(1), None, P, 8, None)) == L.LORA_E_WORKSPACE
    assert code(lib.lora_kv_free(ref(b), 2, arr(1, 1), None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_free(ref(b), 1, arr(3), None)) == L.LORA_E_INDEX
    assert code(lib.lora_kv_free(ref(b), -1, None, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_free(ref(b), 1, None, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_trim(ref(b), 0, 0, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_trim(ref(b), 1, -1, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_copy(ref(c), 1, arr(10), arr(0), None)) == L.LORA_E_INDEX
    assert code(lib.lora_kv_copy(ref(c), 2, arr(0, 1), arr(5, 5), None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_copy(ref(c), 2, arr(0, 1), arr(1, 2), None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_compact(ref(c), ref(b), None, P, None, P, 1 << 20, None)) == L.LORA_E_ARG
    assert code(lib.lora_kv_compact(ref(c), ref(b), P, P + 2, None, P, 1 << 20, None)) == L.LORA_E_ALIGN
    assert code(lib.lora_kv_compact(ref(c), ref(b), P, P, None, P, 8, None)) == L.LORA_E_WORKSPACE


def test_tensor_descriptions_are_checked():
    torch = pytest.importorskip("torch")
    k = torch.zeros((1, 2, 2, 16, 8), dtype=torch.float16)
    KV.Cache(k, k.clone())
    for bad in (k.float(), k[:, :1], k.transpose(2, 3).contiguous().transpose(2, 3), k[0]):
        with pytest.raises(ValueError):
            KV.Cache(k, bad)
    with pytest.raises(ValueError):
        KV.Cache(k.float(), k.float())
    t, n = torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    KV.Seqs(t, n, 5), KV.Book(t, n, n, 16)
    for bt, bn in ((t.long(), n), (t[:, :3], n), (t, n[:2]), (t[0], n), (t, n.float())):
        with pytest.raises(ValueError):
            KV.Seqs(bt, bn, 5)
        with pytest.raises(ValueError):
            KV.Book(bt, bn, n, 16)


def test_loads_into_lds_wait_for_their_scalar_registers():
    # a buffer load needs 5 wait states after a vector instruction that wrote one of
    # its scalar registers; inside a statement only the statement itself leaves them
    path = os.path.join(ROOT, "paper_2401_11240_amd", "csrc", "lora_attn.hip")
    stmts = [m for m in re.findall(r'asm volatile\("([^"]*)"', open(path).read()) if "buffer_load" in m]
    assert stmts
    for stmt in stmts:
        before = stmt[:stmt.index("buffer_load")]
        assert sum(int(n) + 1 for n in re.findall(r"s_nop (\d+)", before)) >= 5, stmt


def test_sizes_past_32_bits_are_refused():
    lib = KV._lib()
    b = book(n_seqs=1 << 16, ld_table=1 << 15)
    assert code(lib.lora_kv_free(C.byref(b), 0, None, None)) == L.LORA_E_SHAPE
    s = seqs(ld_table=1 << 27, max_len=(1 << 30) + 1)
    assert code(lib.lora_kv_append(C.byref(cache()), 0, C.byref(s), None, 3, P, 256, P, 256, None)) == L.LORA_E_SHAPE
    b = book(n_pages=(1 << 30) + 1)
    assert code(lib.lora_kv_free(C.byref(b), 0, None, None)) == L.LORA_E_SHAPE
    s = seqs(n_seqs=(1 << 31) - 1, ld_table=1, max_len=16)
    c = cache(n_kv_heads=1, head_dim=128)
    rows = (1 << 31) - 1
    assert code(lib.lora_kv_append(C.byref(c), 0, C.byref(s), None, rows, P, 128, P, 128, None)) == L.LORA_E_SHAPE
