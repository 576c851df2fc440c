"""Bad arguments of the calls that carry step lengths are refused before any GPU
work (device pointers here are made-up addresses that no call may touch)."""
import ctypes as C
import os

import pytest

from paper_2401_11240_amd import build as B
from paper_2401_11240_amd import kv as KV
from paper_2401_11240_amd import lora as L
from test_kv_cpu import P, arr, book, cache, code


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(B.lib_path()):
        B.build()
    L.load()


def grow(b, add=P, max_len=64, step=P + 4096, info=None, ws=P, n=1 << 20):
    return code(KV._lib().lora_kv_grow_step(b and C.byref(b), add, max_len, step, info, ws, n, None))


def fork(b, step=P + 4096, parents=(0,), children=(1,)):
    return code(KV._lib().lora_kv_fork_step(C.byref(cache()), C.byref(b), len(parents), arr(*parents), arr(*children), step,
                                            None, P, 1 << 20, None))


def test_step_lengths_are_checked():
    assert grow(None) == L.LORA_E_ARG
    assert grow(book(page_rows=17)) == L.LORA_E_SHAPE
    assert grow(book(), step=None) == L.LORA_E_ARG
    assert grow(book(), step=P + 4098) == L.LORA_E_ALIGN
    for at in (P, P + 8, P - 8):                     # lens is [P, P + 12)
        assert grow(book(), step=at) == L.LORA_E_OVERLAP
        assert fork(book(), step=at) == L.LORA_E_OVERLAP
    assert grow(book(), max_len=-1) == L.LORA_E_ARG
    assert grow(book(), max_len=65) == L.LORA_E_SHAPE
    assert grow(book(), add=None) == L.LORA_E_ARG
    assert grow(book(), add=P + 2) == L.LORA_E_ALIGN
    assert grow(book(), info=P + 2) == L.LORA_E_ALIGN
    assert grow(book(), ws=None) == L.LORA_E_ARG
    assert grow(book(), n=8) == L.LORA_E_WORKSPACE
    assert fork(book(), step=None) == L.LORA_E_ARG
    assert fork(book(), step=P + 4097) == L.LORA_E_ALIGN
    assert fork(book(), parents=(0,), children=(3,)) == L.LORA_E_INDEX
    assert fork(book(), parents=(0, 1), children=(1, 2)) == L.LORA_E_ARG
    assert fork(book(page_rows=32)) == L.LORA_E_SHAPE


def test_tensors_on_the_host_and_arrays_of_other_types_are_refused():
    # nothing is launched: every call raises before it reaches the library
    torch = pytest.importorskip("torch")
    i32 = dict(dtype=torch.int32)
    k = torch.zeros((1, 4, 2, 16, 8), dtype=torch.float16)
    c = KV.Cache(k, k.clone())
    tables, lens, refs, info = (torch.zeros(n, **i32) for n in ((3, 4), 3, 4, 2))
    seqs, book = KV.Seqs(tables, lens, 64), KV.Book(tables, lens, refs, 16)
    ws = torch.zeros(1 << 10, dtype=torch.uint8)
    off, q = torch.zeros(4, **i32), torch.zeros((3, 16), dtype=torch.float16)
    calls = [lambda: KV.lora_kv_append(c, 0, seqs, off, 3, q, 16, q, 16), lambda: KV.lora_kv_grow(book, lens, info, ws, 1024),
             lambda: KV.lora_attn_decode(1, c, 0, seqs, 2, q, 16, q, 16, 1.0),
             lambda: KV.lora_attn_prompt(1, c, 0, seqs, off, 3, 2, q, 16, q, 16, 1.0),
             lambda: KV.lora_kv_grow_step(book, lens, 64, lens.clone(), info, ws, 1024),
             lambda: KV.lora_kv_fork(c, book, [0], [1], info, ws, 1024),
             lambda: KV.lora_kv_fork_step(c, book, [0], [1], lens.clone(), info, ws, 1024),
             lambda: KV.lora_kv_free(book, [0]), lambda: KV.lora_kv_trim(book, 4), lambda: KV.lora_kv_copy(c, [0], [1]),
             lambda: KV.lora_kv_compact(c, book, tables, refs, info, ws, 1024)]
    for call in calls:
        with pytest.raises(ValueError, match="device tensors"):
            call()
    meta = torch.zeros(3, device="meta", **i32)
    for make in (lambda: KV.Seqs(tables, meta, 64), lambda: KV.Book(tables, lens, meta, 16),
                 lambda: KV.Cache(k, k.to("meta"))):
        with pytest.raises(ValueError, match="one device"):
            make()
    assert KV._words("add", lens, 3, book) == lens.data_ptr() and KV._words("add", None, 3, book) == 0
    assert KV._words("add", P, 3, book) == P and KV._space(ws, 1024, book) == ws.data_ptr()
    for bad in (lens.long(), lens.float(), lens.short(), lens[:2], torch.zeros(6, **i32)[::2], meta):
        with pytest.raises(ValueError, match="add"):
            KV._words("add", bad, 3, book)
    for bad in (ws[:1023], torch.zeros(2048, dtype=torch.uint8)[::2], ws.to("meta")):
        with pytest.raises(ValueError, match="ws"):
            KV._space(bad, 1024, book)
