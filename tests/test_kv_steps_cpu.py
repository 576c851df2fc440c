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
