"""A call of sparse attention takes nothing from the host's memory once it has launched something: if it had to give up then, its
launches would be in no order with what comes later."""
from __future__ import annotations

import ctypes as C
import os
import subprocess

import pytest

from paper_2607_10987_b200 import binding as B
from tests import test_order_cpu as O
from tests.test_sparse_cpu import Pool


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("memory") / "libmemory.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(O.ROOT, "include"), "-I", O.CSRC,
                           "-I", os.path.join(O.CUDA, "include"), "-x", "c++", os.path.join(O.CSRC, "pool.cu"), os.path.join(O.CSRC, "sparse.cu"),
                           os.path.join(O.ROOT, "tests", "sparse_alloc_model.cpp"), "-o", out])
    lib = C.CDLL(out)
    for name, (res, args) in B.SYMBOLS.items():
        if hasattr(lib, name):
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args
    lib.order_stream.restype = C.c_void_p
    lib.order_name.restype = C.c_char_p
    return lib


@pytest.mark.parametrize("tokens,launches", [(1, 1), (2, 2), (5, 5)])
def test_a_split_choice_needs_no_memory_behind_its_first_launch(lib, tokens, launches):
    pool = Pool(lib)
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(a, O.BS * (O.BLK - 1))
    lib.order_no_memory_behind_launches(1)
    first = lib.order_ops()
    pool.select(b, [c] * 1024, [tokens] * 1024)
    lib.order_no_memory_behind_launches(0)
    mine = [i for i in range(first, lib.order_ops()) if lib.order_name(i) == b"choose"]
    assert len(mine) == launches
    later = pool.append(a, [c], [5])["copy"]
    assert all(pool.before(m, later) for m in mine)
    pool.close()
