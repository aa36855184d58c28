"""What the score kernels rely on in how a choice of blocks is cut (shape_model.cpp)."""
from __future__ import annotations

import ctypes as C
import os
import random
import subprocess

from tests import test_order_cpu as O


def test_shapes(tmp_path):
    with open(os.path.join(O.CSRC, "select_blocks.cu")) as f:
        text = f.read()
    (tmp_path / "shape.inc").write_text(text[text.index("static size_t score_smem"):text.index("template <int HP, int THREADS>\nstatic cudaError_t score_go")])
    so = str(tmp_path / "libshape.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", os.path.join(O.ROOT, "include"), "-I", O.CSRC, "-I",
                           os.path.join(O.CUDA, "include"), f'-DSHAPE_SOURCE="{tmp_path / "shape.inc"}"', os.path.join(O.ROOT, "tests", "shape_model.cpp"),
                           "-o", so])
    lib = C.CDLL(so)
    lib.shape_of.argtypes = [C.c_int] * 5 + [C.c_longlong, C.c_int, C.POINTER(C.c_longlong)]
    rng, out, seen = random.Random(3), (C.c_longlong * 10)(), set()
    for _ in range(20000):
        H, G, D = rng.choice([1, 2, 3, 4, 5, 8, 13, 16, 17, 40]), rng.choice([1, 2, 3, 4, 7, 8, 16, 31, 33, 64, 100, 200]), 8 * rng.randint(1, 32)
        n = int(2 ** rng.uniform(0, 10))
        max_nq = rng.choice([1, 1, int(2 ** rng.uniform(0, 16))])
        lib.shape_of(H, G, D, n, max_nq, n * int(2 ** rng.uniform(0, 30 if max_nq > 1 else 20)), rng.choice([148, 20]), out)
        tile, heads, cols, slabs, reps, buffers, together, blocks, smem, most = out
        assert buffers == (2 if reps > 1 else 1)  # the next m-tile's codes go into the other buffer
        assert 1 <= reps <= 1 << 16 and reps * blocks <= 1 << 23
        assert smem <= most <= 227 * 1024 and 128 * slabs >= 2 * D
        assert cols in (32, 64, 128) and heads >= G and (heads % 32 == 0 or heads in (1, 2, 4, 8, 16))
        assert tile == 1 or tile * heads <= cols  # larger groups go through the rows in passes
        if together:
            assert max_nq == 1 and H * heads <= cols and H * blocks <= 128 and heads <= 32 and blocks >= 8
            # a warp's 32 rows of sums lie within 32 columns
            assert max(1, 32 // blocks) * heads <= 32
        else:
            assert blocks == 128
        seen.add((buffers, together, cols))
    assert len(seen) == 9  # whole records (together) are for many m-tiles, so with two buffers
