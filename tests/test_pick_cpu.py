"""The selection of blocks from their scores, thread by thread on the CPU (pick_model.cpp): the lists, and what becomes of scores that are
void because a wait ran out before they were written."""
from __future__ import annotations

import os
import re
import subprocess

import numpy as np
import pytest

from tests import test_order_cpu as O


@pytest.fixture(scope="module")
def pick(tmp_path_factory):
    at = tmp_path_factory.mktemp("pick")
    with open(os.path.join(O.CSRC, "select_blocks.cu")) as f:
        text = f.read()
    text = text[text.index("constexpr int PICK_FEW"):text.index("static size_t score_smem")]
    text = re.sub(r"extern __shared__ [^;]* keys_s\[\];", "uint32_t *const keys_s = shared_keys;", text)
    text = re.sub(r"asm volatile\([^;]*griddepcontrol[^;]*;[^;]*;", "", text)
    assert "asm" not in text
    (at / "pick.inc").write_text(text)
    subprocess.check_call(["g++", "-std=c++20", "-O1", "-g", "-fsanitize=address", "-static-libasan", "-pthread", "-I", os.path.join(O.CUDA, "include"),
                           f'-DPICK_SOURCE="{at / "pick.inc"}"', os.path.join(O.ROOT, "tests", "pick_model.cpp"), "-o", str(at / "pick")])

    env = {k: v for k, v in os.environ.items() if k != "LD_PRELOAD"}  # the sanitizer wants to be loaded first
    env["ASAN_OPTIONS"] = "detect_leaks=0"

    def run(keys, keep, sink, recent, warps=4, stay=True):
        keys = np.ascontiguousarray(keys, dtype=np.uint32)
        room = (len(keys) + 3) // 4 * 4 if stay else 0
        done = subprocess.run([str(at / "pick"), *map(str, (warps, len(keys), keep, sink, recent, room))], input=keys.tobytes(), capture_output=True,
                              timeout=120, env=env)
        assert done.returncode == 0, done.stderr.decode()[-3000:]
        return np.frombuffer(done.stdout, dtype=np.int32).tolist()

    return run


def chosen(keys, keep, sink, recent):
    n = len(keys)
    if n <= keep:
        return list(range(n)) + [-1] * (keep - n)
    forced = [b for b in range(n) if b < sink or b >= n - recent]
    rest = sorted(range(sink, n - recent), key=lambda b: (-int(keys[b]), b))
    return sorted(forced + rest[:keep - len(forced)])


def scores(kind, n, rng):
    if kind == "spread":
        return rng.integers(1, 1 << 32, n, dtype=np.uint64)
    if kind == "near":  # a few values, many times each
        return 0x80000000 + rng.integers(0, 7, n)
    return 0xbf800000 + rng.integers(0, 1 << 22, n) // (1 + (rng.random(n) < 0.5) * (1 << 20))


@pytest.mark.parametrize("kind", ["spread", "near", "lumps"])
@pytest.mark.parametrize("n,keep,sink,recent", [(2000, 64, 1, 4), (2000, 1500, 3, 7), (130, 8, 0, 1), (5, 8, 1, 1), (1031, 5, 1, 4)])
def test_lists(pick, kind, n, keep, sink, recent):
    keys = scores(kind, n, np.random.default_rng(n + keep))
    for warps, stay in ((4, True), (8, False)):
        assert pick(keys, keep, sink, recent, warps, stay) == chosen(keys, keep, sink, recent)


@pytest.mark.parametrize("stay", [True, False])
@pytest.mark.parametrize("kind", ["fewer scores than wanted", "fewer, in one part", "none", "one", "anything"])
def test_void_scores_stay_within_the_list(pick, kind, stay):
    n, keep, sink, recent = 2000, 1500, 1, 4
    rng = np.random.default_rng(5)
    keys = np.zeros(n, dtype=np.uint64)
    if kind.startswith("fewer"):
        keys[::2] = rng.integers(0x90000000, 0xb0000000, n // 2)
        if "part" in kind:  # 256 parts from the smallest to the largest: most scores in the ninth from above
            keys[::2] = 0x90000000 + (247 << 16) + 99
            keys[0:8:2] = 0x90000000
            keys[100:108:2] = 0x90ffffff
    elif kind == "one":
        keys[777] = 0xc0000000
    elif kind == "anything":
        keys[:] = rng.integers(0, 1 << 32, n, dtype=np.uint64) * (rng.random(n) < 0.9)
    got = pick(keys, keep, sink, recent, stay=stay)
    assert all(0 <= b < n for b in got) and all(a < b for a, b in zip(got, got[1:]))
