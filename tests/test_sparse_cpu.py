"""Host side of sparse attention and of a batch's tables, without a device: struct layouts, refusals, and the order of the calls across
streams, on the model of the CUDA runtime (sparse_model.cpp)."""
from __future__ import annotations

import ctypes as C
import os
import subprocess

import pytest

import __graft_entry__ as entry
from paper_2607_10987_b200 import binding as B
from tests import test_order_cpu as O

INVALID, INCOMPAT, SMALL, CUDA = B.AAF_ERR_INVALID_ARG, B.AAF_ERR_INCOMPAT, B.AAF_ERR_DST_TOO_SMALL, B.AAF_ERR_CUDA


def test_struct_sizes_match_the_header():
    assert C.sizeof(B.aaf_kv_select_desc) == 32 and C.sizeof(B.aaf_kv_batch_desc) == 64


def test_null_pool_is_rejected():
    entry.build()
    one = (C.c_int32 * 1)(0)
    assert B.aaf_kv_summary_bytes(None) == 0
    assert B.aaf_kv_summarize(None, 0, 0, 1, one, None, None, 0, None) == INVALID
    assert B.aaf_kv_select(None, 0, None, 1, one, None, None, None, 0, None, None, None, 0, None) == INVALID
    assert B.aaf_kv_attend_blocks(None, 0, None, 1, one, None, None, None, 1, None, None, None, 0, None) == INVALID
    assert B.aaf_kv_batch_tables(None, None, 1, one, None, None) == INVALID


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("sparse") / "libsparse.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(O.ROOT, "include"), "-I", O.CSRC,
                           "-I", os.path.join(O.CUDA, "include"), "-x", "c++", os.path.join(O.CSRC, "pool.cu"), os.path.join(O.CSRC, "sparse.cu"),
                           os.path.join(O.ROOT, "tests", "sparse_model.cpp"), "-o", out])
    lib = C.CDLL(out)
    for name, (res, args) in B.SYMBOLS.items():
        if hasattr(lib, name):
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args
    for name in ("order_stream", "order_replace_stream", "order_where"):
        getattr(lib, name).restype = C.c_void_p
    for name in ("order_name", "order_wrong"):
        getattr(lib, name).restype = C.c_char_p
    lib.order_replace_stream.argtypes = [C.c_void_p, C.c_int]
    lib.order_capture.argtypes = [C.c_void_p, C.c_int]
    lib.order_fail.argtypes = [C.c_char_p, C.c_int]
    return lib


class Pool(O.Pool):
    def summarize(self, st, ctxs, n_new=None, want=0, layer=0, dtype=0, room=1 << 40, at=None):
        return self.call("summarize", layer, dtype, len(ctxs), self.ints(ctxs), None if n_new is None else self.ints(n_new),
                         self.base if at is None else at, room, st, want=want)

    def select(self, st, ctxs, n_q=None, want=0, layer=0, summary_room=1 << 40, room=1 << 40, **kw):
        d = dict(struct_size=C.sizeof(B.aaf_kv_select_desc), dtype=0, n_q_heads=O.H, keep=4, sink=1, recent=1, q_stride=O.H * O.D)
        p = {k: kw.pop(k, self.base) for k in ("q", "summary", "blocks", "scores", "ws")}
        d.update(kw)
        return self.call("select", layer, C.byref(B.aaf_kv_select_desc(**d)), len(ctxs), self.ints(ctxs), None if n_q is None else self.ints(n_q),
                         p["q"], p["summary"], summary_room, p["blocks"], p["scores"], p["ws"], room, st, want=want)

    def attend_blocks(self, st, ctxs, n_q=None, want=0, layer=0, keep=4, room=1 << 40, blocks=0, out=0, heads=O.H):
        return self.call("attend_blocks", layer, C.byref(self._attn(heads)), len(ctxs), self.ints(ctxs), None if n_q is None else self.ints(n_q),
                         self.base, blocks or self.base, keep, out or self.base, None, self.base, room, st, want=want)

    def tables(self, st, ctxs, n_new=None, want=0, **kw):
        d = dict(struct_size=C.sizeof(B.aaf_kv_batch_desc), rows=40, tokens=4000, cols=O.BLK, tables=self.base, lens=None, offsets=None,
                 token_row=None, positions=None, slots=None)
        d.update(kw)
        return self.call("batch_tables", C.byref(B.aaf_kv_batch_desc(**d)), len(ctxs), self.ints(ctxs), None if n_new is None else self.ints(n_new),
                         st, want=want)


@pytest.fixture
def pool(lib):
    p = Pool(lib)
    yield p
    p.close()


CALLS = {"summarize": lambda p, s, c, **kw: p.summarize(s, [c], **kw), "choose": lambda p, s, c, **kw: p.select(s, [c], **kw),
         "attend_blocks": lambda p, s, c, **kw: p.attend_blocks(s, [c], **kw), "tables": lambda p, s, c, **kw: p.tables(s, [c], **kw)}


def test_summary_sizes(lib, pool):
    record = O.H * 2 * O.D + 16
    assert lib.aaf_kv_summary_bytes(pool.h) == O.L * O.NB * record
    st = lib.order_stream()
    _, c = pool.imp(st, 160)
    assert pool.summarize(st, [c], room=O.L * O.NB * record)
    assert not pool.summarize(st, [c], room=O.L * O.NB * record - 1, want=SMALL)
    assert pool.select(st, [c], summary_room=O.L * O.NB * record)
    assert not pool.select(st, [c], summary_room=O.L * O.NB * record - 1, want=SMALL)


def test_refusals(lib, pool):
    st = lib.order_stream()
    _, c = pool.imp(st, 160)
    at = lib.order_ops()
    for kw in (dict(layer=-2), dict(layer=O.L), dict(dtype=2), dict(at=pool.base + 8), dict(n_new=[0]), dict(n_new=[161])):
        assert not pool.summarize(st, [c], want=INVALID, **kw)
    for kw in (dict(layer=-1), dict(layer=O.L), dict(dtype=-1), dict(n_q_heads=0), dict(n_q_heads=3), dict(keep=0), dict(keep=B.AAF_LIST_MAX_BLOCKS + 1),
               dict(sink=-1), dict(recent=0), dict(keep=3, sink=2, recent=2), dict(recent=2147483647, sink=2147483647), dict(q_stride=O.H * O.D - 8),
               dict(q_stride=O.H * O.D + 4), dict(q=pool.base + 2), dict(summary=None), dict(blocks=None), dict(blocks=pool.base + 2),
               dict(scores=pool.base + 1), dict(ws=pool.base + 4), dict(struct_size=31), dict(n_q=[0]), dict(n_q=[161])):
        assert not pool.select(st, [c], want=INVALID, **kw), kw
    assert not pool.select(st, [c], room=lib.aaf_kv_attend_workspace_bytes(pool.h) - 1, want=SMALL)
    for kw in (dict(layer=-1), dict(layer=O.L), dict(keep=0), dict(keep=B.AAF_LIST_MAX_BLOCKS + 1), dict(blocks=pool.base + 2), dict(out=pool.base + 8),
               dict(n_q=[0]), dict(n_q=[161]), dict(heads=3)):
        assert not pool.attend_blocks(st, [c], want=INVALID, **kw), kw
    assert not pool.attend_blocks(st, [c], room=lib.aaf_kv_attend_workspace_bytes(pool.h) - 1, want=SMALL)
    for kw in (dict(tables=None), dict(tables=pool.base + 2), dict(slots=pool.base + 4), dict(n_new=[0]), dict(n_new=[161]), dict(struct_size=8)):
        assert not pool.tables(st, [c], want=INVALID, **kw), kw
    for kw in (dict(rows=0), dict(rows=-5), dict(tokens=0), dict(cols=9), dict(cols=-1)):
        assert not pool.tables(st, [c], want=SMALL, **kw), kw
    assert pool.tables(st, [c], cols=0, tables=None, lens=pool.base)
    for name, call in CALLS.items():
        assert not call(pool, st, c + 1, want=B.AAF_ERR_BAD_CTX)
        assert not call(pool, st, -1, want=B.AAF_ERR_BAD_CTX)
    assert lib.order_ops() == at + 1


def test_tables_beyond_the_kernels_ints_are_refused(lib, pool):
    st = lib.order_stream()
    _, c = pool.imp(st, 160)
    for kw in (dict(cols=(1 << 30) + 1), dict(cols=(1 << 31) - 1), dict(cols=(1 << 31) - 1, rows=1), dict(rows=(1 << 30) + 1), dict(tokens=(1 << 31) - 1)):
        assert not pool.tables(st, [c], want=B.AAF_ERR_TOO_MANY, **kw), kw
    assert pool.tables(st, [c], cols=1 << 30, rows=1)
    assert pool.tables(st, [c], cols=(1 << 31) - 1, tables=None, lens=pool.base)  # not looked at


@pytest.mark.parametrize("call", CALLS)
def test_refused_in_a_capture_and_beside_one_not(lib, pool, call):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    lib.order_capture(a, 1)
    assert not CALLS[call](pool, a, c, want=INVALID)
    assert CALLS[call](pool, b, c)
    assert not pool.wrongs()


@pytest.mark.parametrize("call", CALLS)
def test_order_behind_payload_work_and_metadata_on_other_streams(lib, pool, call):
    a, b = lib.order_stream(), lib.order_stream()
    ran, c = pool.imp(a, 160)
    mine = CALLS[call](pool, b, c)[call]
    assert pool.before(ran["copy"], mine) and pool.before(ran["plan_import"], mine)
    for name, other in CALLS.items():
        d = lib.order_stream()
        theirs = other(pool, d, c)[name]
        assert pool.before(mine, theirs)
        mine = theirs
    assert pool.before(mine, pool.append(a, [c], [5])["copy"])


@pytest.mark.parametrize("writer", O.ROW_WRITERS)
@pytest.mark.parametrize("call", CALLS)
def test_a_table_row_is_rewritten_behind_its_readers(lib, pool, call, writer):
    a, b = lib.order_stream(), lib.order_stream()
    _, old = pool.imp(b, 160)
    _, read = pool.imp(b, 160)
    seen = [CALLS[call](pool, a, c)[call] for c in (old, read)]
    pool.evict(b, [old])
    ran = O.ROW_WRITERS[writer](pool, b, read, 0)
    plan = [i for name, i in ran.items() if name.startswith("plan_") or name == "fork"]
    assert len(plan) == 1 and all(pool.before(s, plan[0]) for s in seen)


@pytest.mark.parametrize("call", CALLS)
def test_the_stream_may_go_once_a_call_on_another_has_returned(lib, pool, call):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    mine = CALLS[call](pool, a, c)[call]
    pool.attend(b, [c])
    lib.order_replace_stream(a, 0)
    O.every_call(pool, b, c)
    pool.close()
    pool.h = None
    assert lib.order_host_knows(mine)
    assert not pool.wrongs()


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("what", ["cudaEventRecord", "cudaStreamWaitEvent", "launch"])
def test_a_failure_leaves_the_pool_unusable(lib, pool, call, what):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(a, 160)
    lib.order_fail((call if what == "launch" else what).encode(), 1)
    CALLS[call](pool, b, c, want=CUDA)
    for other in CALLS.values():
        assert not other(pool, b, c, want=CUDA)


def test_large_batches_go_through_the_pinned_ring(lib, pool):
    st = lib.order_stream()
    _, c = pool.imp(st, 160)
    for call in (pool.summarize, pool.select, pool.attend_blocks):
        assert "memcpy" not in call(st, [c] * 64) and "memcpy" in call(st, [c] * 65)
    assert "memcpy" not in pool.tables(st, [c] * 512, rows=600) and "memcpy" in pool.tables(st, [c] * 513, rows=600)
    for call in (pool.summarize, pool.select, pool.attend_blocks):
        assert not call(st, [c] * 1025, want=B.AAF_ERR_TOO_MANY)


def test_a_choice_for_more_tokens_than_the_workspace_holds_scores_of(lib, pool):
    st = lib.order_stream()
    _, c = pool.imp(st, 16 * (O.BLK - 1))
    at_once = 65536 * (O.D + 2) // ((O.BLK - 1 + 3) // 4 * 4 * O.H)
    for tokens, launches in ((at_once, 1), (at_once + 1, 2), (3 * at_once, 3)):
        first = lib.order_ops()
        pool.select(st, [c, c], [tokens - 1, 1])
        assert lib.order_ops() - first == launches
    first = lib.order_ops()  # a launch takes no more records than the workspace of the pool has room for
    pool.select(st, [c] * 1024, [1] * 1024)
    names = [lib.order_name(i) for i in range(first, lib.order_ops())]
    assert names.count(b"choose") == -(-1024 // at_once)
