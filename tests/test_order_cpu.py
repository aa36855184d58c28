"""Order of a pool's work across streams, on the CPU: the library's host side (pool.cu) runs on a model of the CUDA runtime
(order_model.cpp) that computes nothing and remembers for every launch what had to be over before it."""
from __future__ import annotations

import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2607_10987_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_10987_b200", "csrc")
CUDA = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
L, H, D, BS, NB, CTX, BLK = 1, 2, 64, 16, 4096, 32, 2048


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("order") / "liborder.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                           "-I", os.path.join(CUDA, "include"), "-x", "c++", os.path.join(CSRC, "pool.cu"),
                           os.path.join(ROOT, "tests", "order_model.cpp"), "-o", out])
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


class Pool:
    """A pool on the model.  Calls take the stream first and return the names and numbers of what they launched."""

    def __init__(self, lib):
        self.lib = lib
        lib.order_reset()
        self.mem = (C.c_char * 4096)()
        base = (C.addressof(self.mem) + 1023) // 1024 * 1024  # nothing is read or written through it
        d = B.make_desc(L, H, D, BS, 2, NB, CTX, BLK, 0, 0, 0, 0)
        size = lib.aaf_kv_pool_workspace_bytes(C.byref(d))
        self.ws = (C.c_char * (size + 256))()
        d.pool_base, d.layer_stride_bytes = base, NB * 2 * BS * H * D * 2
        d.workspace, d.workspace_bytes = (C.addressof(self.ws) + 255) // 256 * 256, size
        self.desc, self.base, self.h = d, base, C.c_void_p()
        assert lib.aaf_kv_pool_create(C.byref(d), C.byref(self.h)) == 0
        self.status = 0

    def close(self):
        self.lib.aaf_kv_pool_destroy(self.h)

    def _ran(self, first, status, want):
        self.status = status
        if want is not None:
            assert status == want, status
        return {self.lib.order_name(i).decode(): i for i in range(first, self.lib.order_ops())}

    def call(self, name, *args, want=0):
        first = self.lib.order_ops()
        return self._ran(first, getattr(self.lib, "aaf_kv_" + name)(self.h, *args), want)

    def ints(self, v):
        return (C.c_int32 * len(v))(*v)

    def imp(self, st, tokens, want=0):
        x = B.aaf_kv_xfer_desc()
        x.n_layers, x.n_kv_heads, x.head_dim, x.elt_bytes, x.n_tokens = L, H, D, 2, tokens
        out = C.c_int32(-1)
        ran = self.call("import", self.base, C.byref(x), C.byref(out), st, want=want)
        return ran, out.value

    def reserve(self, st, ctxs, n_new, want=0):
        return self.call("reserve", len(ctxs), self.ints(ctxs), self.ints(n_new), st, want=want)

    def append(self, st, ctxs, n_new, want=0):
        src = (C.c_void_p * len(ctxs))(*[self.base] * len(ctxs))
        return self.call("append", len(ctxs), self.ints(ctxs), self.ints(n_new), src, st, want=want)

    def fork(self, st, ctx, k=1, want=0):
        out = (C.c_int32 * k)()
        ran = self.call("fork", ctx, k, out, st, want=want)
        return ran, list(out)

    def compose(self, st, ctxs, want=0):
        out = C.c_int32(-1)
        ran = self.call("compose", len(ctxs), self.ints(ctxs), B.AAF_COMPOSE_SHARE, C.byref(out), st, want=want)
        return ran, out.value

    def evict(self, st, ctxs, want=0):
        return self.call("evict", len(ctxs), self.ints(ctxs), st, want=want)

    def materialize(self, st, ctx, tokens, want=0):
        return self.call("materialize", ctx, 0, tokens, self.base, 1 << 40, None, st, want=want)

    def store(self, st, ctxs, n_new, want=0, heads=0, q=None, q_out=None, q_stride=0, q_out_stride=0):
        d = B.aaf_kv_store_desc(C.sizeof(B.aaf_kv_store_desc), 0, heads, 0, 0, 1.0, None, None, q, q_out, self.base, self.base, q_stride, q_out_stride,
                                H * D, H * D)
        return self.call("store", 0, C.byref(d), len(ctxs), self.ints(ctxs), self.ints(n_new), st, want=want)

    def _attn(self, heads=H):
        return B.aaf_kv_attn(C.sizeof(B.aaf_kv_attn), 0, heads, 0, 0.1, 0.0, None, None, heads * D)

    def attend(self, st, ctxs, n_q=None, want=0, heads=H):
        return self.call("attend", 0, C.byref(self._attn(heads)), len(ctxs), self.ints(ctxs), None if n_q is None else self.ints(n_q), self.base,
                         self.base, None, self.base, 1 << 40, st, want=want)

    def mass(self, st, ctxs, want=0, heads=H):
        return self.call("attn_mass", 0, C.byref(self._attn(heads)), len(ctxs), self.ints(ctxs), None, self.base, self.base, None, self.base, 1 << 20, st,
                         want=want)

    def prune(self, st, ctx, budget, want=0):
        out = C.c_int32(-1)
        ran = self.call("prune", ctx, self.base, budget, 0, 0, self.base, None, C.byref(out), st, want=want)
        return ran, out.value

    def before(self, a, b):
        return bool(self.lib.order_before(a, b))

    def wrongs(self):
        return [self.lib.order_wrong(i).decode() for i in range(self.lib.order_wrongs())]


@pytest.fixture
def pool(lib):
    p = Pool(lib)
    yield p
    p.close()


READERS = {"attend": lambda p, s, c: p.attend(s, [c])["attend"], "store": lambda p, s, c: p.store(s, [c], [1])["store"],
           "mass": lambda p, s, c: p.mass(s, [c])["mass"], "prune": lambda p, s, c: p.prune(s, c, 5)[0]["gather"],
           "materialize": lambda p, s, c: p.materialize(s, c, 5)["copy"]}


@pytest.mark.parametrize("reader", READERS)
def test_a_reserve_that_copies_nothing_keeps_the_order_behind_an_import(lib, pool, reader):
    a, b = lib.order_stream(), lib.order_stream()
    ran, c = pool.imp(a, 160)
    assert "copy" not in pool.reserve(b, [c], [16])
    assert pool.before(ran["copy"], READERS[reader](pool, b, c))


@pytest.mark.parametrize("reader", READERS)
def test_a_merge_of_whole_blocks_keeps_the_order_behind_an_import(lib, pool, reader):
    a, b = lib.order_stream(), lib.order_stream()
    ran, c = pool.imp(a, 160)
    merged, m = pool.compose(b, [c, c])
    assert "copy" not in merged
    if reader == "store":  # a store takes slots of its own
        pool.reserve(b, [m], [1])
    assert pool.before(ran["copy"], READERS[reader](pool, b, m))


@pytest.mark.parametrize("calls", [1, 2, 3])
def test_calls_that_copy_nothing_keep_the_order_of_all_work_before_them(lib, pool, calls):
    a, b, d = lib.order_stream(), lib.order_stream(), lib.order_stream()
    ran, c = pool.imp(a, 160)
    stored = pool.store(a, [c], [1])["store"]
    for _ in range(calls):  # the two piece buffers take turns
        pool.reserve(b, [c], [16])
    read = pool.attend(d, [c])["attend"]
    assert pool.before(ran["copy"], read) and pool.before(stored, read)
    copied = pool.append(d, [c], [5])["copy"]
    assert pool.before(read, copied) and pool.before(stored, copied)


def test_the_copies_of_a_pool_run_one_after_the_other(lib, pool):
    st = [lib.order_stream() for _ in range(3)]
    ran, c = pool.imp(st[0], 160)
    copies = [ran["copy"]]
    for i in range(1, 9):
        pool.reserve(st[(i + 1) % 3], [c], [16])
        copies.append(pool.materialize(st[i % 3], c, 20)["copy"])
    for x, y in zip(copies, copies[1:]):
        assert pool.before(x, y)
    assert not pool.wrongs()


def every_call(pool, st, c):
    """One of each kind on `st`; c: a context that nothing else names."""
    pool.attend(st, [c])
    pool.mass(st, [c])
    pool.reserve(st, [c], [16])
    pool.store(st, [c], [1])
    pool.append(st, [c], [3])
    pool.materialize(st, c, 5)
    _, kids = pool.fork(st, c, 2)
    _, merged = pool.compose(st, [c, kids[0]])
    _, small = pool.prune(st, c, 5)
    pool.evict(st, kids + [merged, small])
    pool.imp(st, 40)


@pytest.mark.parametrize("first", READERS)
def test_a_stream_may_be_destroyed_once_a_call_on_another_has_returned(lib, pool, first):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    _, other = pool.imp(b, 160)
    read = READERS[first](pool, a, c)
    pool.fork(b, other)  # orders nothing behind the reader
    lib.order_replace_stream(a, 0)
    second = pool.materialize(b, c, 5)
    every_call(pool, b, c)
    assert pool.before(read, second["copy"])
    assert lib.aaf_kv_sync_status(pool.h) == 0
    assert not pool.wrongs()


@pytest.mark.parametrize("first", READERS)
def test_the_last_reader_s_stream_may_be_captured_meanwhile(lib, pool, first):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    read = READERS[first](pool, a, c)
    lib.order_capture(a, 1)
    at = lib.order_ops()
    second = pool.attend(b, [c])["attend"]
    every_call(pool, b, c)
    assert pool.before(read, second)
    assert not any(lib.order_captured(i) for i in range(at, lib.order_ops()))
    assert not pool.wrongs()


@pytest.mark.parametrize("second", READERS)
def test_a_new_stream_under_an_old_handle_is_another_stream(lib, pool, second):
    a = lib.order_stream()
    ran, c = pool.imp(a, 160)
    a = lib.order_replace_stream(a, 1)
    assert pool.before(ran["copy"], READERS[second](pool, a, c))
    a = lib.order_replace_stream(a, 1)
    assert pool.before(ran["copy"], pool.append(a, [c], [5])["copy"])


@pytest.mark.parametrize("second", READERS)
def test_streams_whose_ids_cannot_be_had_are_taken_for_different_ones(lib, pool, second):
    a, b = lib.order_stream(), lib.order_stream()
    lib.order_fail(b"cudaStreamGetId", -1)
    ran, c = pool.imp(a, 160)
    pool.attend(a, [c])
    assert pool.before(ran["copy"], READERS[second](pool, b, c))


def imp_batch(pool, st, want):
    x = B.aaf_kv_xfer_desc()
    x.n_layers, x.n_kv_heads, x.head_dim, x.elt_bytes, x.n_tokens = L, H, D, 2, 40
    descs, src, out = (B.aaf_kv_xfer_desc * 1)(x), (C.c_void_p * 1)(pool.base), (C.c_int32 * 1)()
    return pool.call("import_batch", 1, src, descs, out, st, want=want)


def imp_chunked(pool, st, want):
    x = B.aaf_kv_xfer_desc()
    x.n_layers, x.n_kv_heads, x.head_dim, x.elt_bytes, x.n_tokens = L, H, D, 2, 40
    return pool.call("import_host_chunked", pool.base, C.byref(x), pool.base, 1 << 40, 32, C.byref(C.c_int32()), st, want=want)


# calls that write the table row of `old` (a handle that was read and is free again) or of `read` (one that was read and lives)
ROW_WRITERS = {"import": lambda p, s, read, want: p.imp(s, 40, want=want)[0], "import_batch": lambda p, s, read, want: imp_batch(p, s, want),
               "import_host_chunked": lambda p, s, read, want: imp_chunked(p, s, want),
               "fork": lambda p, s, read, want: p.fork(s, read, want=want)[0], "compose": lambda p, s, read, want: p.compose(s, [read], want=want)[0],
               "prune": lambda p, s, read, want: p.prune(s, read, 5, want=want)[0],
               "append": lambda p, s, read, want: p.append(s, [read], [3], want=want), "reserve": lambda p, s, read, want: p.reserve(s, [read], [3], want=want)}


@pytest.mark.parametrize("writer", ROW_WRITERS)
def test_a_table_row_is_not_rewritten_when_the_wait_for_its_readers_fails(lib, pool, writer):
    a, b = lib.order_stream(), lib.order_stream()
    _, old = pool.imp(b, 160)
    _, read = pool.imp(b, 160)
    seen = pool.attend(a, [old, read])["attend"]
    pool.evict(b, [old])
    lib.order_fail(b"cudaStreamWaitEvent", 1)
    assert not ROW_WRITERS[writer](pool, b, read, B.AAF_ERR_CUDA), "a planner was launched all the same"
    pool.attend(b, [read], want=B.AAF_ERR_CUDA)


@pytest.mark.parametrize("writer", ROW_WRITERS)
def test_a_table_row_is_rewritten_behind_its_readers(lib, pool, writer):
    a, b = lib.order_stream(), lib.order_stream()
    _, old = pool.imp(b, 160)
    _, read = pool.imp(b, 160)
    seen = pool.attend(a, [old, read])["attend"]
    pool.evict(b, [old])
    ran = ROW_WRITERS[writer](pool, b, read, 0)
    plan = [i for name, i in ran.items() if name.startswith("plan_") or name == "fork"]
    assert len(plan) == 1 and pool.before(seen, plan[0])


@pytest.mark.parametrize("last", READERS)
def test_destroying_a_pool_waits_for_its_work_on_every_stream(lib, pool, last):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    _, other = pool.imp(b, 40)
    ran = READERS[last](pool, a, c)
    pool.fork(b, other)
    pool.close()
    pool.h = None
    assert lib.order_host_knows(ran)
    assert not pool.wrongs()


def test_calls_beside_a_capture_wait_on_the_host_without_ending_it(lib, pool):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    lib.order_capture(a, 1)
    for _ in range(20):  # more batches in the pinned ring than it has room for at once
        pool.attend(b, [c] * 70)
    for _ in range(6):   # as many blocks as the pool has, so that the device's count is asked for
        _, big = pool.imp(b, 16000)
        pool.reserve(b, [big], [1])
        pool.prune(b, big, 2)
        pool.evict(b, [big])
    pool.close()
    pool.h = None
    assert not pool.wrongs()
    assert not any(lib.order_captured(i) for i in range(lib.order_ops()))


def test_a_store_in_place_has_one_stride(lib, pool):
    st = lib.order_stream()
    _, c = pool.imp(st, 160)
    q = dict(heads=2, q=pool.base, q_stride=2 * D)
    pool.store(st, [c], [3], q_out=pool.base, q_out_stride=2 * D, **q)
    pool.store(st, [c], [3], q_out=pool.base + 4096, q_out_stride=4 * D, **q)
    assert not pool.store(st, [c], [3], q_out=pool.base, q_out_stride=4 * D, want=B.AAF_ERR_INVALID_ARG, **q)
    pool.store(st, [c], [1], q_out=pool.base, q_out_stride=4 * D, **q)  # no stride is used


def test_tokens_of_2_to_the_31_elements_are_refused(lib, pool):
    st = lib.order_stream()
    _, c = pool.imp(st, 160)
    most = (1 << 31) // D - H
    for call in (pool.attend, pool.mass):
        assert call(st, [c], heads=most)
        assert not call(st, [c], heads=most + H, want=B.AAF_ERR_INVALID_ARG)


def test_threads_with_a_pool_each_launch_a_kernel_for_the_first_time(tmp_path):
    out = str(tmp_path / "threads")
    gcc = ["g++", "-std=c++17", "-O1", "-g", "-pthread", "-fsanitize=thread"]
    if subprocess.run(gcc + ["-x", "c++", "-", "-o", out], input="int main() {}", text=True, capture_output=True).returncode or \
            subprocess.run([out], capture_output=True).returncode:
        pytest.skip("no thread sanitizer here")
    subprocess.check_call(gcc + ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", os.path.join(CUDA, "include"),
                                 os.path.join(ROOT, "tests", "smem_threads.cpp"), "-o", out])
    run = subprocess.run([out], capture_output=True, text=True)
    assert "WARNING: ThreadSanitizer" not in run.stderr, run.stderr
    assert run.returncode == 0, run.stderr


@pytest.mark.parametrize("seed", range(12))
def test_random_calls_on_random_streams_keep_every_order_that_they_need(lib, pool, seed):
    """Payload kernels (copies, readers) all run one after the other; they come behind the metadata before them; and a table row is
    written behind the readers that were given it."""
    r = random.Random(seed)
    streams = [lib.order_stream() for _ in range(4)]
    live, payload, meta, readers = {}, [], [], {}

    def did(ran, rows=()):
        for name, i in ran.items():
            if name in ("select", "memcpy"):
                continue
            if name.startswith("plan_") or name in ("fork", "evict"):
                for h in rows:
                    for j in readers.pop(h, ()):
                        assert pool.before(j, i), (name, h)
                meta.append(i)
            else:
                for j in payload[-6:] + meta[-6:]:
                    assert pool.before(j, i), (pool.lib.order_name(j), name)
                payload.append(i)

    for _ in range(150):
        st = r.choice(streams)
        kind = r.choice(["imp", "reserve", "append", "fork", "compose", "evict", "materialize", "attend", "store", "mass", "prune", "attend", "swap"])
        if kind == "swap":  # a stream that was used goes, another one comes, under its handle or not
            i = r.randrange(4)
            st = streams[(i + 1) % 4]
            if live:
                did(pool.materialize(st, r.choice(list(live)), 1))
                streams[i] = lib.order_replace_stream(streams[i], r.randrange(2))
            continue
        if kind == "imp" or not live:
            if len(live) < 24:
                n = r.choice([16, 160, 37])
                ran, c = pool.imp(st, n)
                live[c] = n
                did(ran, [c])
            continue
        c = r.choice(list(live))
        if kind in ("reserve", "append"):
            n = r.choice([1, 16, 5])
            did(getattr(pool, kind)(st, [c], [n]), [c])
            live[c] += n
        elif kind in ("fork", "compose", "prune"):
            if len(live) < 24:
                if kind == "fork":
                    ran, (new,) = pool.fork(st, c)
                    n = live[c]
                elif kind == "compose":
                    other = r.choice(list(live))
                    ran, new = pool.compose(st, [c, other])
                    n = live[c] + live[other]
                else:
                    ran, new = pool.prune(st, c, 1)
                    n = 1
                live[new] = n
                did(ran, [new])
                if kind == "prune":
                    readers.setdefault(c, []).append(ran["gather"])
        elif kind == "evict":
            did(pool.evict(st, [c]))
            del live[c]
        elif kind == "materialize":
            did(pool.materialize(st, c, live[c]))
        else:
            if kind == "store":
                status = pool.lib.order_ops()
                ran = pool.store(st, [c], [1], want=None)
                if pool.status:
                    assert not ran and status == pool.lib.order_ops()
                    continue
            else:
                ran = getattr(pool, kind)(st, [c])
            did(ran)
            readers.setdefault(c, []).extend(ran.values())
    assert lib.aaf_kv_sync_status(pool.h) == 0
    assert not pool.wrongs()


@pytest.mark.parametrize("first", ["mass", "attend", "store"])
def test_a_prune_selects_behind_what_computes_its_scores_on_another_stream(lib, pool, first):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    ran = READERS[first](pool, a, c)
    assert pool.before(ran, pool.prune(b, c, 5)[0]["select"])


@pytest.mark.parametrize("last", READERS)
def test_introspection_while_the_last_call_s_stream_is_captured(lib, pool, last):
    a, b = lib.order_stream(), lib.order_stream()
    _, c = pool.imp(b, 160)
    ran = READERS[last](pool, a, c)
    lib.order_capture(a, 1)
    assert lib.aaf_kv_sync_status(pool.h) == 0
    assert lib.order_host_knows(ran)
    stats = B.aaf_kv_stats()
    assert lib.aaf_kv_pool_stats(pool.h, C.byref(stats)) == 0
    pool.close()
    pool.h = None
    assert not pool.wrongs()
