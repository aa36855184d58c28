"""Calls of one pool on several streams, with a device that is held back where the order matters."""
from __future__ import annotations

import pytest
import torch

from paper_2607_10987_b200 import binding as B
from tests import serve_reference as R

pytestmark = pytest.mark.gpu

LATE = 20_000_000  # cycles that a stream is held back: some 10 ms


def busy_import(pool, stream, rows, tokens):
    """An import that is still under way when this returns."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(LATE)
        st, h = pool.imp(rows, tokens)
    assert st == 0
    return R.Ctx(h, rows)


def two_streams():
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for s in (a, b):
        s.wait_stream(torch.cuda.current_stream())
    return a, b


@pytest.mark.parametrize("how", ["reserve", "merge"])
def test_a_call_that_copies_nothing_keeps_the_order_behind_an_import_on_another_stream(how):
    pool = R.make_pool(1, 2, 64, 16, 1024)
    rows, q = R.rand((1, 2, 4096, 2, 64), 1), R.rand((1, 8, 64), 2)
    torch.cuda.synchronize()
    a, b = two_streams()
    ctx = busy_import(pool, a, rows, 4096)
    with torch.cuda.stream(b):
        if how == "reserve":
            h, new = ctx.handle, R.rand((1, 2, 64), 3)
            assert pool.reserve([h], [1])[0] == 0
            assert pool.store(0, [h], [1], new, new)[0] == 0
            known = R.Ctx(h, torch.cat((rows, new.view(1, 1, 1, 2, 64).expand(1, 2, 1, 2, 64)), 2))
        else:
            st, h = pool.compose([ctx.handle])
            assert st == 0
            known = R.Ctx(h, rows)
        st, got = pool.attend(0, [h], [1], q)
        assert st == 0
    torch.cuda.synchronize()
    assert pool.sync_status() == 0
    R.check_attend(got, R.attend_ref([known], [1], q), torch.bfloat16, 64, False)


def test_the_last_reader_s_stream_is_captured_meanwhile():
    """Warm-up calls on a stream, then its capture; beside it the pool is used on another one, by every kind of wait that a call
    makes on the host: many batches in the pinned ring, a reserve and a prune for which the device's block count is asked."""
    pool = R.make_pool(1, 2, 64, 16, 64)
    c = R.add_ctx(pool, 320, 1)
    q = R.rand((70, 8, 64), 1)
    scores, kept = torch.rand(320, device="cuda"), torch.empty(16, dtype=torch.int32, device="cuda")
    many = [c.handle] * 70
    torch.cuda.synchronize()
    a, b = two_streams()
    with torch.cuda.stream(b):
        out, lse = torch.empty_like(q), q.new_empty((70, 8), dtype=torch.float32)
    x = torch.zeros(1, device="cuda")
    with torch.cuda.stream(a):
        st, first = pool.attend(0, many, None, q)
    assert st == 0
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a):
        x.add_(1.0)
        with torch.cuda.stream(b):
            stats = [pool.attend(0, many, None, q, out=out, lse=lse)[0] for _ in range(20)]
            for _ in range(60):
                st, h = pool.prune(c.handle, scores, 16, kept=kept)
                stats += [st, pool.reserve([h], [16])[0], pool.evict([h])[0]]
    assert not any(stats)
    graph.replay()
    torch.cuda.synchronize()
    assert float(x) == 1 and pool.sync_status() == 0
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    R.check_attend((out, lse), R.attend_ref([c] * 70, [1] * 70, q), torch.bfloat16, 64, False)


def test_streams_come_and_go_between_calls():
    pool = R.make_pool(1, 2, 64, 16, 400)
    c = R.add_ctx(pool, 2000, 1)
    q = R.rand((1, 8, 64), 2)
    ref = R.attend_ref([c], [1], q)
    for _ in range(20):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            st, got = pool.attend(0, [c.handle], None, q)
            assert st == 0
        st, rows = pool.materialize(c.handle, 0, 2000)
        assert st == 0 and torch.equal(rows.view(torch.bfloat16).view(c.rows.shape), c.rows)
        R.check_attend(got, ref, torch.bfloat16, 64, False)
    assert pool.sync_status() == 0


def test_a_first_call_in_a_capture_leaves_no_scratch_of_the_graph_s_memory():
    pool = R.make_pool(1, 2, 64, 16, 64)
    c = R.add_ctx(pool, 320, 1)
    q = R.rand((1, 8, 64), 1)
    x = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1.0)
        st, got = pool.attend(0, [c.handle], None, q)
    assert st == B.AAF_ERR_INVALID_ARG and got is None and pool._attend_ws is None
    graph.replay()
    st, got = pool.attend(0, [c.handle], None, q)
    assert st == 0
    torch.cuda.synchronize()
    assert float(x) == 1 and pool.sync_status() == 0
    R.check_attend(got, R.attend_ref([c], [1], q), torch.bfloat16, 64, False)


def test_introspection_and_the_end_of_a_pool_beside_a_capture_of_its_stream():
    pool = R.make_pool(1, 2, 64, 16, 64)
    c = R.add_ctx(pool, 320, 1)
    q = R.rand((1, 8, 64), 1)
    x = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    a, b = two_streams()
    with torch.cuda.stream(a):
        st, got = pool.attend(0, [c.handle], None, q)
    assert st == 0
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a):
        x.add_(1.0)
        status, stats, table = pool.sync_status(), pool.stats(), pool.table(c.handle)
        pool.close()
    graph.replay()
    torch.cuda.synchronize()
    assert float(x) == 1 and status == 0 and stats["live_ctx"] == 1 and len(table) == 20
    R.check_attend(got, R.attend_ref([c], [1], q), torch.bfloat16, 64, False)
