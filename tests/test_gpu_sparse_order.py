"""Order of sparse attention's calls across streams, where a wrong one shows in the results."""
from __future__ import annotations

import pytest
import torch

from tests import serve_reference as R
from tests import sparse_reference as S
from tests.test_gpu_sparse import pool_of, settle

pytestmark = pytest.mark.gpu


def lists(rows, q, keep, sink, recent, zero=False):
    """What select is to return for one token, from the context's rows or from a summary that holds nothing yet."""
    codes, exps = S.summary_ref(rows[0, 0], 16)
    if zero:
        codes, exps = torch.zeros_like(codes), torch.zeros_like(exps)
    heads, group, last = rows.shape[3], q.shape[0] // rows.shape[3], (rows.shape[2] - 1) // 16
    return [S.select_ref(S.scores_ref(codes[:, h], exps[:, h], q[h * group:(h + 1) * group]), last, keep, sink, recent) for h in range(heads)]


def test_a_choice_on_another_stream_knows_the_summary():
    pool, ctxs = pool_of(2, 64, 16, [1000, 700])
    h = [c.handle for c in ctxs]
    q, summary = R.rand((2, 8, 64), 1), pool.new_summary().zero_()
    blocks = torch.full((2, 2, 8), -1, dtype=torch.int32, device="cuda")
    pool.attend_blocks(0, h, None, q, blocks)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    with torch.cuda.stream(streams[0]):
        torch.cuda._sleep(20_000_000)
        assert pool.summarize(0, h, None, summary, torch.bfloat16)[0] == 0
    with torch.cuda.stream(streams[1]):
        assert pool.select(0, h, None, q, summary, 8, sink=1, recent=2, blocks=blocks)[0] == 0
    with torch.cuda.stream(streams[2]):
        st, got = pool.attend_blocks(0, h, None, q, blocks)
        assert st == 0
    settle(pool)
    for i, c in enumerate(ctxs):
        want = lists(c.rows, q[i], 8, 1, 2)
        assert want != lists(c.rows, q[i], 8, 1, 2, zero=True)  # a choice that had come first would show
        assert blocks[i].tolist() == want
    R.check_attend(got, S.attend_blocks_ref(ctxs, [1, 1], q, torch.tensor([lists(c.rows, q[i], 8, 1, 2) for i, c in enumerate(ctxs)], device="cuda"),
                                            16), torch.bfloat16, 64, False)


def test_a_summary_on_another_stream_waits_for_the_choice_that_reads_the_old_one():
    pool, ctxs = pool_of(2, 64, 16, [1000])
    h, c = [ctxs[0].handle], ctxs[0]
    q, summary = R.rand((1, 8, 64), 1), pool.new_summary().zero_()
    blocks = torch.full((1, 2, 8), -1, dtype=torch.int32, device="cuda")
    pool.attend_blocks(0, h, None, q, blocks)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(20_000_000)
        assert pool.select(0, h, None, q, summary, 8, sink=1, recent=2, blocks=blocks)[0] == 0
    with torch.cuda.stream(torch.cuda.Stream()):
        assert pool.summarize(0, h, None, summary, torch.bfloat16)[0] == 0
    settle(pool)
    old = lists(c.rows, q[0], 8, 1, 2, zero=True)
    assert old != lists(c.rows, q[0], 8, 1, 2) and blocks[0].tolist() == old
