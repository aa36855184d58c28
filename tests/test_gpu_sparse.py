"""Sparse attention over the pool and the tables of a batch against plain definitions in 64 bits, through the package's entry
points."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from paper_2607_10987_b200 import binding as B
from tests import serve_reference as R
from tests import sparse_reference as S

pytestmark = pytest.mark.gpu


def settle(pool):
    torch.cuda.synchronize()
    assert pool.sync_status() == 0


def pool_of(heads, dim, block, lens, dtype=torch.bfloat16, seed=1, layers=1, extra=8, fill=math.nan):
    blocks = sum(-(-t // block) for t in lens) + extra
    pool = R.make_pool(layers, heads, dim, block, blocks, max_ctx=len(lens) + 8, dtype=dtype, seed=seed, fill=fill)
    return pool, [R.add_ctx(pool, t, seed * 100 + i) for i, t in enumerate(lens)]


# ------------------------------------------------------------------------------------------ summaries
def check_summary(pool, summary, ctx, layers=None, first_block=0):
    table = torch.from_numpy(pool.table(ctx.handle)).cuda()
    for layer in range(pool.L) if layers is None else layers:
        codes, exps = S.read_summary(summary, layer, table, pool.H, pool.D)
        want, want_e = S.summary_ref(ctx.rows[layer, 0], pool.BS)
        assert torch.equal(codes[first_block:], want[first_block:]) and torch.equal(exps[first_block:], want_e[first_block:])
        # bounds are bounds
        hi, lo = (codes * torch.exp2(exps)[:, :, None, None]).unbind(2)
        k = ctx.rows[layer, 0].double()
        at = torch.arange(len(ctx), device="cuda") // pool.BS
        fine = torch.isfinite(k) & (k.abs() <= S.MOST) & (at >= first_block)[:, None, None]
        assert ((k <= hi[at]) | ~fine).all() and ((k >= lo[at]) | ~fine).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,dim,block", [(2, 64, 16), (8, 128, 16), (1, 8, 16), (3, 96, 5), (1, 256, 1), (5, 80, 40), (17, 16, 64), (2, 40, 33)])
def test_summaries(heads, dim, block, dtype):
    pool, ctxs = pool_of(heads, dim, block, [1, 2, 15, 16, 17, 64, 65, 300], dtype, layers=2)
    summary = pool.new_summary()
    summary.random_(-128, 128)
    before = summary.clone()
    assert pool.summarize(None, [c.handle for c in ctxs], None, summary, dtype)[0] == 0
    settle(pool)
    for c in ctxs:
        check_summary(pool, summary, c)
    used = np.concatenate([pool.table(c.handle) for c in ctxs])
    other = torch.ones(pool.NB, dtype=torch.bool, device="cuda")
    other[torch.from_numpy(used).long().cuda()] = False
    assert torch.equal(summary[:, other], before[:, other])  # blocks of nobody, and the filling
    assert torch.equal(summary[:, :, heads * (2 * dim + 1):], before[:, :, heads * (2 * dim + 1):])


@pytest.mark.parametrize("new", [[1, 1, 1], [16, 17, 1], [5, 33, 200]])
def test_summaries_of_the_last_tokens_blocks(new):
    lens = [100, 64, 200]
    pool, ctxs = pool_of(2, 64, 16, lens, layers=3)
    summary = pool.new_summary().zero_()
    assert pool.summarize(1, [c.handle for c in ctxs], new, summary, torch.bfloat16)[0] == 0
    settle(pool)
    for c, n in zip(ctxs, new):
        check_summary(pool, summary, c, [1], (len(c) - n) // 16)
        old = torch.from_numpy(pool.table(c.handle)[:(len(c) - n) // 16]).long().cuda()
        assert (summary[1, old] == 0).all()
    assert (summary[0] == 0).all() and (summary[2] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_summaries_of_odd_values(dtype):
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    sub = tiny * torch.finfo(dtype).eps
    special = [math.nan, math.inf, -math.inf, big, -big, tiny, -tiny, sub, -sub, 0.0, -0.0, 127.0, 127.5, 1.9921875, 2.0, -1.984375]
    rows = torch.zeros(1, 2, 16 * (len(special) + 2), 2, 16, dtype=dtype, device="cuda")
    for i, x in enumerate(special):  # one such value in a block of zeros; head 1: among others
        rows[0, 0, 16 * i + i % 16, 0, 3] = x
        rows[0, 0, 16 * i + 5, 1, 7] = x
        rows[0, 0, 16 * i + 6, 1, 8] = 1.0
        rows[0, 0, 16 * i + 7, 1, 7] = -1.5
    rows[0, 0, -32:-16] = tiny  # a block of the same
    rows[0, 0, -16:] = math.nan
    pool = R.make_pool(1, 2, 16, 16, len(special) + 6, dtype=dtype)
    c = R.add_ctx(pool, rows.shape[2], 0, rows)
    summary = pool.new_summary()
    assert pool.summarize(0, [c.handle], None, summary, dtype)[0] == 0
    settle(pool)
    check_summary(pool, summary, c)


def test_summaries_many_sequences_and_repeated_contexts():
    lens = [1 + 37 * i % 211 for i in range(90)]
    pool, ctxs = pool_of(2, 64, 16, lens)
    summary = pool.new_summary()
    order = list(range(90)) + [3, 3, 50]
    assert pool.summarize(0, [ctxs[i].handle for i in order], None, summary, torch.bfloat16)[0] == 0
    settle(pool)
    for c in ctxs:
        check_summary(pool, summary, c)


# ------------------------------------------------------------------------------------------ selection
def check_select(pool, ctxs, n_q, q, keep, sink, recent, summary=None):
    if summary is None:
        summary = pool.new_summary()
        summary.random_(-128, 128)
        assert pool.summarize(None, [c.handle for c in ctxs], None, summary, q.dtype)[0] == 0
    tokens = sum(n_q)
    scores = torch.full((tokens, pool.H, keep), 7.0, device="cuda")
    st, blocks = pool.select(0, [c.handle for c in ctxs], n_q, q, summary, keep, sink=sink, recent=recent, scores=scores)
    assert st == 0
    settle(pool)
    group, at = q.shape[1] // pool.H, 0
    for c, nq in zip(ctxs, n_q):
        codes, exps = S.read_summary(summary, 0, torch.from_numpy(pool.table(c.handle)).cuda(), pool.H, pool.D)
        for j in range(nq):
            last = (len(c) - nq + j) // pool.BS
            for h in range(pool.H):
                s = S.scores_ref(codes[:last + 1, h], exps[:last + 1, h], q[at + j, h * group:(h + 1) * group])
                want = S.select_ref(s, last, keep, sink, recent)
                got = blocks[at + j, h].tolist()
                assert got == want + [-1] * (keep - len(want)), (len(c), j, h)
                assert scores[at + j, h].tolist() == [s[b] for b in want] + [-math.inf] * (keep - len(want))
        at += nq
    return blocks, summary


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 64, 16), (8, 4, 128, 16), (1, 1, 8, 16), (3, 5, 96, 5), (1, 7, 256, 1), (2, 16, 80, 3),
                                                   (1, 40, 16, 16), (2, 2, 40, 8), (1, 130, 24, 16), (3, 3, 128, 16)])
def test_select_ragged(heads, group, dim, block, dtype):
    lens = [1, 2, 16, 17, 63, 130, 513, 700]
    pool, ctxs = pool_of(heads, dim, block, lens, dtype)
    q = R.rand((len(lens), heads * group, dim), 5, dtype, 3.0)
    check_select(pool, ctxs, [1] * len(lens), q, 6, 1, 2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,group,dim,tokens,times", [(8, 4, 128, 16 * 700 + 5, 20), (2, 16, 64, 16 * 3000 + 1, 20), (3, 5, 96, 16 * 1500, 30),
                                                          (16, 1, 40, 16 * 399 + 9, 20), (1, 32, 256, 16 * 4900 + 2, 24), (5, 2, 8, 16 * 1111, 25),
                                                          (8, 8, 128, 16 * 300 + 7, 64)])
def test_select_from_whole_records(heads, group, dim, tokens, times, dtype):
    # so many blocks that all heads of a block are taken together; three of the choices are looked at
    pool = R.make_pool(1, heads, dim, 16, 4910, max_ctx=4, dtype=dtype)
    longest = R.add_ctx(pool, tokens, 1)
    summary = pool.new_summary()
    assert pool.summarize(0, [longest.handle], None, summary, dtype)[0] == 0
    q = R.rand((times, heads * group, dim), 5, dtype, 3.0)
    scores = torch.empty(times, heads, 9, device="cuda")
    st, blocks = pool.select(0, [longest.handle] * times, None, q, summary, 9, sink=1, recent=2, scores=scores)
    assert st == 0
    settle(pool)
    codes, exps = S.read_summary(summary, 0, torch.from_numpy(pool.table(longest.handle)).cuda(), heads, dim)
    last = (len(longest) - 1) // 16
    for i in (0, times // 2, times - 1):
        for h in range(heads):
            s = S.scores_ref(codes[:, h], exps[:, h], q[i, h * group:(h + 1) * group])
            want = S.select_ref(s, last, 9, 1, 2)
            assert blocks[i, h].tolist() == want
            assert scores[i, h].tolist() == [s[b] for b in want]


@pytest.mark.parametrize("keep,sink,recent", [(1, 0, 1), (4, 0, 4), (4, 3, 1), (7, 2, 2), (33, 1, 4), (64, 0, 1), (100, 10, 20), (300, 1, 1)])
def test_select_budgets(keep, sink, recent):
    pool, ctxs = pool_of(2, 64, 16, [1030, 500, 90])
    q = R.rand((3, 8, 64), 5)
    check_select(pool, ctxs, [1, 1, 1], q, keep, sink, recent)


@pytest.mark.parametrize("heads,group,dim", [(2, 4, 128), (1, 3, 64), (1, 1, 64), (1, 20, 64), (2, 2, 96), (1, 40, 64), (1, 2, 256), (2, 4, 40),
                                             (1, 9, 8)])
@pytest.mark.parametrize("n_q", [[2, 5], [33, 16], [70, 1]])
def test_select_for_many_tokens(heads, group, dim, n_q):
    pool, ctxs = pool_of(heads, dim, 16, [300, 411])
    check_select(pool, ctxs, n_q, R.rand((sum(n_q), heads * group, dim), 5), 9, 1, 2)


@pytest.mark.parametrize("tokens,block", [(70, 4), (600, 2)])
def test_select_from_the_first_token_on(tokens, block):
    pool, ctxs = pool_of(1, 64, block, [tokens])
    check_select(pool, ctxs, [tokens], R.rand((tokens, 2, 64), 5), 5, 1, 2)


def test_select_equal_scores_go_to_the_lower_block():
    pool = R.make_pool(1, 1, 64, 16, 300)
    rows = torch.ones(1, 2, 16 * 200 + 3, 1, 64, dtype=torch.bfloat16, device="cuda")
    rows[0, 0, 16 * 77:16 * 78] = 2.0
    rows[0, 0, 16 * 120:16 * 140] = 0.5
    c = R.add_ctx(pool, rows.shape[2], 0, rows)
    q = torch.ones(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    blocks, summary = check_select(pool, [c], [1], q, 20, 1, 2)
    assert blocks[0, 0].tolist() == list(range(17)) + [77, 199, 200]
    check_select(pool, [c], [1], -q, 20, 0, 1, summary)  # all scores negative
    check_select(pool, [c], [1], torch.zeros_like(q), 20, 0, 1, summary)


@pytest.mark.parametrize("n_q", [1, 20])
def test_select_equal_scores_of_a_long_context(n_q):
    # nothing but equal scores, and a few that differ, over more blocks than a CTA looks after
    pool = R.make_pool(1, 2, 16, 4, 8000)
    rows = torch.ones(1, 2, 4 * 7000 + 1, 2, 16, dtype=torch.bfloat16, device="cuda")
    c = R.add_ctx(pool, rows.shape[2], 0, rows)
    q = torch.ones(n_q, 4, 16, dtype=torch.bfloat16, device="cuda")
    check_select(pool, [c], [n_q], q, 3000, 7, 5)
    rows[0, 0, 4 * 6000:4 * 6003, 0] = 2.0
    rows[0, 0, 4 * 100:4 * 3100, 1] = 0.5
    pool = R.make_pool(1, 2, 16, 4, 8000)
    c = R.add_ctx(pool, rows.shape[2], 0, rows)
    check_select(pool, [c], [n_q], q, 5000, 7, 5)


def test_select_scores_from_minus_to_plus_infinity():
    # products far beyond the type's range, both signs, and small ones: whole binades apart, many equal
    rows = R.rand((1, 2, 4 * 1500, 1, 16), 3)
    size = torch.randint(-100, 120, (1500,), device="cuda").repeat_interleave(4)
    rows[0, 0] = torch.where(torch.rand(6000, 1, 1, device="cuda") < 0.3, 0.0, rows[0, 0].float().sign() * torch.exp2(size.float())[:, None, None])
    rows[0, 0, 4000:5000] = -1e30
    pool = R.make_pool(1, 1, 16, 4, 1600)
    c = R.add_ctx(pool, 6000, 0, rows)
    q = R.rand((4, 2, 16), 5).sign()
    q[1] *= 1e30
    q[2] *= 1e-30
    q[3] = 1e30
    _, summary = check_select(pool, [c], [4], q, 40, 1, 1)
    for keep in (200, 700, 1100, 1499):
        check_select(pool, [c], [4], q, keep, 1, 1, summary)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_select_odd_values(dtype):
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    rows = R.rand((1, 2, 16 * 40 + 9, 2, 64), 3, dtype)
    for i, x in enumerate([math.nan, math.inf, -math.inf, big, -big, tiny]):
        rows[0, 0, 16 * (3 * i + 1) + i, 0, 5] = x
        rows[0, 0, 16 * (3 * i + 2):16 * (3 * i + 3), 1] = x
    pool = R.make_pool(1, 2, 64, 16, 60, dtype=dtype)
    c = R.add_ctx(pool, rows.shape[2], 0, rows)
    q = R.rand((6, 4, 64), 4, dtype)
    q[0] *= tiny
    q[1, :, 5] = math.inf
    q[2, :, 7] = math.nan
    q[3] = math.nan
    q[4] = q[4].sign() * big
    q[5, :, 5] = -math.inf
    check_select(pool, [c], [6], q, 12, 1, 1)


def test_select_long_contexts():
    # most of the scores outside one CTA's first pieces; ragged beside it
    lens = [60001, 9, 20000]
    pool, ctxs = pool_of(2, 64, 16, lens)
    check_select(pool, ctxs, [1, 1, 1], R.rand((3, 8, 64), 5), 100, 1, 4)
    check_select(pool, ctxs, [3, 2, 9], R.rand((14, 8, 64), 5), 100, 1, 4)


def test_select_more_blocks_than_shared_memory_holds_scores_of():
    pool = R.make_pool(1, 2, 8, 1, 60000, max_ctx=4)
    c = R.add_ctx(pool, 50001, 1)
    check_select(pool, [c], [3], R.rand((3, 4, 8), 2), 700, 1, 4)


def test_select_more_blocks_than_the_workspace_holds_scores_of():
    most = 65536 * 10 // 4
    pool = R.make_pool(1, 4, 8, 1, most + 600, max_ctx=4, max_blk=most + 10)
    c, d = R.add_ctx(pool, most, 1), R.add_ctx(pool, 500, 2)
    q = R.rand((5, 4, 8), 2)
    check_select(pool, [c, d], [2, 3], q, 50, 1, 4)  # a token at a time
    assert pool.reserve([c.handle], [1])[0] == 0
    assert pool.select(0, [c.handle], None, q[:1], pool.new_summary(), 50)[0] == B.AAF_ERR_TOO_LONG


def test_select_in_several_launches():
    # so many tokens that their scores do not fit into the workspace at once; a context's tokens go to two of the launches
    lens, n_q = [16 * 700 + 3, 16 * 600], [130, 90]
    pool, ctxs = pool_of(8, 8, 16, lens)
    check_select(pool, ctxs, n_q, R.rand((220, 8, 8), 5), 6, 1, 2)


def test_select_many_sequences_strided_queries_and_no_scores():
    lens = [1 + 53 * i % 400 for i in range(90)]
    pool, ctxs = pool_of(2, 64, 16, lens)
    wide = R.rand((90, 12, 64), 5)
    q = wide[:, 2:10]
    blocks, summary = check_select(pool, ctxs, [1] * 90, q, 5, 1, 1)
    st, again = pool.select(0, [c.handle for c in ctxs], None, q, summary, 5)
    assert st == 0 and torch.equal(again, blocks)


# ------------------------------------------------------------------------------------------ attention over listed blocks
def random_lists(pool, ctxs, n_q, keep, seed, whole=False):
    """Lists in any order, with entries that name nothing and repeated blocks."""
    r = np.random.default_rng(seed)
    rows = []
    for c, nq in zip(ctxs, n_q):
        nblk = -(-len(c) // pool.BS)
        for _ in range(nq):
            per = []
            for _ in range(pool.H):
                e = r.integers(0, nblk, keep)
                if not whole:
                    e[r.random(keep) < 0.2] = -1
                    e[r.random(keep) < 0.03] = nblk + r.integers(0, 5)
                    e[r.random(keep) < 0.03] = -2147483648
                    e[r.random(keep) < 0.03] = 2147483647
                per.append(e)
            rows.append(per)
    return torch.tensor(np.array(rows), dtype=torch.int32, device="cuda")


def check_blocks(pool, ctxs, n_q, q, blocks, layer=0, **kw):
    st, got = pool.attend_blocks(layer, [c.handle for c in ctxs], n_q, q, blocks, **kw)
    assert st == 0
    settle(pool)
    R.check_attend(got, S.attend_blocks_ref(ctxs, n_q, q, blocks, pool.BS, layer, **kw), q.dtype, pool.D, False)
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 64, 16), (8, 4, 128, 16), (1, 1, 128, 1), (3, 5, 96, 8), (2, 16, 128, 64), (4, 8, 64, 5),
                                                   (1, 8, 256, 16), (2, 1, 80, 24), (1, 32, 64, 32), (1, 3, 8, 16), (1, 17, 128, 16),
                                                   (1, 50, 64, 16), (2, 9, 256, 16), (1, 24, 40, 7), (3, 5, 96, 16), (2, 2, 80, 32), (1, 12, 200, 48)])
def test_listed_ragged(heads, group, dim, block, dtype):
    lens = [1, 2, 15, 16, 17, 63, 130, 513]
    pool, ctxs = pool_of(heads, dim, block, lens, dtype)
    n_q = [1] * len(lens)
    q = R.rand((len(lens), heads * group, dim), 7, dtype, 2.0)
    for keep in (1, 3, 20):
        check_blocks(pool, ctxs, n_q, q, random_lists(pool, ctxs, n_q, keep, keep))


@pytest.mark.parametrize("n_q", [[2, 1, 5], [40, 3, 1], [63, 64, 65]])
@pytest.mark.parametrize("heads,group,dim", [(2, 4, 128), (1, 3, 64)])
def test_listed_many_tokens(n_q, heads, group, dim):
    pool, ctxs = pool_of(heads, dim, 16, [200, 64, 300])
    q = R.rand((sum(n_q), heads * group, dim), 7, scale=2.0)
    check_blocks(pool, ctxs, n_q, q, random_lists(pool, ctxs, n_q, 6, 1))


@pytest.mark.parametrize("lens,keep", [([20000], 500), ([20000], 1250), ([9001, 3], 200), ([50] * 3 + [5000], 300), ([100], 1000)])
@pytest.mark.parametrize("heads,group,dim", [(2, 4, 64), (8, 8, 128), (1, 1, 256)])
def test_listed_split_and_joined(lens, keep, heads, group, dim):
    pool, ctxs = pool_of(heads, dim, 16, lens)
    q = R.rand((len(lens), heads * group, dim), 7, scale=2.0)
    check_blocks(pool, ctxs, [1] * len(lens), q, random_lists(pool, ctxs, [1] * len(lens), keep, 3))


@pytest.mark.parametrize("kw", [dict(softcap=5.0), dict(softcap=30.0), dict(window=1), dict(window=100), dict(window=5000), dict(scale=-0.3),
                                dict(scale=0.0), dict(slopes=True), dict(softcap=20.0, window=64, slopes=True), dict(spans=True),
                                dict(spans=True, slopes=True, window=200)])
def test_listed_options(kw):
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = 2.0 ** (-8.0 * torch.arange(1, 9, device="cuda") / 8)
    n_q = [1, 4, 2, 3]
    if kw.get("spans"):
        kw["spans"] = torch.tensor([[0, 1], [5, 40], [-7, 100000], [30, 30], [50, 20], [100, 700], [0, 650], [3, 1300], [1299, 1300], [0, 2]],
                                   dtype=torch.int32, device="cuda")
    for dim in (64, 128):
        pool, ctxs = pool_of(2, dim, 16, [1, 50, 700, 1300])
        q = R.rand((10, 8, dim), 7, scale=2.0)
        check_blocks(pool, ctxs, n_q, q, random_lists(pool, ctxs, n_q, 12, 5), **kw)


def test_all_blocks_listed_is_attention():
    lens, n_q = [1, 33, 700, 2049], [1, 3, 1, 5]
    for dim in (64, 128, 256):
        pool, ctxs = pool_of(2, dim, 16, lens)
        q = R.rand((10, 8, dim), 7, scale=2.0)
        blocks = torch.arange(129, dtype=torch.int32, device="cuda").expand(10, 2, 129).contiguous()
        st, got = pool.attend_blocks(0, [c.handle for c in ctxs], n_q, q, blocks)
        assert st == 0
        settle(pool)
        R.check_attend(got, R.attend_ref(ctxs, n_q, q), torch.bfloat16, dim, False)


def test_bias_of_far_listed_blocks_keeps_its_digits():
    # the listed blocks are tens of thousands of tokens away: scores that differ by little on top of a large bias
    slopes = torch.tensor([0.5, 0.25, 1.0, 0.125], device="cuda")
    pool, ctxs = pool_of(2, 64, 16, [50000])
    q = R.rand((1, 4, 64), 7)
    for lists in ([3, 4, 7], [3] * 200 + [4] * 100):  # a warp by itself, parts that are joined
        blocks = torch.tensor(lists, dtype=torch.int32, device="cuda").expand(1, 2, len(lists)).contiguous()
        check_blocks(pool, ctxs, [1], q, blocks, slopes=slopes)


def test_empty_lists_and_rows_that_see_nothing():
    pool, ctxs = pool_of(2, 64, 16, [300, 5])
    q = R.rand((2, 4, 64), 7)
    for keep in (1, 40, 600):
        blocks = torch.full((2, 2, keep), -1, dtype=torch.int32, device="cuda")
        out, lse = check_blocks(pool, ctxs, [1, 1], q, blocks)
        assert (out == 0).all() and (lse == -math.inf).all()
        blocks[0, 0, keep // 2] = 3  # behind the window; the other heads' lists stay empty
        out, lse = check_blocks(pool, ctxs, [1, 1], q, blocks, window=10)
        assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_what_is_not_listed_or_not_seen_has_no_influence(dim):
    # slots behind a context's end hold NaN already (the pool is full of them); here blocks that no list names, and keys behind the window
    rows = R.rand((1, 2, 400, 2, dim), 3)
    bad = rows.clone()
    bad[0, :, 32:48] = math.nan
    bad[0, 1, 352:356] = math.inf  # block 22, in part behind the window
    pool = R.make_pool(1, 2, dim, 16, 64)
    a, b = R.add_ctx(pool, 400, 0, rows), R.add_ctx(pool, 400, 0, bad)
    q = R.rand((1, 8, dim), 7, scale=2.0)
    blocks = torch.tensor([0, 1, 3, 22, 24], dtype=torch.int32, device="cuda").expand(1, 2, 5).contiguous()
    got = [check_blocks(pool, [c], [1], q, blocks, window=44) for c in (a, b)]
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("keep", [5, 300])
def test_infinite_values_that_are_listed(keep, dtype):
    rows = R.rand((1, 2, 400, 1, 64), 3, dtype)
    rows[0, 1, 100, 0, 5] = math.inf
    rows[0, 1, 200, 0, 6] = -math.inf
    rows[0, 1, 201, 0, 7] = math.nan
    pool = R.make_pool(1, 1, 64, 16, 64, dtype=dtype)
    c = R.add_ctx(pool, 400, 0, rows)
    q = R.rand((1, 4, 64), 7, dtype, 0.5)
    blocks = torch.full((1, 1, keep), -1, dtype=torch.int32, device="cuda")
    blocks[0, 0, 0], blocks[0, 0, -1], blocks[0, 0, keep // 2] = 6, 12, 20
    out, _ = check_blocks(pool, [c], [1], q, blocks)
    assert (out[0, :, 5] == math.inf).all() and (out[0, :, 6] == -math.inf).all() and torch.isnan(out[0, :, 7]).all()


def test_listed_keys_of_minus_infinity():
    rows = R.rand((1, 2, 64, 1, 64), 3)
    rows[0, 0, 16:32] = -math.inf
    rows[0, 1, 16:32] = 3.0
    pool = R.make_pool(1, 1, 64, 16, 64)
    c = R.add_ctx(pool, 64, 0, rows)
    q = R.rand((1, 2, 64), 7).abs()
    for lists in ([1], [1, 3], [1] * 100):
        check_blocks(pool, [c], [1], q, torch.tensor([[lists]], dtype=torch.int32, device="cuda"))


def test_listed_many_sequences_strides_and_same_bits_again():
    lens = [1 + 53 * i % 400 for i in range(90)]
    pool, ctxs = pool_of(2, 64, 16, lens)
    wide = R.rand((90, 12, 64), 5)
    q = wide[:, 2:10]
    blocks = random_lists(pool, ctxs, [1] * 90, 9, 3)
    out, lse = check_blocks(pool, ctxs, [1] * 90, q, blocks)
    st, (out2, lse2) = pool.attend_blocks(0, [c.handle for c in ctxs], None, q.contiguous(), blocks)
    assert st == 0 and torch.equal(out, out2) and torch.equal(lse, lse2)


def test_listed_layers_forks_and_repeated_contexts():
    pool, ctxs = pool_of(2, 64, 16, [200, 77], layers=3)
    st, kids = pool.fork(ctxs[0].handle, 3)
    assert st == 0
    all_ctx = ctxs + [R.Ctx(k, ctxs[0].rows) for k in kids] + [ctxs[1]]
    q = R.rand((6, 8, 64), 7)
    blocks = random_lists(pool, all_ctx, [1] * 6, 5, 3)
    for layer in range(3):
        check_blocks(pool, all_ctx, [1] * 6, q, blocks, layer=layer)


# ------------------------------------------------------------------------------------------ tables
@pytest.mark.parametrize("block", [1, 5, 16, 64])
@pytest.mark.parametrize("pads", [(0, 0, 0), (3, 50, 7), (1, 1, 2000)])
def test_batch_tables(block, pads):
    lens, new = [1, 2, 15, 16, 17, 700, 64], [1, 1, 15, 3, 17, 300, 64]
    pool, ctxs = pool_of(1, 8, block, lens)
    order = [5, 0, 3, 3, 1, 6, 2, 4]
    handles, ls, ns = [ctxs[i].handle for i in order], [lens[i] for i in order], [new[i] for i in order]
    rows, tokens, cols = len(order) + pads[0], sum(ns) + pads[1], -(-700 // block) + pads[2]
    st, got = pool.batch_tables(handles, ns, rows=rows, tokens=tokens, cols=cols)
    assert st == 0
    settle(pool)
    want = S.batch_tables_ref([pool.table(h).tolist() for h in handles], ls, ns, block, rows, tokens, cols)
    assert {k: v.tolist() for k, v in got.items()} == want


def test_batch_tables_of_one_token_each_some_arrays_and_more_contexts_than_kernel_parameters_hold():
    lens = [1 + 41 * i % 300 for i in range(100)]
    pool, ctxs = pool_of(1, 8, 16, lens)
    handles = [c.handle for c in ctxs]
    want = S.batch_tables_ref([pool.table(h).tolist() for h in handles], lens, [1] * 100, 16, 100, 100, 19)
    st, got = pool.batch_tables(handles)
    assert st == 0
    settle(pool)
    assert {k: v.tolist() for k, v in got.items()} == want
    some = {"slots": torch.full((100,), 5, device="cuda"), "lens": torch.full((100,), 5, dtype=torch.int32, device="cuda")}
    st, got = pool.batch_tables(handles, out=some)
    assert st == 0 and got is some
    settle(pool)
    assert some["slots"].tolist() == want["slots"] and some["lens"].tolist() == want["lens"]


@pytest.mark.parametrize("n", [64, 65, 512, 513])
def test_batch_tables_of_many_rows(n):
    lens, new = [1 + 7 * i % 40 for i in range(n)], [1 + i % (1 + 7 * i % 40) for i in range(n)]
    pool, ctxs = pool_of(1, 8, 8, lens)
    handles = [c.handle for c in ctxs]
    st, got = pool.batch_tables(handles, new, rows=n + 2)
    assert st == 0
    settle(pool)
    want = S.batch_tables_ref([pool.table(h).tolist() for h in handles], lens, new, 8, n + 2, sum(new), 5)
    assert {k: v.tolist() for k, v in got.items()} == want


def test_slots_name_the_rows_that_store_writes():
    pool, ctxs = pool_of(2, 64, 16, [40, 16], layers=2)
    handles, new = [c.handle for c in ctxs], [5, 20]
    assert pool.reserve(handles, new)[0] == 0
    k, v = R.rand((25, 2, 64), 1), R.rand((25, 2, 64), 2)
    assert pool.store(1, handles, new, k, v)[0] == 0
    st, got = pool.batch_tables(handles, new)
    assert st == 0
    settle(pool)
    s = got["slots"]
    assert torch.equal(pool.mem[1, s // 16, 0, s % 16], k) and torch.equal(pool.mem[1, s // 16, 1, s % 16], v)


# ------------------------------------------------------------------------------------------ refusals, streams, all together
def test_refusals_change_nothing():
    pool, ctxs = pool_of(2, 64, 16, [100, 40])
    h = [c.handle for c in ctxs]
    q, summary = R.rand((2, 8, 64), 1), pool.new_summary().zero_()
    blocks = torch.zeros(2, 2, 4, dtype=torch.int32, device="cuda")
    bf = torch.bfloat16
    assert pool.summarize(0, [77], None, summary, bf)[0] == B.AAF_ERR_BAD_CTX
    for layer in (-2, 1, 5):
        assert pool.summarize(layer, h, None, summary, bf)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.summarize(0, h, [0, 1], summary, bf)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.summarize(0, h, [101, 1], summary, bf)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.summarize(0, [], [], summary, bf)[0] == B.AAF_ERR_INVALID_ARG
    for bad in (summary[:, 1:], summary.view(torch.uint8), summary.cpu()):
        with pytest.raises(ValueError):
            pool.summarize(0, h, None, bad, bf)
    with pytest.raises(ValueError):
        pool.summarize(0, h, None, summary, torch.float32)
    for kw in (dict(keep=0), dict(keep=-3), dict(keep=4, recent=0), dict(keep=4, sink=-1), dict(keep=4, sink=3, recent=2)):
        assert pool.select(0, h, None, q, summary, **kw)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.select(1, h, None, q, summary, 4)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.select(0, h, [1, 41], R.rand((42, 8, 64), 1), summary, 4)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.select(0, [h[0], 50], None, q, summary, 4)[0] == B.AAF_ERR_BAD_CTX
    assert pool.select(0, h, None, q[:, :7], summary, 4)[0] == B.AAF_ERR_INVALID_ARG
    for bad in (blocks[:, :, :3], blocks.long(), blocks.cpu()):
        with pytest.raises(ValueError):
            pool.select(0, h, None, q, summary, 4, blocks=bad)
    with pytest.raises(ValueError):
        pool.select(0, h, None, q, summary, 4, scores=blocks)
    assert pool.attend_blocks(1, h, None, q, blocks)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.attend_blocks(0, h, None, q, blocks, softcap=-1.0)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.attend_blocks(0, [99, h[0]], None, q, blocks)[0] == B.AAF_ERR_BAD_CTX
    assert pool.attend_blocks(0, h, None, q, blocks[:, :, :0])[0] == B.AAF_ERR_INVALID_ARG
    for bad in (blocks[:1], blocks.long(), blocks.transpose(1, 2)):
        with pytest.raises(ValueError):
            pool.attend_blocks(0, h, None, q, bad)
    for kw in (dict(rows=1), dict(tokens=1), dict(cols=6), dict(rows=-1)):
        assert pool.batch_tables(h, **kw)[0] == B.AAF_ERR_DST_TOO_SMALL
    assert pool.batch_tables(h, [1, 41])[0] == B.AAF_ERR_INVALID_ARG
    assert pool.batch_tables([h[0], 60])[0] == B.AAF_ERR_BAD_CTX
    with pytest.raises(ValueError):
        pool.batch_tables(h, out={"lens": torch.zeros(3, dtype=torch.int32, device="cuda")})
    settle(pool)
    assert (summary == 0).all() and (blocks == 0).all()


def test_pools_without_summaries():
    for heads, dim, elt in ((2, 264, 2), (2, 12, 2), (16, 64, 1)):
        pool = B.KVPool(1, heads, dim, 16, elt, 8, 4, 8)
        assert pool.summary_bytes() == 0
        with pytest.raises(ValueError):
            pool.new_summary()
        st, h = pool.imp(torch.zeros(pool.bpt * 20, dtype=torch.uint8, device="cuda"), 20)
        one, room = (B.C.c_int32 * 1)(h), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
        assert B.aaf_kv_summarize(pool.h, 0, 0, 1, one, None, room.data_ptr(), room.numel(), None) == B.AAF_ERR_INCOMPAT
        d = B.aaf_kv_select_desc(B.C.sizeof(B.aaf_kv_select_desc), 0, heads, 4, 1, 1, heads * dim)
        assert B.aaf_kv_select(pool.h, 0, d, 1, one, None, room.data_ptr(), room.data_ptr(), room.numel(), room.data_ptr(), None, room.data_ptr(),
                               room.numel(), None) == B.AAF_ERR_INCOMPAT
        st, got = pool.batch_tables([h])  # tables know nothing of elements
        assert st == 0 and got["tables"].tolist() == [pool.table(h).tolist()]


def test_calls_in_a_capture_are_refused():
    pool, ctxs = pool_of(2, 64, 16, [100])
    h, q, summary = [ctxs[0].handle], R.rand((1, 8, 64), 1), pool.new_summary()
    blocks = torch.zeros(1, 2, 4, dtype=torch.int32, device="cuda")
    assert pool.attend_blocks(0, h, None, q, blocks)[0] == 0
    tables = pool.batch_tables(h)[1]
    out, lse = torch.empty_like(q), torch.empty(1, 8, device="cuda")
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph.capture_begin()
        got = [pool.summarize(0, h, None, summary, torch.bfloat16)[0], pool.select(0, h, None, q, summary, 4, blocks=blocks)[0],
               pool.attend_blocks(0, h, None, q, blocks, out=out, lse=lse)[0], pool.batch_tables(h, out=tables)[0]]
        keep = torch.zeros(1, device="cuda")
        graph.capture_end()
    assert got == [B.AAF_ERR_INVALID_ARG] * 4
    check_blocks(pool, ctxs, [1], q, blocks)


def test_summaries_choice_and_attention_on_streams_of_their_own():
    """Each call on another stream than the one before, with a device that is held back: the pool's calls are ordered."""
    pool, ctxs = pool_of(2, 64, 16, [1000, 700])
    h = [c.handle for c in ctxs]
    q, summary = R.rand((2, 8, 64), 1), pool.new_summary().zero_()
    blocks = torch.zeros(2, 2, 8, dtype=torch.int32, device="cuda")
    pool.attend_blocks(0, h, None, q, blocks)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    with torch.cuda.stream(streams[0]):
        torch.cuda._sleep(20_000_000)
        assert pool.summarize(0, h, None, summary, torch.bfloat16)[0] == 0
    with torch.cuda.stream(streams[1]):
        assert pool.select(0, h, None, q, summary, 8, blocks=blocks)[0] == 0
    with torch.cuda.stream(streams[2]):
        st, got = pool.attend_blocks(0, h, None, q, blocks)
        assert st == 0
    settle(pool)
    assert (blocks[:, :, -1] >= 0).all()
    R.check_attend(got, S.attend_blocks_ref(ctxs, [1, 1], q, blocks, 16), torch.bfloat16, 64, False)


def test_an_eviction_waits_for_the_calls_that_read_the_table():
    pool, ctxs = pool_of(2, 64, 16, [1000], extra=4)
    h, q, summary = [ctxs[0].handle], R.rand((1, 8, 64), 1), pool.new_summary()
    table = pool.table(h[0]).tolist()
    blocks = torch.arange(63, dtype=torch.int32, device="cuda").expand(1, 2, 63).contiguous()
    pool.attend_blocks(0, h, None, q, blocks)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(20_000_000)
        assert pool.summarize(0, h, None, summary, torch.bfloat16)[0] == 0
        st, got = pool.attend_blocks(0, h, None, q, blocks)
        st2, tables = pool.batch_tables(h)
        assert st == st2 == 0
        assert pool.evict(h)[0] == 0
        other = R.rand((1, 2, 1000, 2, 64), 9)
    st, new = pool.imp(other, 1000)  # the freed handle and blocks, on another stream
    assert st == 0 and new == h[0]
    settle(pool)
    assert tables["tables"].tolist() == [table]
    R.check_attend(got, S.attend_blocks_ref(ctxs, [1], q, blocks, 16), torch.bfloat16, 64, False)
    want, _ = S.summary_ref(ctxs[0].rows[0, 0], 16)
    assert torch.equal(S.read_summary(summary, 0, torch.tensor(table), 2, 64)[0], want)


def test_an_unusable_pool_refuses():
    pool, ctxs = pool_of(2, 64, 16, [100])
    h, q, summary = [ctxs[0].handle], R.rand((1, 8, 64), 1), pool.new_summary()
    blocks = torch.zeros(1, 2, 4, dtype=torch.int32, device="cuda")
    assert B.aaf_kv_debug_mark_unusable(pool.h) == 0
    assert pool.summarize(0, h, None, summary, torch.bfloat16)[0] == B.AAF_ERR_CUDA
    assert pool.select(0, h, None, q, summary, 4)[0] == B.AAF_ERR_CUDA
    assert pool.attend_blocks(0, h, None, q, blocks)[0] == B.AAF_ERR_CUDA
    assert pool.batch_tables(h)[0] == B.AAF_ERR_CUDA


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_serving_loop(dtype):
    """A prompt, forked agents, decoding steps layer by layer: reserve, store, summarize, select, attend_blocks, the tables of the batch;
    tails that are copied on write, a merge and a pruned context among them."""
    layers, heads, group, dim, block, keep = 2, 2, 4, 64, 16, 6
    pool = R.make_pool(layers, heads, dim, block, 256, dtype=dtype)
    summary = pool.new_summary()
    root = R.add_ctx(pool, 215, 1)
    assert pool.summarize(None, [root.handle], None, summary, dtype)[0] == 0
    st, kids = pool.fork(root.handle, 3)
    assert st == 0
    agents = [root] + [R.Ctx(k, root.rows.clone()) for k in kids]
    inv = torch.tensor(B.rope_freqs(dim)[0], dtype=torch.float64, device="cuda")
    for step, new in enumerate([[1] * 4, [3, 1, 20, 2], [1] * 4, [1] * 4]):
        if step == 2:  # a merge that packs its second half anew, and a context of what mattered
            st, merged = pool.compose([agents[1].handle, agents[2].handle])
            assert st == 0
            agents[3] = R.Ctx(merged, torch.cat((agents[1].rows, agents[2].rows), 2))
            kept = torch.empty(100, dtype=torch.int32, device="cuda")
            st, small = pool.prune(agents[0].handle, torch.rand(len(agents[0]), device="cuda"), 100, sink=4, recent=8, kept=kept)
            assert st == 0
            agents[0] = R.Ctx(small, agents[0].rows[:, :, kept.long()])
            assert pool.summarize(None, [merged, small], None, summary, dtype)[0] == 0
        h, tokens = [a.handle for a in agents], sum(new)
        assert pool.reserve(h, new)[0] == 0
        fresh = torch.empty(layers, 2, tokens, heads, dim, dtype=dtype, device="cuda")
        results = []
        for layer in range(layers):
            q, k, v = (R.rand((tokens, n, dim), 100 * step + 10 * layer + i, dtype) for i, n in enumerate((heads * group, heads, heads)))
            assert pool.store(layer, h, new, k, v, q=q, rope=B.Rope(dim, inv))[0] == 0
            assert pool.summarize(layer, h, new, summary, dtype)[0] == 0
            st, blocks = pool.select(layer, h, new, q, summary, keep, sink=1, recent=2)
            assert st == 0
            st, got = pool.attend_blocks(layer, h, new, q, blocks)
            assert st == 0
            results.append((q, blocks, got))
        st, tables = pool.batch_tables(h, new, rows=6, tokens=tokens + 3)
        assert st == 0
        settle(pool)
        slots = tables["slots"][:tokens]
        for layer in range(layers):
            fresh[layer] = pool.mem[layer, slots // block, :, slots % block].transpose(0, 1)
        at = 0
        for a, n in zip(agents, new):
            a.rows = torch.cat((a.rows, fresh[:, :, at:at + n]), 2)
            at += n
        for layer, (q, blocks, got) in enumerate(results):
            R.check_attend(got, S.attend_blocks_ref(agents, new, q, blocks, block, layer=layer), dtype, dim, False)
            for a in agents:
                check_summary(pool, summary, a, [layer])
            at = 0
            for a, n in zip(agents, new):
                codes, exps = S.read_summary(summary, layer, torch.from_numpy(pool.table(a.handle)).cuda(), heads, dim)
                for j in range(n):
                    last = (len(a) - n + j) // block
                    for hd in range(heads):
                        s = S.scores_ref(codes[:, hd], exps[:, hd], q[at + j, hd * group:(hd + 1) * group])
                        want = S.select_ref(s, last, keep, 1, 2)
                        assert blocks[at + j, hd].tolist() == want + [-1] * (keep - len(want))
                at += n
