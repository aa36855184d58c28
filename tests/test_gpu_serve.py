"""The operators that compute with the pool's payload (store with rotary positions, attention, attention mass, token
pruning) against plain definitions in 64 bits, through the package's entry points."""
from __future__ import annotations

import ctypes as C
import math

import pytest
import torch

from paper_2607_10987_b200 import binding as B
from tests import serve_reference as R

pytestmark = pytest.mark.gpu


def run_attend(pool, ctxs, n_q, q, **kw):
    st, got = pool.attend(kw.pop("layer", 0), [c.handle for c in ctxs], n_q, q, **kw)
    assert st == 0
    torch.cuda.synchronize()
    assert pool.sync_status() == 0
    return got


def case(heads, group, dim, block, lens, n_q=None, dtype=torch.bfloat16, seed=1, **kw):
    n_q = n_q or [1] * len(lens)
    blocks = sum(-(-t // block) for t in lens) + 4
    pool = R.make_pool(1, heads, dim, block, blocks, max_ctx=len(lens) + 2, dtype=dtype, seed=seed)
    ctxs = [R.add_ctx(pool, t, seed * 100 + i) for i, t in enumerate(lens)]
    q = R.rand((sum(n_q), heads * group, dim), seed + 7, dtype, 2.0)
    got = run_attend(pool, ctxs, n_q, q, **kw)
    ref = R.attend_ref(ctxs, n_q, q, **kw)
    many = max(n_q) * group > (32 if dim <= 64 else 16 if dim <= 128 else 8)
    R.check_attend(got, ref, dtype, dim, p_rounded=many)
    return pool, ctxs, q, got


# ------------------------------------------------------------------------------------------ attend: one token
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 64, 16), (8, 4, 128, 16), (1, 1, 128, 1), (3, 5, 96, 8), (2, 16, 128, 64),
                                                   (4, 8, 64, 5), (1, 8, 256, 16), (2, 1, 80, 16), (1, 32, 64, 32), (1, 3, 8, 16)])
def test_decode_ragged(heads, group, dim, block, dtype):
    case(heads, group, dim, block, [1, 2, 15, 16, 17, 63, 64, 65, 127, 130, 513, 777], dtype=dtype)


@pytest.mark.parametrize("lens", [[1], [64], [65], [4097], [9001, 3], [1] * 40 + [2000]])
def test_decode_split_and_joined(lens):
    case(2, 4, 64, 16, lens)
    case(8, 8, 128, 16, lens)


def test_decode_more_sequences_than_kernel_parameters_hold():
    case(2, 2, 64, 16, [1 + 13 * i % 300 for i in range(90)])


@pytest.mark.parametrize("kw", [dict(softcap=5.0), dict(softcap=30.0), dict(window=1), dict(window=100), dict(window=5000),
                                dict(scale=0.5), dict(slopes=True), dict(softcap=20.0, window=64, slopes=True)])
def test_decode_options(kw):
    if kw.get("slopes"):
        kw = dict(kw, slopes=2.0 ** (-8.0 * torch.arange(1, 9, device="cuda") / 8))
    case(2, 4, 64, 16, [1, 50, 700, 1300], **kw)
    case(2, 4, 128, 16, [1, 50, 700, 1300], n_q=[1, 2, 4, 3], **kw)


def test_bias_far_from_the_span_keeps_its_digits():
    # every visible key is thousands of tokens away: the scores differ by little on top of a large bias
    slopes = torch.tensor([0.5, 0.25], device="cuda")
    spans = torch.tensor([[10, 40]], dtype=torch.int32, device="cuda")
    pool, ctxs, q, got = case(1, 2, 64, 16, [9000], slopes=slopes, spans=spans)
    assert torch.isfinite(got[1]).all()


@pytest.mark.parametrize("n_q", [[2], [3, 1, 4], [4, 4, 4, 4]])
def test_few_tokens(n_q):
    case(2, 4, 64, 16, [40 + 333 * i for i in range(len(n_q))], n_q=n_q)
    case(2, 4, 128, 16, [40 + 333 * i for i in range(len(n_q))], n_q=n_q)


# ------------------------------------------------------------------------------------------ attend: many tokens
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,group,dim,block", [(2, 4, 64, 16), (2, 4, 128, 16), (1, 3, 96, 8), (1, 2, 256, 16), (2, 1, 80, 7),
                                                   (1, 64, 128, 32)])
def test_extend_ragged(heads, group, dim, block, dtype):
    case(heads, group, dim, block, [1, 40, 64, 300, 700], n_q=[1, 40, 17, 65, 129], dtype=dtype)


@pytest.mark.parametrize("kw", [dict(softcap=20.0), dict(window=33), dict(slopes=True), dict(softcap=50.0, slopes=True, window=200)])
@pytest.mark.parametrize("dim", [64, 128])
def test_extend_options(kw, dim):
    if kw.get("slopes"):
        kw = dict(kw, slopes=2.0 ** (-8.0 * torch.arange(1, 9, device="cuda") / 8))
    case(2, 4, dim, 16, [600, 333], n_q=[256, 333], **kw)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_masks_as_spans(dim):
    lens, n_q = [500, 260], [500, 200]
    rows = []
    starts = [0, 37, 38, 300, 411]
    for p in range(500):  # documents
        rows.append((max(s for s in starts if s <= p), p + 1))
    for p in range(60, 260):  # prefix, seen in both directions
        rows.append((0, max(p + 1, 190)))
    spans = torch.tensor(rows, dtype=torch.int32, device="cuda")
    case(2, 2, dim, 16, lens, n_q=n_q, spans=spans)
    # clipped to the context, empty and inverted spans: rows of zeros
    odd = spans.clone()
    odd[::7] = torch.tensor([-5, 100000], dtype=torch.int32)
    odd[3::7] = torch.tensor([9, 9], dtype=torch.int32)
    odd[4::7] = torch.tensor([50, 20], dtype=torch.int32)
    pool, ctxs, q, (out, lse) = case(2, 2, dim, 16, lens, n_q=n_q, spans=odd)
    assert (out[3::7] == 0).all() and (lse[3::7] == -math.inf).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("block", [8, 16, 32, 64, 128])
def test_extend_long_prompts(block, dim, dtype):
    # several 256-row units, keys cut into parts for the short ones, block sizes that divide a key tile differently
    case(2, 4, dim, block, [1500, 777, 5000, 130], n_q=[700, 777, 30, 129], dtype=dtype)


@pytest.mark.parametrize("group,n_q,lens", [(1, [256, 257, 100], [256, 3000, 129]), (3, [86, 43], [2000, 43]), (7, [300], [301]),
                                            (32, [4, 33], [1000, 1000]), (128, [2, 3], [400, 128])])
def test_extend_groups_that_do_not_divide_the_tile(group, n_q, lens):
    case(1, group, 128, 16, lens, n_q=n_q)
    case(2, group, 64, 16, lens, n_q=n_q)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale", [-0.1, 0.0, 2.0])
def test_extend_scales(scale, dim):
    case(1, 2, dim, 16, [900, 400], n_q=[400, 90], scale=scale)
    case(1, 2, dim, 16, [900, 400], scale=scale)


@pytest.mark.parametrize("n_q", [1, 4, 300])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_scores_that_keep_growing_along_the_keys(dim, n_q):
    # every few tiles the running maximum outgrows what has been summed by far more than a rescale's threshold
    t = 2000
    pool = R.make_pool(1, 1, dim, 16, 256)
    q = R.rand((n_q, 2, dim), 3)
    rows = R.rand((1, 2, t, 1, dim), 4)
    ramp = torch.linspace(0, 6, t, device="cuda")[:, None, None]
    rows[0, 0] = (rows[0, 0].float() * 0.1 + ramp * q[0, :1].float().sign()).to(torch.bfloat16)
    c = R.add_ctx(pool, t, 0, rows)
    got = run_attend(pool, [c], [n_q], q)
    R.check_attend(got, R.attend_ref([c], [n_q], q), torch.bfloat16, dim, p_rounded=n_q > 4)


def test_extend_many_sequences():
    case(1, 4, 64, 16, [20 + 9 * i for i in range(80)], n_q=[10 + i % 11 for i in range(80)])


def test_empty_span_of_single_tokens():
    spans = torch.tensor([[5, 5], [0, 40], [100, 7]], dtype=torch.int32, device="cuda")
    _, _, _, (out, lse) = case(2, 4, 64, 16, [80, 40, 900], spans=spans)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all() and (out[2] == 0).all()
    assert torch.isfinite(lse[1]).all()


def test_mixed_batch_of_prefill_and_single_tokens():
    case(2, 4, 128, 16, [700, 90, 1, 3000, 65], n_q=[1, 90, 1, 1, 33])
    case(8, 4, 128, 16, [300] * 70, n_q=[1, 40] * 35)


@pytest.mark.parametrize("dim,n_q", [(64, [4]), (128, [4]), (64, [70]), (128, [70]), (256, [30])])
def test_nonfinite_values_reach_only_the_rows_that_see_them(dim, n_q):
    t = 200
    pool = R.make_pool(1, 2, dim, 16, 64)
    rows = R.rand((1, 2, t, 2, dim), 5)
    first = t - n_q[0]
    rows[0, 1, t - 1, 0, 3] = math.inf       # seen by the last row only
    rows[0, 1, t - 2, 1, 5] = math.nan
    rows[0, 1, first + 1, 0, 7] = -math.inf  # seen by all rows but the first
    rows[0, 0, t - 1, 1, :] = math.nan       # a key
    c = R.add_ctx(pool, t, 0, rows)
    q = R.rand((n_q[0], 4, dim), 6, scale=2.0)
    out, lse = run_attend(pool, [c], n_q, q)
    assert torch.isfinite(out[0]).all()
    assert (out[1:, :2, 7] == -math.inf).all()
    assert torch.isfinite(out[:-2, 2:]).all() and torch.isnan(out[-2:, 2:, 5]).all()
    assert torch.isfinite(out[:-1, :2, 3]).all() and (out[-1, :2, 3] == math.inf).all()
    assert torch.isnan(out[-1, 2:]).all() and torch.isnan(lse[-1, 2:]).all()
    clean = rows.clone()
    clean[0, :, t - 2:] = 0
    clean[0, 1, first + 1, 0, 7] = 0
    ref = R.attend_ref([R.Ctx(0, clean)], n_q, q)
    keep = torch.ones(out.shape[-1], dtype=torch.bool, device="cuda")
    keep[7] = False
    part = (out[:-2, :, keep], lse[:-2])
    R.check_attend(part, (ref[0][:-2, :, keep], ref[1][:-2], ref[2][:-2, :, keep], ref[3]), torch.bfloat16, dim, p_rounded=n_q[0] > 16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,n_q,t,opts", [(64, 1, 40, {}), (128, 1, 40, {}), (128, 1, 5000, {}), (256, 1, 40, {}), (128, 4, 300, {}),
                                            (128, 1, 300, dict(softcap=20.0)), (64, 90, 300, {}), (96, 90, 300, {})])
def test_an_infinite_value_that_is_seen_is_infinite(dim, n_q, t, opts, dtype):
    pool = R.make_pool(1, 2, dim, 16, 400, dtype=dtype)
    rows = R.rand((1, 2, t, 2, dim), 5, dtype)
    rows[0, 1, 3, 0, 3] = math.inf
    rows[0, 1, 20, 1, 5] = -math.inf
    rows[0, 1, 21, 1, 6], rows[0, 1, 22, 1, 6] = -math.inf, math.inf
    c = R.add_ctx(pool, t, 0, rows)
    q = R.rand((n_q, 4, dim), 6, dtype, 0.5)
    out, lse = run_attend(pool, [c], [n_q], q, **opts)
    assert (out[:, :2, 3] == math.inf).all() and (out[:, 2:, 5] == -math.inf).all() and torch.isnan(out[:, 2:, 6]).all()
    R.check_attend((out, lse), R.attend_ref([c], [n_q], q, **opts), dtype, dim, p_rounded=n_q * 2 > 8)


@pytest.mark.parametrize("dim,n_q,t", [(64, 1, 40), (128, 1, 40), (128, 1, 5000), (256, 1, 40), (128, 4, 300), (64, 90, 300), (128, 90, 3000),
                                       (96, 90, 300), (96, 90, 3000)])
def test_a_row_of_scores_of_minus_infinity_is_zero(dim, n_q, t):
    """Also where values are infinite: no weight is left to multiply them."""
    pool = R.make_pool(1, 2, dim, 16, 400)
    rows = R.rand((1, 2, t, 2, dim), 5)
    rows[0, 0, :, 0, 0] = -math.inf
    rows[0, 1, 3:40:7, 0, 2] = math.inf
    c = R.add_ctx(pool, t, 0, rows)
    q = R.rand((n_q, 4, dim), 6)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    out, lse = run_attend(pool, [c], [n_q], q)
    assert (out[:, :2] == 0).all() and (lse[:, :2] == -math.inf).all()
    assert torch.isfinite(out[:, 2:]).all() and torch.isfinite(lse[:, 2:]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("opts", [{}, dict(softcap=30.0)])
def test_nonfinite_values_in_split_ranges(dim, opts):
    t, n_q = 3000, 70
    pool = R.make_pool(1, 1, dim, 16, 200)
    rows = R.rand((1, 2, t, 1, dim), 5)
    rows[0, 1, t - 1, 0, 3] = math.nan
    rows[0, 1, t - 40, 0, 7] = math.inf
    c = R.add_ctx(pool, t, 0, rows)
    q = R.rand((n_q, 2, dim), 6, scale=2.0)
    out, lse = run_attend(pool, [c], [n_q], q, **opts)
    assert torch.isfinite(out[:-1, :, 3]).all() and torch.isnan(out[-1, :, 3]).all()
    assert torch.isfinite(out[:n_q - 40, :, 7]).all() and (out[n_q - 40:, :, 7] == math.inf).all()
    clean = rows.clone()
    clean[0, 1, t - 1, 0, 3] = clean[0, 1, t - 40, 0, 7] = 0
    keep = [i for i in range(dim) if i not in (3, 7)]
    ref = R.attend_ref([R.Ctx(0, clean)], [n_q], q, **opts)
    R.check_attend((out[:, :, keep], lse), (ref[0][:, :, keep], ref[1], ref[2][:, :, keep], ref[3]), torch.bfloat16, dim, True)


def test_layers_blocks_shared_by_forks_and_repeated_contexts():
    pool = R.make_pool(3, 2, 64, 16, 256)
    root = R.add_ctx(pool, 333, 1)
    st, kids = pool.fork(root.handle, 3)
    assert st == 0
    tails = [R.rand((3, 2, 10 + i, 2, 64), 50 + i) for i in range(3)]
    assert pool.append(kids, [10, 11, 12], tails)[0] == 0
    ctxs = [R.Ctx(h, torch.cat((root.rows, t), 2)) for h, t in zip(kids, tails)] + [root]
    ctxs += [ctxs[0], root]
    n_q = [1, 5, 2, 1, 3, 40]
    for layer in range(3):
        q = R.rand((sum(n_q), 8, 64), layer, scale=2.0)
        got = run_attend(pool, ctxs, n_q, q, layer=layer)
        R.check_attend(got, R.attend_ref(ctxs, n_q, q, layer=layer), torch.bfloat16, 64, True)


@pytest.mark.parametrize("opts", [{}, dict(softcap=20.0), dict(slopes=True), dict(window=700)])
@pytest.mark.parametrize("dim,heads,group", [(128, 8, 4), (64, 8, 2)])
def test_forked_contexts_read_their_shared_blocks_together(dim, heads, group, opts):
    if opts.get("slopes"):
        opts = dict(opts, slopes=2.0 ** (-8.0 * torch.arange(1, heads * group + 1, device="cuda") / (heads * group)))
    pool = R.make_pool(1, heads, dim, 16, 1200, max_ctx=64)
    root = R.add_ctx(pool, 2100, 1)
    alone = R.add_ctx(pool, 777, 2)
    st, kids = pool.fork(root.handle, 9)
    assert st == 0
    own = [1, 2, 5, 16, 17, 300, 33, 64, 4]
    tails = [R.rand((1, 2, t, heads, dim), 60 + i) for i, t in enumerate(own)]
    assert pool.append(kids[:9], own, tails)[0] == 0
    ctxs = [R.Ctx(h, torch.cat((root.rows, t), 2)) for h, t in zip(kids, tails)]
    st, more = pool.fork(ctxs[5].handle, 7)  # a second generation, without tokens of its own
    assert st == 0
    ctxs += [R.Ctx(h, ctxs[5].rows) for h in more] + [alone, root]
    order = [3, 17, 0, 9, 10, 16, 11, 1, 2, 4, 12, 5, 13, 6, 7, 14, 8, 15, 3]
    batch = [ctxs[i] for i in order]
    for n_q in ([1] * len(batch), [1 + i % 2 for i in range(len(batch))], [1] * 10 + [40] + [1] * (len(batch) - 11)):
        n_q = [min(a, len(c)) for a, c in zip(n_q, batch)]
        q = R.rand((sum(n_q), heads * group, dim), sum(n_q), scale=2.0)
        got = run_attend(pool, batch, n_q, q, **opts)
        R.check_attend(got, R.attend_ref(batch, n_q, q, **opts), torch.bfloat16, dim, True)
        again = run_attend(pool, batch, n_q, q, **opts)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_forked_contexts_more_than_kernel_parameters_hold():
    pool = R.make_pool(1, 8, 64, 16, 800, max_ctx=120)
    root = R.add_ctx(pool, 1030, 1)
    st, kids = pool.fork(root.handle, 100)
    tails = [R.rand((1, 2, 1 + i % 7, 8, 64), 60 + i) for i in range(100)]
    assert pool.append(kids, [1 + i % 7 for i in range(100)], tails)[0] == 0
    ctxs = [R.Ctx(h, torch.cat((root.rows, t), 2)) for h, t in zip(kids, tails)]
    q = R.rand((100, 16, 64), 3, scale=2.0)
    got = run_attend(pool, ctxs, [1] * 100, q)
    R.check_attend(got, R.attend_ref(ctxs, [1] * 100, q), torch.bfloat16, 64, True)


def test_nonfinite_values_of_shared_blocks_reach_the_forks():
    pool = R.make_pool(1, 8, 128, 16, 400)
    rows = R.rand((1, 2, 1600, 8, 128), 5)
    rows[0, 1, 1599, 0, 3] = math.inf
    rows[0, 1, 700, 1, 4] = math.nan
    root = R.add_ctx(pool, 1600, 0, rows)
    st, kids = pool.fork(root.handle, 6)
    assert pool.reserve(kids[:3], [1, 1, 1])[0] == 0
    kv = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda")
    assert pool.store(0, kids[:3], [1, 1, 1], kv, kv)[0] == 0
    q = R.rand((6, 32, 128), 6, scale=2.0)
    st, (out, lse) = pool.attend(0, kids, None, q)
    assert st == 0
    assert (out[:, :4, 3] == math.inf).all() and torch.isnan(out[:, 4:8, 4]).all() and torch.isfinite(lse).all()
    rest = out.clone()
    rest[:, :4, 3], rest[:, 4:8, 4] = 0, 0
    assert torch.isfinite(rest).all()
    # two queries each, the first of them before the last shared token
    st, (out, lse) = pool.attend(0, kids[3:], [2, 2, 2], q)
    assert st == 0 and torch.isfinite(out[0::2, :4, 3]).all() and (out[1::2, :4, 3] == math.inf).all()


def test_strided_queries_and_same_bits_again():
    pool = R.make_pool(1, 2, 64, 16, 256)
    ctxs = [R.add_ctx(pool, t, t) for t in (100, 901)]
    fused = R.rand((41, 12 * 64), 3, scale=2.0)
    q = fused[:, 128:128 + 8 * 64].unflatten(1, (8, 64))
    first = run_attend(pool, ctxs, [1, 40], q)
    R.check_attend(first, R.attend_ref(ctxs, [1, 40], q), torch.bfloat16, 64, True)
    for _ in range(3):
        again = run_attend(pool, ctxs, [1, 40], q)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_workspace_that_another_pool_has_used():
    """The first call of a pool meets values that the 256-row kernel cannot keep apart and leaves its mark in the workspace:
    the first call of the next pool with the same workspace does not take it for its own."""
    dim, t, n_q = 64, 300, 90
    q = R.rand((n_q, 4, dim), 6, scale=2.0)
    pools, ctxs = [], []
    for i in range(2):
        pool = R.make_pool(1, 2, dim, 16, 64)
        rows = R.rand((1, 2, t, 2, dim), 5 + i)
        if i == 0:
            rows[0, 1, t - 1, 0, 3] = math.inf
        pools.append(pool)
        ctxs.append(R.add_ctx(pool, t, 0, rows))
    ws = torch.zeros(B.aaf_kv_attend_workspace_bytes(pools[0].h), dtype=torch.uint8, device="cuda")
    fresh = R.make_pool(1, 2, dim, 16, 64)
    want = run_attend(fresh, [R.add_ctx(fresh, t, 0, ctxs[1].rows)], [n_q], q)
    for i in range(2):
        pools[i]._attend_ws = ws
        got = run_attend(pools[i], [ctxs[i]], [n_q], q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_calls_on_two_streams_share_the_workspace():
    pool = R.make_pool(1, 8, 128, 16, 700)
    ctxs = [R.add_ctx(pool, 5000, 1), R.add_ctx(pool, 4100, 2)]
    qs = [R.rand((1, 32, 128), 10 + i, scale=2.0) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for rep in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                st, got = pool.attend(0, [ctxs[i].handle], None, qs[i])
                assert st == 0
                outs.append(got)
    torch.cuda.synchronize()
    for i in range(2):
        R.check_attend(outs[i], R.attend_ref([ctxs[i]], [1], qs[i]), torch.bfloat16, 128, False)
        for rep in range(10):
            assert torch.equal(outs[i][0], outs[2 * rep + i][0])


def test_evicting_and_reusing_a_handle_waits_for_the_attention_that_reads_it():
    pool = R.make_pool(1, 8, 128, 16, 1100)
    big = R.add_ctx(pool, 16000, 1)
    q = R.rand((1, 64, 128), 4, scale=2.0)
    want = run_attend(pool, [big], [1], q)[0]
    spare = R.rand((1, 2, 500, 8, 128), 9)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(side):
            for _ in range(4):
                st, got = pool.attend(0, [big.handle], None, q)
            assert pool.evict([big.handle])[0] == 0
            st, h = pool.imp(spare, 500)  # the same handle: its table row is written again
            assert st == 0 and h == big.handle
            assert pool.evict([h])[0] == 0
            st, h = pool.imp(big.rows, 16000)
            assert st == 0 and h == big.handle
        torch.cuda.synchronize()
        assert torch.equal(got[0], want)


# ------------------------------------------------------------------------------------------ store
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,rot,inter", [(64, 64, False), (128, 128, False), (128, 64, True), (96, 24, False), (64, 10, False),
                                           (64, 14, True), (128, 0, False), (80, 80, False), (8, 2, True)])
def test_store_rotates_and_writes_only_its_slots(dim, rot, inter, dtype):
    layers, heads, group, block = 2, 3, 2, 16
    pool = R.make_pool(layers, heads, dim, block, 128, dtype=dtype)
    lens, new = [100, 7, 33, 16], [1, 7, 20, 16]
    handles = [R.add_ctx(pool, t, t).handle for t in lens]
    before = pool.mem.clone()
    total = sum(new)
    q, k, v = (R.rand((total, h, dim), 20 + i, dtype) for i, h in enumerate((heads * group, heads, heads)))
    inv = torch.tensor(B.rope_freqs(max(rot, 2), 10000.0)[0][:rot // 2], dtype=torch.float64, device="cuda")
    rope = B.Rope(rot, inv, interleaved=inter, mscale=1.25)
    for far in (False, True):
        idx = torch.tensor([t - n + j for t, n in zip(lens, new) for j in range(n)], device="cuda")
        pos = idx * 1000 + 2 ** 33 + 7 if far else idx
        q_out = torch.empty_like(q)
        st, _ = pool.store(1, handles, new, k, v, q=q, q_out=q_out, rope=rope, pos=pos if far else None)
        assert st == 0
        torch.cuda.synchronize()
        want = before.double()
        kr, qr = R.rotate_ref(k, pos, inv, rot, inter, 1.25), R.rotate_ref(q, pos, inv, rot, inter, 1.25)
        stored = torch.zeros(pool.mem.shape[1:4], dtype=torch.bool, device="cuda")
        at = 0
        for h, t, n in zip(handles, lens, new):
            table = torch.tensor(pool.table(h).tolist(), device="cuda")
            slot = torch.arange(t - n, t, device="cuda")
            want[1, table[slot // block], 0, slot % block] = kr[at:at + n]
            want[1, table[slot // block], 1, slot % block] = v[at:at + n].double()
            stored[table[slot // block], :, slot % block] = True
            at += n
        # half a step of the result, and the angle's rounding to 32 bits (half turns below 1: 2^-24 * pi) plus that of sine,
        # cosine (2 * 2^-23 each) and the sum's two products (2 * 2^-24) on |a| + |b|
        h = R.half_step(dtype)
        slack = 1.25 * (math.pi * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23) * 2

        def near(got, ref, raw):
            lim = h * ref.abs() + slack * raw.abs().amax(-1, keepdim=True).double() * (1 + h) + 1e-7 * (dtype == torch.float16)
            assert ((got.double() - ref).abs() <= lim).all()

        near(q_out, qr, q)
        got = pool.mem.double()
        assert torch.equal(pool.mem[0].view(torch.int16), before[0].view(torch.int16))
        assert torch.equal(pool.mem[1][~stored].view(torch.int16), before[1][~stored].view(torch.int16))
        near(got[1, :, 0][stored[:, 0]], want[1, :, 0][stored[:, 0]], want[1, :, 0][stored[:, 0]])
        assert torch.equal(got[1, :, 1][stored[:, 1]], want[1, :, 1][stored[:, 1]])
    # in place, and from views into a fused projection
    fused = torch.cat((q.flatten(1), k.flatten(1), v.flatten(1)), 1).contiguous()
    a, b = q[0].numel(), k[0].numel()
    fq, fk, fv = fused[:, :a].unflatten(1, q.shape[1:]), fused[:, a:a + b].unflatten(1, k.shape[1:]), fused[:, a + b:].unflatten(1, v.shape[1:])
    keep = pool.mem.clone()
    assert pool.store(1, handles, new, fk, fv, q=fq, rope=rope, pos=pos)[0] == 0
    torch.cuda.synchronize()
    assert torch.equal(fq, q_out) and torch.equal(pool.mem.view(torch.int16), keep.view(torch.int16))
    assert torch.equal(fk, k) and torch.equal(fv, v)


def test_store_odd_shapes_of_tokens():
    """Wide heads, many of them, and a single token whose stride is never used."""
    pool = R.make_pool(1, 2, 1032, 8, 16, fill=0.0)
    c = R.add_ctx(pool, 9, 1)
    q, k, v = R.rand((1, 700, 1032), 2), R.rand((1, 2, 1032), 3), R.rand((1, 2, 1032), 4)
    inv = 10000.0 ** (-torch.arange(0, 512, dtype=torch.float64, device="cuda") / 512)
    odd = torch.as_strided(k, (1, 2, 1032), (13, 1032, 1))
    out = torch.empty_like(q)
    assert pool.store(0, [c.handle], [1], odd, v, q=q, q_out=out, rope=B.Rope(1024, inv))[0] == 0
    torch.cuda.synchronize()
    pos = torch.tensor([8], device="cuda")
    slot = pool.mem[0, pool.table(c.handle).tolist()[1], :, 0]
    slack = (math.pi * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23) * 2  # as in the test above
    for got, x in ((out[0], q), (slot[0], k)):
        ref = R.rotate_ref(x, pos, inv, 1024, False, 1.0)[0]
        lim = 2.0 ** -8 * ref.abs() + slack * x.double().abs().amax() * (1 + 2.0 ** -8)
        assert ((got.double() - ref).abs() <= lim).all()
    assert torch.equal(slot[1], v[0])
    d = B.aaf_kv_store_desc(C.sizeof(B.aaf_kv_store_desc), 0, 2 ** 28, 0, 0, 1.0, None, None, q.data_ptr(), q.data_ptr(), k.data_ptr(),
                            v.data_ptr(), 2 ** 40, 2 ** 40, 2064, 2064)
    h, one = (C.c_int32 * 1)(c.handle), (C.c_int32 * 1)(1)
    assert B.aaf_kv_store(pool.h, 0, d, 1, h, one, None) == B.AAF_ERR_INVALID_ARG


def test_store_many_sequences_and_long_prefill():
    pool = R.make_pool(1, 2, 64, 16, 700, max_ctx=80)
    n = 70
    handles = [R.add_ctx(pool, 20 + i, i).handle for i in range(n)]
    k, v = R.rand((n, 2, 64), 1), R.rand((n, 2, 64), 2)
    assert pool.store(0, handles, [1] * n, k, v)[0] == 0
    torch.cuda.synchronize()
    for i, h in enumerate(handles):
        tab, t = pool.table(h), 19 + i
        assert torch.equal(pool.mem[0, int(tab[t // 16]), 0, t % 16], k[i]) and torch.equal(pool.mem[0, int(tab[t // 16]), 1, t % 16], v[i])
    long = R.add_ctx(pool, 5003, 9)
    k, v = R.rand((5003, 2, 64), 3), R.rand((5003, 2, 64), 4)
    assert pool.store(0, [long.handle], [5003], k, v)[0] == 0
    st, buf = pool.materialize(long.handle, 0, 5003)
    torch.cuda.synchronize()
    got = buf.view(torch.bfloat16).view(2, 5003, 2, 64)
    assert torch.equal(got[0], k) and torch.equal(got[1], v)


def test_store_refuses_slots_that_other_contexts_share():
    pool = R.make_pool(1, 2, 64, 16, 128)
    root = R.add_ctx(pool, 37, 1)
    k, v = R.rand((8, 2, 64), 1), R.rand((8, 2, 64), 2)
    assert pool.store(0, [root.handle], [8], k, v)[0] == 0
    st, kids = pool.fork(root.handle, 2)
    before = pool.mem.clone()
    for h in [root.handle] + kids:
        assert pool.store(0, [h], [8], k, v)[0] == B.AAF_ERR_INVALID_ARG
        assert pool.store(0, [h], [1], k[:1], v[:1])[0] == B.AAF_ERR_INVALID_ARG
    assert pool.reserve(kids, [3, 5])[0] == 0
    assert pool.store(0, kids, [3, 5], k, v)[0] == 0
    assert pool.store(0, kids[:1], [4], k[:4], v[:4])[0] == B.AAF_ERR_INVALID_ARG
    st, merged = pool.compose([kids[0], kids[1]])
    assert st == 0
    assert pool.store(0, [merged], [1], k[:1], v[:1])[0] == B.AAF_ERR_INVALID_ARG
    assert pool.store(0, [kids[1]], [1], k[:1], v[:1])[0] == B.AAF_ERR_INVALID_ARG
    st, copy = pool.compose([kids[0], kids[1]], B.AAF_COMPOSE_COPY_ALL)
    assert pool.store(0, [copy], [8], k, v)[0] == 0
    st, buf = pool.materialize(root.handle, 0, 37)
    torch.cuda.synchronize()
    want = root.rows.clone()
    want[0, 0, 29:], want[0, 1, 29:] = k, v
    assert torch.equal(buf.view(torch.bfloat16).view(want.shape), want)  # the parent's rows are what they were
    del before


# ------------------------------------------------------------------------------------------ reserve
def test_reserve_grows_like_append_and_copies_a_shared_tail():
    a, b = R.make_pool(2, 2, 64, 16, 96, fill=0.0), R.make_pool(2, 2, 64, 16, 96, fill=0.0)
    for pool in (a, b):
        root = R.add_ctx(pool, 37, 1)
        pool.kids = pool.fork(root.handle, 10)[1]
    new = [1 + 3 * i for i in range(10)]
    zero = torch.zeros(2 * 2 * 2 * 64 * 40, dtype=torch.bfloat16, device="cuda")
    assert a.append(a.kids, new, [zero] * 10)[0] == 0 and b.reserve(b.kids, new)[0] == 0
    torch.cuda.synchronize()
    for h in a.kids:
        assert a.table(h).tolist() == b.table(h).tolist()
    assert a.refcounts().tolist() == b.refcounts().tolist() and a.free_list().tolist() == b.free_list().tolist()
    assert torch.equal(a.mem, b.mem)
    assert a.stats()["cow_count"] == b.stats()["cow_count"] == 10
    assert b.reserve(b.kids[:1], [0])[0] == B.AAF_ERR_INVALID_ARG
    assert b.reserve([b.kids[0]] * 2, [1, 1])[0] == B.AAF_ERR_INVALID_ARG
    assert b.reserve(b.kids[:1], [100000])[0] == B.AAF_ERR_TOO_LONG
    assert b.reserve(b.kids, [150] * 10)[0] == B.AAF_ERR_OOM_BLOCKS


# ------------------------------------------------------------------------------------------ mass
@pytest.mark.parametrize("heads,group,dim,block,n_q", [(2, 4, 64, 16, [1, 1, 1]), (8, 4, 128, 16, [1, 3, 32]), (3, 5, 96, 8, [7, 1, 20]),
                                                       (1, 1, 256, 16, [1, 9, 2])])
@pytest.mark.parametrize("opts", [{}, dict(softcap=20.0), dict(window=90, slopes=True)])
def test_mass(heads, group, dim, block, n_q, opts):
    if opts.get("slopes"):
        opts = dict(opts, slopes=2.0 ** (-8.0 * torch.arange(1, heads * group + 1, device="cuda") / (heads * group)))
    lens = [65, 700, 131]
    pool = R.make_pool(1, heads, dim, block, sum(-(-t // block) for t in lens) + 2)
    ctxs = [R.add_ctx(pool, t, t) for t in lens]
    hs = [c.handle for c in ctxs]
    q = R.rand((sum(n_q), heads * group, dim), 3, scale=2.0)
    _, lse, _, big = R.attend_ref(ctxs, n_q, q, **opts)
    lse = lse.float()
    prev = torch.rand(3, 710, device="cuda")
    want = R.mass_ref(ctxs, n_q, q, lse, prev, **opts)
    # each weight is off by the score's error (see check_attend) and the exponential's; sums of at most n rows add n * 2^-24
    ds = dim * 2.0 ** -23 * big + 16 * 2.0 ** -24 * (big + 16)
    for in_place in (False, True):
        mass = prev.clone() if in_place else torch.full_like(prev, -7.0)
        st, _ = pool.attn_mass(0, hs, n_q, q, lse, mass, prev=mass if in_place else prev, **opts)
        assert st == 0
        torch.cuda.synchronize()
        for i, t in enumerate(lens):
            rows = n_q[i] * heads * group
            lim = (ds + 2.0 ** -22 + rows * 2.0 ** -24) * want[i] + 1e-30
            assert ((mass[i, :t].double() - want[i]).abs() <= lim).all()
            assert torch.equal(mass[i, t:], prev[i, t:] if in_place else torch.full_like(prev, -7.0)[i, t:])
    again = torch.empty_like(prev)
    other = torch.empty_like(prev)
    assert pool.attn_mass(0, hs, n_q, q, lse, again, **opts)[0] == 0 and pool.attn_mass(0, hs, n_q, q, lse, other, **opts)[0] == 0
    torch.cuda.synchronize()
    for i, t in enumerate(lens):
        assert torch.equal(again[i, :t], other[i, :t])
        assert abs(float(again[i, :t].double().sum()) - n_q[i] * heads * group) < 1e-3 * n_q[i] * heads * group  # each row gives one


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,heads,group,block,n_q", [(128, 8, 4, 16, [32, 5, 100]), (64, 2, 3, 8, [43, 6, 131]), (128, 1, 32, 64, [1, 3, 9]),
                                                       (64, 4, 1, 128, [17, 128, 1])])
@pytest.mark.parametrize("opts", [{}, dict(softcap=20.0), dict(window=300, slopes=True)])
def test_mass_of_many_rows(dim, heads, group, block, n_q, opts, dtype):
    if opts.get("slopes"):
        opts = dict(opts, slopes=2.0 ** (-8.0 * torch.arange(1, heads * group + 1, device="cuda") / (heads * group)))
    lens = [1501, 300, 140]
    pool = R.make_pool(2, heads, dim, block, sum(-(-t // block) for t in lens) + 2, dtype=dtype)
    ctxs = [R.add_ctx(pool, t, t) for t in lens]
    hs = [c.handle for c in ctxs]
    q = R.rand((sum(n_q), heads * group, dim), 3, dtype, 2.0)
    _, lse, _, big = R.attend_ref(ctxs, n_q, q, layer=1, **opts)
    lse = lse.float()
    lse[1] = -math.inf  # a row that is said to have seen nothing
    prev = torch.rand(3, 1600, device="cuda")
    want = R.mass_ref(ctxs, n_q, q, lse, prev, layer=1, **opts)
    ds = dim * 2.0 ** -23 * big + 16 * 2.0 ** -24 * (big + 16)
    mass, again = torch.full_like(prev, -7.0), torch.full_like(prev, -7.0)
    assert pool.attn_mass(1, hs, n_q, q, lse, mass, prev=prev, **opts)[0] == 0
    assert pool.attn_mass(1, hs, n_q, q, lse, again, prev=prev, **opts)[0] == 0
    torch.cuda.synchronize()
    assert pool.sync_status() == 0 and torch.equal(mass, again)
    for i, t in enumerate(lens):
        lim = (ds + 2.0 ** -22 + n_q[i] * heads * group * 2.0 ** -24) * want[i] + 1e-30
        assert ((mass[i, :t].double() - want[i]).abs() <= lim).all()
        assert (mass[i, t:] == -7.0).all()


@pytest.mark.parametrize("dim,group,n_q", [(64, 4, 1), (128, 4, 1), (256, 3, 1), (128, 4, 5), (64, 3, 50)])
def test_mass_of_a_key_of_minus_infinity(dim, group, n_q):
    """Every row's score is -inf there: the key gets nothing, also where rows do not fill a tile."""
    pool = R.make_pool(1, 2, dim, 16, 64)
    rows = R.rand((1, 2, 700, 2, dim), 5)
    rows[0, 0, 7, :, 0] = -math.inf
    c = R.add_ctx(pool, 700, 0, rows)
    q = R.rand((n_q, 2 * group, dim), 6)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    out, lse = run_attend(pool, [c], [n_q], q)
    mass = torch.full((1, 700), 3.0, device="cuda")
    assert pool.attn_mass(0, [c.handle], [n_q], q, lse, mass)[0] == 0
    torch.cuda.synchronize()
    total = 2 * group * n_q
    assert torch.isfinite(out).all() and float(mass[0, 7]) == 0.0 and abs(float(mass.double().sum()) - total) < 1e-3 * total


def test_mass_with_spans_and_rows_that_see_nothing():
    pool = R.make_pool(1, 2, 64, 16, 64)
    c = R.add_ctx(pool, 300, 1)
    spans = torch.tensor([[0, 50], [7, 7], [100, 300], [60, 20]], dtype=torch.int32, device="cuda")
    q = R.rand((4, 4, 64), 2, scale=2.0)
    out, lse = run_attend(pool, [c], [4], q, spans=spans)
    mass = torch.full((1, 300), 5.0, device="cuda")
    assert pool.attn_mass(0, [c.handle], [4], q, lse, mass, spans=spans)[0] == 0
    torch.cuda.synchronize()
    want = R.mass_ref([c], [4], q, lse, spans=spans)[0]
    assert ((mass[0].double() - want).abs() <= 1e-4 * want + 1e-12).all()
    assert (mass[0, 50:100] == 0).all() and abs(float(mass.sum()) - 8) < 1e-3
    assert pool.attn_mass(0, [c.handle], [4], q, lse, mass[:, :200], spans=spans)[0] == B.AAF_ERR_DST_TOO_SMALL


# ------------------------------------------------------------------------------------------ prune
@pytest.mark.parametrize("tokens,budget,sink,recent", [(1, 1, 0, 0), (50, 50, 3, 4), (50, 1, 0, 0), (50, 1, 1, 0), (50, 1, 0, 1),
                                                       (300, 100, 4, 32), (300, 36, 4, 32), (300, 299, 0, 0), (5000, 1234, 4, 100),
                                                       (4096, 4095, 7, 0)])
@pytest.mark.parametrize("kind", ["random", "ties", "odd"])
def test_prune(tokens, budget, sink, recent, kind):
    pool = R.make_pool(2, 3, 16, 16, 2 * (-(-tokens // 16)) + 3)
    c = R.add_ctx(pool, tokens, tokens)
    g = torch.Generator(device="cuda").manual_seed(tokens + budget)
    s = torch.randn(tokens, generator=g, device="cuda")
    if kind == "ties":
        s = (s * 2).round() / 2
        s[::5] = -0.0
    if kind == "odd":
        s[::7], s[1::7], s[2::7], s[3::11] = math.nan, -math.inf, math.inf, 1e-42
    kept = torch.full((budget,), -1, dtype=torch.int32, device="cuda")
    ks = torch.zeros(budget, device="cuda")
    st, h = pool.prune(c.handle, s, budget, sink=sink, recent=recent, kept=kept, kept_scores=ks)
    assert st == 0 and pool.ctx_len(h) == budget
    want = R.prune_ref(s.tolist(), budget, sink, recent)
    assert kept.tolist() == want
    assert torch.equal(ks.view(torch.int32), s[kept.long()].view(torch.int32))
    st, buf = pool.materialize(h, 0, budget)
    st2, old = pool.materialize(c.handle, 0, tokens)
    torch.cuda.synchronize()
    assert pool.sync_status() == 0
    assert torch.equal(buf.view(torch.bfloat16).view(2, 2, budget, 3, 16), c.rows[:, :, kept.long()])
    assert torch.equal(old.view(torch.bfloat16).view(c.rows.shape), c.rows)
    cat = pool.export_catalog()
    torch.cuda.synchronize()
    assert cat["origin"].tolist() == [1, 4] and cat["parent"].tolist() == [-1, c.handle]
    assert pool.evict([c.handle])[0] == 0 and pool.evict([h])[0] == 0
    assert len(pool.free_list()) == pool.NB and (pool.refcounts() == 0).all()


def test_prune_then_reuse_of_the_evicted_blocks_waits_for_the_gather():
    pool = R.make_pool(8, 8, 128, 16, 700)
    c = R.add_ctx(pool, 8000, 1)
    s = torch.rand(8000, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        st, h = pool.prune(c.handle, s, 2000, sink=4, recent=64)
        assert st == 0 and pool.evict([c.handle])[0] == 0
        st, x = pool.imp(torch.zeros(8 * 2 * 8000 * 8 * 128, dtype=torch.bfloat16, device="cuda"), 8000)
        assert st == 0
        st, buf = pool.materialize(h, 0, 2000)
    torch.cuda.synchronize()
    kept = R.prune_ref(s.tolist(), 2000, 4, 64)
    assert torch.equal(buf.view(torch.bfloat16).view(8, 2, 2000, 8, 128), c.rows[:, :, kept])


def test_prune_refusals_change_nothing():
    pool = R.make_pool(1, 2, 64, 16, 12, max_ctx=3)
    c = R.add_ctx(pool, 100, 1)
    s = torch.rand(100, device="cuda")
    for kw in (dict(budget=0), dict(budget=101), dict(budget=10, sink=-1), dict(budget=10, recent=-1), dict(budget=10, sink=6, recent=5),
               dict(budget=10, sink=11)):
        assert pool.prune(c.handle, s, **kw)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.prune(c.handle, s, 96)[0] == B.AAF_ERR_OOM_BLOCKS
    assert pool.prune(2, s, 10)[0] == B.AAF_ERR_BAD_CTX
    R.add_ctx(pool, 3, 2), R.add_ctx(pool, 3, 3)
    assert pool.prune(c.handle, s, 10)[0] == B.AAF_ERR_OOM_CTX
    assert pool.stats()["live_ctx"] == 3 and pool.stats()["free_blocks"] == 12 - 7 - 2
    with pytest.raises(ValueError):
        pool.prune(c.handle, s[:50], 10)


# ------------------------------------------------------------------------------------------ refusals
def test_attend_refusals():
    pool = R.make_pool(1, 2, 64, 16, 32)
    c = R.add_ctx(pool, 100, 1)
    q = R.rand((1, 4, 64), 1)
    ok = lambda **kw: pool.attend(kw.pop("layer", 0), kw.pop("ctxs", [c.handle]), kw.pop("n_q", None), kw.pop("q", q), **kw)[0]
    assert ok() == 0
    assert ok(layer=1) == ok(layer=-1) == B.AAF_ERR_INVALID_ARG
    assert ok(ctxs=[5]) == B.AAF_ERR_BAD_CTX
    assert ok(scale=math.nan) == ok(scale=math.inf) == ok(softcap=-1.0) == ok(window=-1) == B.AAF_ERR_INVALID_ARG
    assert ok(q=R.rand((101, 4, 64), 1), n_q=[101]) == B.AAF_ERR_INVALID_ARG
    assert ok(q=R.rand((0, 4, 64), 1), n_q=[0]) == B.AAF_ERR_INVALID_ARG
    assert ok(q=R.rand((1, 3, 64), 1)) == B.AAF_ERR_INVALID_ARG
    for bad in (q.float(), q[:, :, :32], q.cpu(), R.rand((2, 4, 64), 1), R.rand((1, 64, 4), 1).transpose(1, 2)):
        with pytest.raises(ValueError):
            ok(q=bad)
    with pytest.raises(ValueError):
        ok(slopes=torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError):
        ok(spans=torch.zeros(1, 2, dtype=torch.int64, device="cuda"))
    # misaligned queries, a workspace that is too small
    a = B.aaf_kv_attn(C.sizeof(B.aaf_kv_attn), 0, 4, 0, 0.1, 0.0, None, None, 256)
    one = (C.c_int32 * 1)(c.handle)
    out, ws = torch.empty_like(q), torch.empty(1024, dtype=torch.uint8, device="cuda")
    call = lambda qp, n_ws: B.aaf_kv_attend(pool.h, 0, C.byref(a), 1, one, None, qp, out.data_ptr(), None, ws.data_ptr(), n_ws, None)
    assert call(q.data_ptr() + 2, 1 << 40) == B.AAF_ERR_INVALID_ARG
    assert call(q.data_ptr(), 1024) == B.AAF_ERR_DST_TOO_SMALL
    a.struct_size = 8
    assert call(q.data_ptr(), 1 << 40) == B.AAF_ERR_INVALID_ARG
    a.struct_size, a.q_stride = C.sizeof(a), 252
    assert call(q.data_ptr(), 1 << 40) == B.AAF_ERR_INVALID_ARG
    wide = R.make_pool(1, 1, 264, 16, 8)
    w = R.add_ctx(wide, 10, 1)
    assert wide.attend(0, [w.handle], None, R.rand((1, 2, 264), 1))[0] == B.AAF_ERR_INCOMPAT
    torch.cuda.synchronize()


def test_a_cap_without_a_reciprocal_is_refused():
    pool = R.make_pool(1, 2, 64, 16, 32)
    c = R.add_ctx(pool, 20, 1)
    q = R.rand((1, 4, 64), 1)
    lse, mass = torch.zeros(1, 4, device="cuda"), torch.zeros(1, 20, device="cuda")
    for cap in (1e-40, 1e-45):
        assert pool.attend(0, [c.handle], None, q, softcap=cap)[0] == B.AAF_ERR_INVALID_ARG
        assert pool.attn_mass(0, [c.handle], None, q, lse, mass, softcap=cap)[0] == B.AAF_ERR_INVALID_ARG
    out, _ = run_attend(pool, [c], [1], q, softcap=1e-37)  # every key alike
    assert torch.isfinite(out).all()


def test_a_tiny_cap_over_many_rows():
    """Scores of zero under a cap so small that powers of its reciprocal overflow: every visible key weighs the same."""
    pool = R.make_pool(1, 2, 64, 16, 64)
    c = R.add_ctx(pool, 300, 1)
    q = torch.zeros(90, 4, 64, dtype=torch.bfloat16, device="cuda")
    got = run_attend(pool, [c], [90], q, softcap=1e-37)
    R.check_attend(got, R.attend_ref([c], [90], q), torch.bfloat16, 64, True)
    assert pool.attend(0, [c.handle], [90], q, scale=3e38)[0] == B.AAF_ERR_INVALID_ARG  # scale * log2(e) is not finite


def test_store_refusals():
    pool = R.make_pool(2, 2, 64, 16, 32)
    c = R.add_ctx(pool, 20, 1)
    k = R.rand((2, 2, 64), 1)
    inv = torch.ones(32, dtype=torch.float64, device="cuda")
    assert pool.store(2, [c.handle], [2], k, k)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.store(0, [c.handle, c.handle], [1, 1], k, k)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.store(0, [9], [2], k, k)[0] == B.AAF_ERR_BAD_CTX
    assert pool.store(0, [c.handle], [21], R.rand((21, 2, 64), 1), R.rand((21, 2, 64), 1))[0] == B.AAF_ERR_INVALID_ARG
    wide = B.Rope(66, torch.ones(33, dtype=torch.float64, device="cuda"))
    assert pool.store(0, [c.handle], [2], k, k, rope=wide)[0] == B.AAF_ERR_INVALID_ARG
    assert pool.store(0, [c.handle], [2], k, k, rope=B.Rope(64, inv, mscale=math.nan))[0] == B.AAF_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        pool.store(0, [c.handle], [2], k, k.half())
    with pytest.raises(ValueError):
        pool.store(0, [c.handle], [2], k, k, pos=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        B.Rope(64, inv.float())


def test_calls_during_capture_are_refused():
    pool = R.make_pool(1, 2, 64, 16, 32)
    c = R.add_ctx(pool, 20, 1)
    q, k = R.rand((1, 4, 64), 1), R.rand((1, 2, 64), 1)
    out, lse = run_attend(pool, [c], None or [1], q)
    s = torch.rand(20, device="cuda")
    kept = torch.empty(4, dtype=torch.int32, device="cuda")
    mass = torch.zeros(1, 20, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mass.add_(1.0)
        st = [pool.attend(0, [c.handle], None, q, out=out, lse=lse)[0], pool.store(0, [c.handle], [1], k, k)[0],
              pool.attn_mass(0, [c.handle], None, q, lse, mass)[0], pool.prune(c.handle, s, 4, kept=kept)[0]]
    assert st == [B.AAF_ERR_INVALID_ARG] * 4
    graph.replay()
    torch.cuda.synchronize()
    assert (mass == 1).all() and pool.stats()["live_ctx"] == 1
    run_attend(pool, [c], [1], q)


def test_reserve_during_capture_is_refused():
    pool = R.make_pool(1, 2, 64, 16, 32)
    c = R.add_ctx(pool, 20, 1)
    x = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1.0)
        st = pool.reserve([c.handle], [1])[0]
    assert st == B.AAF_ERR_INVALID_ARG and pool.ctx_len(c.handle) == 20
    graph.replay()
    assert pool.reserve([c.handle], [1])[0] == 0 and pool.ctx_len(c.handle) == 21
    torch.cuda.synchronize()
    assert float(x) == 1 and pool.sync_status() == 0


def test_calls_beside_a_capture_on_another_stream():
    pool = R.make_pool(1, 2, 64, 16, 32)
    c = R.add_ctx(pool, 20, 1)
    q = R.rand((1, 4, 64), 1, scale=2.0)
    out, lse = run_attend(pool, [c], [1], q)
    want = out.clone()
    x = torch.zeros(1, device="cuda")
    other = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1.0)
        with torch.cuda.stream(other):
            st = pool.attend(0, [c.handle], None, q, out=out, lse=lse)[0]
    graph.replay()
    torch.cuda.synchronize()
    assert st == 0 and float(x) == 1 and torch.equal(out, want) and pool.sync_status() == 0


def test_an_unusable_pool_refuses():
    pool = R.make_pool(1, 2, 64, 16, 32)
    c = R.add_ctx(pool, 20, 1)
    q, k = R.rand((1, 4, 64), 1), R.rand((1, 2, 64), 1)
    B.aaf_kv_debug_mark_unusable(pool.h)
    lse, mass = torch.zeros(1, 4, device="cuda"), torch.zeros(1, 20, device="cuda")
    assert pool.attend(0, [c.handle], None, q)[0] == pool.store(0, [c.handle], [1], k, k)[0] == B.AAF_ERR_CUDA
    assert pool.attn_mass(0, [c.handle], None, q, lse, mass)[0] == pool.reserve([c.handle], [1])[0] == B.AAF_ERR_CUDA
    assert pool.prune(c.handle, torch.rand(20, device="cuda"), 4)[0] == B.AAF_ERR_CUDA


# ------------------------------------------------------------------------------------------ together
def test_a_serving_loop():
    """Two layers: prefill of a prompt, a fork to three agents, decoding steps that store, attend and count what each
    cached token received, then each agent's context pruned by it and decoded on, against dense tensors in 64 bits."""
    layers, heads, group, dim, block = 2, 2, 4, 64, 16
    pool = R.make_pool(layers, heads, dim, block, 256, max_ctx=16)
    inv = torch.tensor(B.rope_freqs(dim, 10000.0, B.AAF_ROPE_LINEAR, factor=2.0)[0], dtype=torch.float64, device="cuda")
    rope = B.Rope(dim, inv)
    seed = [1000]

    def fresh(tokens):
        seed[0] += 1
        return [R.rand((tokens, h, dim), seed[0] * 7 + i) for i, h in enumerate((heads * group, heads, heads))]

    def step(ctxs, n_new, pos=None):
        """One step of all layers; ctxs' rows grow by what was stored.  Returns the last layer's outputs."""
        for c, n in zip(ctxs, n_new):
            c.rows = torch.cat((c.rows, torch.zeros(layers, 2, n, heads, dim, dtype=torch.bfloat16, device="cuda")), 2)
        for layer in range(layers):
            q, k, v = fresh(sum(n_new))
            p = torch.cat([torch.arange(len(c) - n, len(c), device="cuda") for c, n in zip(ctxs, n_new)]) if pos is None else pos
            hs = [c.handle for c in ctxs]
            raw = q.clone()
            assert pool.store(layer, hs, n_new, k, v, q=q, rope=rope, pos=pos)[0] == 0
            got = run_attend(pool, ctxs, n_new, q, layer=layer)
            kr, at = R.rotate_ref(k, p, inv, dim, False, 1.0).to(torch.bfloat16), 0
            assert (q.double() - R.rotate_ref(raw, p, inv, dim, False, 1.0)).abs().max() <= 2.0 ** -8 * 6
            for c, n in zip(ctxs, n_new):
                st, buf = pool.materialize(c.handle, len(c) - n, len(c))
                torch.cuda.synchronize()
                rows = buf.view(torch.bfloat16).view(layers, 2, n, heads, dim)[layer]
                assert (rows[0].double() - kr[at:at + n].double()).abs().max() <= 2.0 ** -7 * 6 and torch.equal(rows[1], v[at:at + n])
                c.rows[layer, :, len(c) - n:] = rows
                at += n
            R.check_attend(got, R.attend_ref(ctxs, n_new, q, layer=layer), torch.bfloat16, dim, max(n_new) * group > 32)
            for c, m in mass.items():
                i = [x.handle for x in ctxs].index(c)
                row = slice(sum(n_new[:i]), sum(n_new[:i + 1]))
                assert pool.attn_mass(layer, [c], [n_new[i]], q[row], got[1][row].contiguous(), m, prev=m)[0] == 0
        return got

    mass = {}
    empty = torch.zeros(layers, 2, 0, heads, dim, dtype=torch.bfloat16, device="cuda")
    root = R.add_ctx(pool, 1, 1)  # a context starts with a token
    assert pool.reserve([root.handle], [69])[0] == 0
    step([root], [69])
    st, kids = pool.fork(root.handle, 3)
    agents = [R.Ctx(h, root.rows.clone()) for h in kids]
    for n_new in ([1, 1, 1], [5, 1, 20], [1, 1, 1]):
        assert pool.reserve(kids, n_new)[0] == 0
        step(agents, n_new)
    for a in agents:
        mass[a.handle] = torch.zeros(1, len(a) + 1, device="cuda")
    assert pool.reserve(kids, [1, 1, 1])[0] == 0
    step(agents, [1, 1, 1])
    pruned, at = [], []
    for a in agents:
        m = mass.pop(a.handle)
        assert abs(float(m.sum()) - layers * heads * group) < 1e-3 * layers * heads * group
        kept = torch.empty(40, dtype=torch.int32, device="cuda")
        st, h = pool.prune(a.handle, m[0], 40, sink=2, recent=8, kept=kept)
        assert st == 0 and kept.tolist() == R.prune_ref(m[0].tolist(), 40, 2, 8)
        pruned.append(R.Ctx(h, a.rows[:, :, kept.long()]))
        at.append(len(a))
    assert pool.evict(kids)[0] == 0
    hs = [c.handle for c in pruned]
    for s in range(3):
        assert pool.reserve(hs, [1, 1, 1])[0] == 0
        step(pruned, [1, 1, 1], pos=torch.tensor([t + s for t in at], device="cuda"))
    assert pool.evict(hs + [root.handle])[0] == 0
    assert len(pool.free_list()) == pool.NB and pool.sync_status() == 0
    del empty
