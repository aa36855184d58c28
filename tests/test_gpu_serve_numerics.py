"""Attention where 16-bit weights, far distances and shared blocks could cost digits, against plain definitions in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

from tests import serve_reference as R

pytestmark = pytest.mark.gpu


def check_with_floor(got, ref, dtype, dim, p_rounded, keys, floor_bits, v_max):
    """check_attend's tolerance, and what the weights' own grid adds: they are held in multiples of 2^-floor_bits of a row's largest
    weight, so each is off by at most half of that, and the sum that they are divided by is at least the largest weight."""
    out, ref_out, slack, big = got[0].double(), *(ref[i] for i in (0, 2, 3))
    h = R.half_step(dtype)
    ds = dim * 2.0 ** -23 * big + 8 * 2.0 ** -24 * (big + 8)
    tol = h * ref_out.abs() + (2 * ds + (h if p_rounded else h * h) + 2.0 ** -20) * slack * (1 + h) + keys * 2.0 ** -(floor_bits + 1) * v_max
    worst = float(((out - ref_out).abs() / tol).max())
    assert worst <= 1.0, f"out: {worst:.2f} of the tolerance"
    lim = ds + 2.0 ** -22 + 4 * 2.0 ** -24 * ref[1].abs()
    assert ((got[1].double() - ref[1]).abs() <= lim).all()


# f16 weights end at 2^-24; with the largest one raised to 2^15 (2^7 where it may be outgrown by 2^8) the grid is 2^-39 (2^-31) of it
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("below", [24.6, 20.3, 15.5])
@pytest.mark.parametrize("dim,group,n_q,p_rounded,raised", [(64, 4, 1, False, 15), (128, 4, 1, False, 15), (64, 4, 4, False, 15), (64, 8, 8, True, 7),
                                                            (128, 8, 4, True, 7), (96, 8, 8, True, 15), (256, 1, 1, False, 15)])
def test_many_small_weights_beside_a_large_one(dim, group, n_q, p_rounded, raised, below, dtype):
    keys, heads, times = 4096, 8, 600  # so many that no context's keys are cut into parts, which have maxima of their own
    pool = R.make_pool(1, heads, dim, 64, keys // 64 + 2, dtype=dtype)
    rows = torch.zeros(1, 2, keys, heads, dim, device="cuda")
    rows[0, 0, 0, :, :8] = 1.0                # one key with a score, all others with none
    rows[0, 1] = R.rand((keys, heads, dim), 1, dtype).float().abs()
    rows[0, 1, 0] = 0.0                       # so that the others make the output
    c = R.add_ctx(pool, keys, 1, rows.to(dtype))
    q = torch.zeros(n_q, heads * group, dim, device="cuda", dtype=dtype)
    q[..., :8] = 1.0
    scale = below * math.log(2.0) / 8
    st, got = pool.attend(0, [c.handle] * times, [n_q] * times, q.repeat(times, 1, 1), scale=scale)
    assert st == 0
    torch.cuda.synchronize()
    assert pool.sync_status() == 0
    got = [x.view(times, n_q, *x.shape[1:]) for x in got]
    assert all(torch.equal(x, x[:1].expand_as(x)) for x in got)
    ref = R.attend_ref([c], [n_q], q, scale=scale)
    grid = 24 + raised if dtype == torch.float16 else 126  # bf16 has the exponents of 32 bits
    check_with_floor([x[0] for x in got], ref, dtype, dim, p_rounded, keys, grid, float(rows.max()))


@pytest.mark.parametrize("n_q", [1, 8])
@pytest.mark.parametrize("dim", [64, 128])
def test_bias_of_distances_that_32_bits_cannot_tell_apart(dim, n_q):
    """Rows whose span lies more than 2^24 keys behind them: neighbouring keys differ by one in distance all the same."""
    seen, far, group = 300, (1 << 24) + 1001, 8
    blocks = (seen + far) // 128 + 2
    pool = R.make_pool(1, 1, dim, 128, blocks, max_ctx=2)
    c = R.add_ctx(pool, seen, 1)
    assert pool.reserve([c.handle], [far])[0] == 0  # slots that nothing was stored in: no row sees them
    q = R.rand((n_q, group, dim), 2, scale=2.0)
    slopes = torch.linspace(0.05, 0.7, group, device="cuda")
    spans = torch.tensor([[3 * j, seen - j] for j in range(n_q)], dtype=torch.int32, device="cuda")
    st, (out, lse) = pool.attend(0, [c.handle], [n_q], q, slopes=slopes, spans=spans)
    assert st == 0
    torch.cuda.synchronize()
    assert pool.sync_status() == 0
    k, v = c.rows[0, :, :, 0].double()
    key = torch.arange(seen, device="cuda")
    refs, lses, slacks, big = [], [], [], 0.0
    for j in range(n_q):
        p = seen + far - n_q + j
        lo, hi = spans[j].tolist()
        x = q[j].double() @ k.T * dim ** -0.5
        big = max(big, float((q[j].double().abs() @ k.abs().T).max()) * dim ** -0.5)
        x = x - slopes.double()[:, None] * ((p - key) - (p - (hi - 1)))  # from the nearest key that is seen
        x = x.masked_fill((key < lo) | (key >= hi), -math.inf)
        w = torch.softmax(x, -1)
        refs.append(w @ v)
        slacks.append(w @ v.abs())
        lses.append(torch.logsumexp(x, -1) - slopes.double() * (p - (hi - 1)))
    # the bias of a visible key is at most 0.7 * 300 = 210 and rounded once more than a score is
    big += 210.0
    R.check_attend((out, None), (torch.stack(refs), None, torch.stack(slacks), big), torch.bfloat16, dim, True)
    ref = torch.stack(lses)
    assert ((lse.double() - ref).abs() <= 4 * 2.0 ** -24 * ref.abs() + 2.0 ** -10).all()


@pytest.mark.parametrize("opts", [{}, dict(softcap=20.0), dict(slopes=True)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,heads,group,members,shared,n_q", [(128, 8, 4, 30, 2100, 1), (128, 8, 4, 26, 2100, 3), (64, 2, 8, 100, 4100, 1),
                                                                (64, 2, 8, 100, 4200, 2), (128, 1, 16, 64, 6300, 1)])
def test_forked_contexts_lose_no_digits_to_the_shared_reading(dim, heads, group, members, shared, n_q, dtype, opts):
    """Rows of contexts forked from one come out as exact as a single context's: weights in two 16-bit parts."""
    pool = R.make_pool(1, heads, dim, 16, shared // 16 + members * 8 + 4, max_ctx=members + 2, dtype=dtype)
    parent = R.add_ctx(pool, shared, 1)
    st, kids = pool.fork(parent.handle, members)
    assert st == 0
    own = [1 + n_q + 7 * i % 50 for i in range(members)]
    tails = [R.rand((1, 2, t, heads, dim), 100 + i, dtype) for i, t in enumerate(own)]
    assert pool.append(kids, own, tails)[0] == 0
    ctxs = [R.Ctx(h, torch.cat((parent.rows, t), 2)) for h, t in zip(kids, tails)]
    q = R.rand((members * n_q, heads * group, dim), 2, dtype, 2.0)
    if opts.get("slopes"):
        opts = dict(slopes=torch.linspace(0.001, 0.02, heads * group, device="cuda"))
    st, got = pool.attend(0, kids, [n_q] * members, q, **opts)
    assert st == 0
    torch.cuda.synchronize()
    assert pool.sync_status() == 0
    st, again = pool.attend(0, kids, [n_q] * members, q, **opts)
    assert st == 0 and all(torch.equal(x, y) for x, y in zip(got, again))
    out, lse, slack, big = R.attend_ref(ctxs, [n_q] * members, q, **opts)
    if "slopes" in opts:
        big += 0.02 * (shared + 64)  # the bias is a part of the score, rounded as it is
    R.check_attend(got, (out, lse, slack, big), dtype, dim, False)


@pytest.mark.parametrize("opts", [{}, dict(softcap=20.0), dict(slopes=True)])
@pytest.mark.parametrize("dim,heads,group", [(128, 8, 4), (64, 8, 2)])
def test_generations_of_forks_in_one_large_batch(dim, heads, group, opts):
    """As many listed contexts as make reading their shared blocks together worth it, of two generations, some several times."""
    if opts.get("slopes"):
        opts = dict(slopes=torch.linspace(0.001, 0.02, heads * group, device="cuda"))
    pool = R.make_pool(1, heads, dim, 16, 1200, max_ctx=64)
    root = R.add_ctx(pool, 2100, 1)
    alone = R.add_ctx(pool, 777, 2)
    st, kids = pool.fork(root.handle, 9)
    assert st == 0
    own = [1, 2, 5, 16, 17, 300, 33, 64, 4]
    tails = [R.rand((1, 2, t, heads, dim), 60 + i) for i, t in enumerate(own)]
    assert pool.append(kids, own, tails)[0] == 0
    ctxs = [R.Ctx(h, torch.cat((root.rows, t), 2)) for h, t in zip(kids, tails)]
    st, more = pool.fork(ctxs[5].handle, 7)
    assert st == 0
    ctxs += [R.Ctx(h, ctxs[5].rows) for h in more] + [alone, root]
    batch = [ctxs[i] for i in [3, 17, 0, 9, 10, 16, 11, 1, 2, 4, 12, 5, 13, 6, 7, 14, 8, 15, 3] * 6]
    for n_q in ([1] * len(batch), [1 + i % 2 for i in range(len(batch))], [1] * 50 + [40] + [1] * (len(batch) - 51)):
        q = R.rand((sum(n_q), heads * group, dim), sum(n_q), scale=2.0)
        st, got = pool.attend(0, [c.handle for c in batch], n_q, q, **opts)
        assert st == 0
        st, again = pool.attend(0, [c.handle for c in batch], n_q, q, **opts)
        assert st == 0 and all(torch.equal(x, y) for x, y in zip(got, again))
        torch.cuda.synchronize()
        assert pool.sync_status() == 0
        out, lse, slack, big = R.attend_ref(batch, n_q, q, **opts)
        if "slopes" in opts:
            big += 0.02 * 2500
        R.check_attend(got, (out, lse, slack, big), torch.bfloat16, dim, max(n_q) > 2)


@pytest.mark.parametrize("times", [1, 7])
def test_nonfinite_values_of_blocks_that_a_large_batch_of_forks_shares(times):
    pool = R.make_pool(1, 8, 128, 16, 400)
    rows = R.rand((1, 2, 1600, 8, 128), 5)
    rows[0, 1, 1599, 0, 3] = math.inf
    rows[0, 1, 1598, 2, 5] = -math.inf
    rows[0, 1, 700, 1, 4] = math.nan
    root = R.add_ctx(pool, 1600, 0, rows)
    st, kids = pool.fork(root.handle, 6)
    assert st == 0 and pool.reserve(kids[:3], [1, 1, 1])[0] == 0
    kv = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda")
    assert pool.store(0, kids[:3], [1, 1, 1], kv, kv)[0] == 0
    q = R.rand((6 * times, 32, 128), 6, scale=2.0)
    st, (out, lse) = pool.attend(0, kids * times, None, q)
    assert st == 0
    torch.cuda.synchronize()
    assert pool.sync_status() == 0 and torch.isfinite(lse).all()
    assert (out[:, :4, 3] == math.inf).all() and (out[:, 8:12, 5] == -math.inf).all() and torch.isnan(out[:, 4:8, 4]).all()
    rest = out.clone()
    rest[:, :4, 3], rest[:, 8:12, 5], rest[:, 4:8, 4] = 0, 0, 0
    assert torch.isfinite(rest).all()
    st, (out, lse) = pool.attend(0, kids[3:] * times, [2] * (3 * times), q)  # the first of two queries before the last shared token
    assert st == 0 and torch.isfinite(out[0::2, :4, 3]).all() and (out[1::2, :4, 3] == math.inf).all()
