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
