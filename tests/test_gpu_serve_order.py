"""Calls of one pool on several streams, with a device that is held back where the order matters."""
from __future__ import annotations

import pytest
import torch

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
