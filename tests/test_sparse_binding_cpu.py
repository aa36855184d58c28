"""The Python calls of sparse attention and of a batch's tables, without a device: what they refuse before anything is allocated or
launched, on the model of the CUDA runtime (sparse_model.cpp) and tensors of the host."""
from __future__ import annotations

import pytest
import torch

from paper_2607_10987_b200 import binding as B
from tests import test_order_cpu as O
from tests.test_sparse_cpu import lib, pool  # noqa: F401 (fixtures)

HEADS = 4


class HostPool(B.KVPool):
    """KVPool's methods over a pool of the model, with host tensors in the place of device tensors."""

    def __init__(self, pool, stream):  # noqa: F811
        self.torch, self.device = torch, torch.device("cpu")
        self._raw_stream = lambda index: stream
        self._codes = {torch.bfloat16: B.AAF_DTYPE_BF16, torch.float16: B.AAF_DTYPE_F16}
        self.L, self.H, self.D, self.BS, self.E, self.NB = O.L, O.H, O.D, O.BS, 2, O.NB
        self.max_ctx, self.max_blk = O.CTX, O.BLK
        self.h, self._like = pool.h, None
        self._attend_ws = torch.empty(B.aaf_kv_attend_workspace_bytes(pool.h), dtype=torch.uint8)

    def close(self):  # the model's pool is closed by its fixture
        pass


@pytest.fixture
def kv(lib, pool, monkeypatch):  # noqa: F811
    monkeypatch.setattr(B, "_lib", lib)
    st = lib.order_stream()
    ctxs = [pool.imp(st, 160)[1] for _ in range(4)]
    return HostPool(pool, st), ctxs


def rows(n):
    return torch.zeros(n, HEADS, O.D, dtype=torch.bfloat16)


CALLS = {
    "summarize": lambda kv, c, n: kv.summarize(0, c, n, kv.new_summary(), torch.bfloat16)[0],
    "select": lambda kv, c, n: kv.select(0, c, n, rows(sum(n)), kv.new_summary(), 4)[0],
    "attend_blocks": lambda kv, c, n: kv.attend_blocks(0, c, n, rows(sum(n)), torch.zeros(sum(n), O.H, 4, dtype=torch.int32))[0],
    "batch_tables": lambda kv, c, n: kv.batch_tables(c, n)[0],
}


@pytest.mark.parametrize("call", CALLS)
def test_as_many_counts_as_contexts(lib, kv, call):  # noqa: F811
    kv, ctxs = kv
    at = lib.order_ops()
    for counts in ([1, 1, 1], [1, 1, 1, 1, 1], [5], []):
        with pytest.raises(ValueError):
            CALLS[call](kv, ctxs, counts)
    assert lib.order_ops() == at
    assert CALLS[call](kv, ctxs, [1, 2, 3, 4]) == 0 and lib.order_ops() == at + 1


def test_numbers_that_do_not_fit_the_library_are_refused(lib, kv):  # noqa: F811
    """They would arrive without their upper bits: a sink of 2^32 as none."""
    kv, ctxs = kv
    c, big, at = ctxs[:1], 1 << 32, lib.order_ops()
    summary, q, blocks = kv.new_summary(), rows(1), torch.zeros(1, O.H, 4, dtype=torch.int32)
    for kw in (dict(sink=big), dict(sink=1 - big), dict(recent=big + 1), dict(keep=big + 4)):
        assert kv.select(0, c, None, q, summary, **{"keep": 4, **kw})[0] == B.AAF_ERR_INVALID_ARG, kw
    for layer in (big, -big):
        assert kv.summarize(layer, c, None, summary, torch.bfloat16)[0] == B.AAF_ERR_INVALID_ARG
        assert kv.select(layer, c, None, q, summary, 4)[0] == B.AAF_ERR_INVALID_ARG
        assert kv.attend_blocks(layer, c, None, q, blocks)[0] == B.AAF_ERR_INVALID_ARG
    assert kv.attend_blocks(0, c, None, q, blocks, window=big + 16)[0] == B.AAF_ERR_INVALID_ARG
    for kw in (dict(rows=big + 1), dict(tokens=big + 1), dict(cols=big + 10)):
        assert kv.batch_tables(c, **kw)[0] == B.AAF_ERR_TOO_MANY, kw
    assert lib.order_ops() == at
