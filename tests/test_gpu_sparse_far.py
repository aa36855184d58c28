"""Sparse attention where offsets pass 32 bits: a pool and a summary of 4.5 GB each."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2607_10987_b200 import binding as B
from tests import serve_reference as R
from tests import sparse_reference as S
from tests.test_gpu_sparse import settle

pytestmark = pytest.mark.gpu


def test_blocks_far_into_a_long_pool():
    layers, heads, dim, block, blocks, dtype = 2, 1, 8, 1, 70_000_000, torch.bfloat16
    used = np.array([blocks - 1, 0, blocks - 2, 1 << 26, (1 << 26) - 1, 1, *range(blocks - 60, blocks - 20)], dtype=np.int32)
    free = np.ones(blocks, dtype=bool)
    free[used] = False
    mem = torch.empty(layers, blocks, 2, block, heads, dim, dtype=dtype, device="cuda")
    pool = B.KVPool(layers, heads, dim, block, 2, blocks, 2, 64, free_order=np.concatenate((used, np.flatnonzero(free).astype(np.int32))),
                    pool_tensor=mem, max_batch=8)
    tokens = len(used)
    rows = R.rand((layers, 2, tokens, heads, dim), 1)
    st, c = pool.imp(rows, tokens)
    assert st == 0
    summary, q = pool.new_summary(), R.rand((3, 4, dim), 2)
    assert summary[1:].numel() > 1 << 31 and mem[1:].numel() * 2 > 1 << 31
    for layer in range(layers):
        assert pool.summarize(layer, [c], None, summary, dtype)[0] == 0
        st, chosen = pool.select(layer, [c], [3], q, summary, 12, sink=1, recent=2)
        assert st == 0
        st, got = pool.attend_blocks(layer, [c], [3], q, chosen)
        assert st == 0
        st, tables = pool.batch_tables([c], [3])
        assert st == 0
        settle(pool)
        assert tables["tables"][0].tolist() == used.tolist() and tables["slots"].tolist() == used[-3:].tolist()
        codes, exps = S.read_summary(summary, layer, torch.from_numpy(used), heads, dim)
        want, want_e = S.summary_ref(rows[layer, 0], block)
        assert torch.equal(codes, want) and torch.equal(exps, want_e)
        for j in range(3):
            s = S.scores_ref(codes[:, 0], exps[:, 0], q[j])
            assert chosen[j, 0].tolist() == S.select_ref(s, tokens - 3 + j, 12, 1, 2)
        R.check_attend(got, S.attend_blocks_ref([R.Ctx(c, rows)], [3], q, chosen, block, layer=layer), dtype, dim, False)
