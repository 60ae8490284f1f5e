"""Chunk operators given what does not fit or does not belong: the damage stays where the documentation says."""
import math

import numpy as np
import pytest
import torch

from chunk_testlib import DEV, Batch, attn_ref, check_attn, gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("short", [1, 9, 24])
def test_attention_after_tables_that_do_not_fit_stays_inside_them(short):
    """The tables live in a larger allocation.  What lies behind them must not matter: the keys of entries that did not fit
    read as zeros."""
    b = Batch([100, 37, 300], [30, 70, 140], seed=40)
    c = b.context()
    n = int(b.kv_indptr[-1])
    m, stride = n - short, max(int(x) for x in np.diff(b.kv_indptr))
    held = torch.full((3, stride), -5, dtype=torch.int32)
    for r in range(3):
        lo, hi = int(b.kv_indptr[r]), int(b.kv_indptr[r + 1])
        held[r, :hi - lo] = torch.from_numpy(b.kv_indices[lo:hi])
    n_held = np.diff(b.kv_indptr).astype(np.int32)
    room = torch.full((n + 64,), -1, dtype=torch.int32, device=DEV)
    out = []
    for tail in (-1, int(b.kv_indices[0]), int(b.kv_indices[-1])):
        room.fill_(tail)
        kvp, qp = torch.empty_like(b.kvp), torch.empty_like(b.qp)
        spare = torch.zeros(1, dtype=torch.int64, device=DEV)
        c.nsd_block_tables(b.ctx_len, gpu(np.asarray(b.new, dtype=np.int32)), held.to(DEV), gpu(n_held), gpu(np.zeros(1, dtype=np.int32)), None,
                           kvp, room[:m], qp, None, None, None, torch.zeros(3, dtype=torch.int32, device=DEV), spare)
        assert c.nsd_get_status()[0] == 6
        assert int(kvp[-1]) == m and (room[m:] == tail).all()
        plan = torch.empty(c.nsd_chunk_plan_bytes(b.max_rows), dtype=torch.uint8, device=DEV)
        c.nsd_chunk_plan(plan, b.max_rows, qp, b.ctx_len, kvp)
        c.nsd_chunk_attn(plan, b.max_rows, b.pool, b.q[0], b.o[0], b.lse[0], room[:m])
        assert c.nsd_get_status()[0] == 6
        out.append((b.o.clone(), b.lse.clone()))
    for o, lse in out[1:]:
        assert torch.equal(o, out[0][0]) and torch.equal(lse, out[0][1])
    pool = torch.cat([torch.nan_to_num(b.pool[0].double(), nan=0.0), torch.zeros_like(b.pool[0, :1]).double()])
    table = b.kv_indices.copy()
    table[m:] = b.num_blocks                                   # a block of zeros
    q = b.q[0, :b.rows].double().reshape(b.rows, b.heads, b.dim)
    check_attn(b.o[0, :b.rows], b.lse[0, :b.rows], attn_ref(q, pool, b.ctx, b.new, b.kv_indptr, table))
    assert math.isfinite(float(b.lse[0, :b.rows].sum()))
