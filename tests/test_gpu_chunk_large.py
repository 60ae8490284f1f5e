"""Chunk operators at the far end of their sizes: offsets that 32 bits do not hold, the largest batch of block tables."""
import numpy as np
import pytest
import torch

from chunk_testlib import BS, DEV, HALF_BF16, attn_ref, check_attn, context, gpu, offsets, rope_ref
from test_gpu_chunk_prep import Tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,dim", [(16, 8, 128), (32, 16, 64)])
def test_a_pool_beyond_32_bits(heads, kv_heads, dim):
    """A slab of 2.4e9 elements, the second layer of two: appended to and read back in its last blocks."""
    num_blocks, ctx, new = 2_400_000_000 // (2 * kv_heads * BS * dim), [0, 300], [200, 5]
    pool = torch.empty((2, num_blocks, 2, kv_heads, BS, dim), dtype=torch.bfloat16, device=DEV)
    c = context(heads, kv_heads, dim, num_blocks, num_layers=2)
    g = torch.Generator().manual_seed(50)
    table = (num_blocks - 1 - torch.randperm(40, generator=g)[:33]).to(torch.int32)     # 13 and 20 blocks
    kvp, qp = offsets([13, 20]), offsets(new)
    # what request 1 holds already
    kv = torch.randn((20, 2, kv_heads, BS, dim), generator=g).to(torch.bfloat16).to(DEV)
    pool[1][table[13:].long().to(DEV)] = kv
    rows = sum(new)
    pos = torch.tensor([list(range(200)) + list(range(300, 305))], dtype=torch.int32)
    flat = torch.tensor([int(table[t // BS]) * BS + t % BS for t in range(200)] + [int(table[13 + t // BS]) * BS + t % BS for t in range(300, 305)])
    x = torch.randn((rows, heads + 2 * kv_heads, dim), generator=g).to(torch.bfloat16).to(DEV)
    q, k, v = x[:, :heads].reshape(rows, -1), x[:, heads:heads + kv_heads].reshape(rows, -1), x[:, heads + kv_heads:].reshape(rows, -1)
    freq = (1e4 ** (-np.arange(dim // 2) / (dim // 2))).astype(np.float32)
    q_out = torch.empty((rows, heads, dim), dtype=torch.bfloat16, device=DEV)
    c.nsd_rope_append(pool, 1, q, k, v, q_out, pos.to(DEV), [dim // 2], gpu(freq), flat.to(DEV))
    y, slack = rope_ref(x.double().cpu().numpy()[:, :heads + kv_heads], pos.numpy(), [dim // 2], freq, False, False)
    stored = pool[1][(flat // BS).to(DEV), :, :, (flat % BS).to(DEV)]                   # [rows][2][kv heads][dim]
    got = torch.cat([q_out, stored[:, 0]], 1).double().cpu().numpy()
    assert (np.abs(got - y) <= HALF_BF16 * np.abs(y) + 1.01 * slack).all()
    assert torch.equal(stored[:, 1], x[:, heads + kv_heads:])
    plan = torch.empty(c.nsd_chunk_plan_bytes(rows), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, rows, gpu(qp), gpu(np.asarray(ctx, dtype=np.int32)), gpu(kvp))
    o, lse = torch.empty_like(q_out), torch.empty((rows, heads), device=DEV)
    c.nsd_chunk_attn(plan, rows, pool, q_out, o, lse, table.to(DEV), layer=1)
    assert c.nsd_get_status() == (0, -1)
    used = pool[1][table.long().to(DEV)].double()
    check_attn(o, lse, attn_ref(q_out.double(), torch.nan_to_num(used), ctx, new, kvp, np.arange(33)))


def test_rows_beyond_32_bits():
    """300 000 single tokens of 64 heads of 128: 2.4e9 elements of q and of o."""
    n, heads, kv_heads, dim = 300_000, 64, 8, 128
    g = torch.Generator(device=DEV).manual_seed(51)
    pool = torch.randn((50, 2, kv_heads, BS, dim), generator=g, device=DEV).to(torch.bfloat16)
    q = torch.empty((n, heads * dim), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    c = context(heads, kv_heads, dim, 50, max_batch=n)
    ramp = torch.arange(n + 1, dtype=torch.int64, device=DEV)
    kvi = (torch.arange(n, device=DEV) * 7 % 50).to(torch.int32)
    o, lse = torch.empty((n, heads, dim), dtype=torch.bfloat16, device=DEV), torch.empty((n, heads), device=DEV)
    plan = torch.empty(c.nsd_chunk_plan_bytes(n), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, n, ramp, torch.full((n,), 11, dtype=torch.int32, device=DEV), ramp)
    c.nsd_chunk_attn(plan, n, pool, q, o, lse, kvi)
    assert c.nsd_get_status() == (0, -1)
    for rows in (torch.arange(100), torch.arange(262_100, 262_200), torch.arange(n - 100, n)):
        rows = rows.to(DEV)
        kv = pool[kvi[rows].long()].double()[:, :, :, :12].repeat_interleave(heads // kv_heads, 2)
        s = torch.einsum("nhd,nhkd->nhk", q[rows].double().view(-1, heads, dim), kv[:, 0]) / dim ** 0.5
        w = torch.softmax(s, -1)
        check_attn(o[rows], lse[rows], (torch.einsum("nhk,nhkd->nhd", w, kv[:, 1]), torch.logsumexp(s, -1), torch.einsum("nhk,nhkd->nhd", w, kv[:, 1].abs())))


def test_tables_of_the_largest_batch():
    import paper_2609_29364_b200 as nsd

    rng = np.random.default_rng(52)
    t = Tables(rng.integers(0, 60, 8192), rng.integers(0, 4, 8192), seed=52, extra=1, begin=5)
    t.call()
    assert t.c.nsd_get_status() == (0, -1)
    t.check()
    t = Tables(np.zeros(8193, dtype=int), np.zeros(8193, dtype=int), seed=53)
    with pytest.raises(nsd.NsdError) as e:
        t.call()
    assert e.value.code == 3
