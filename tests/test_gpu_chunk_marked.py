"""Chunk attention over contexts in which one key decides each row (chunk_marked.py): keys at the edges of tiles, blocks,
windows, documents and prefixes, at every place where the work may be cut, the last visible one and the first that is not."""
import numpy as np
import pytest
import torch

from chunk_marked import Marked, edges
from chunk_testlib import DEV, Batch, check_attn, context, gpu

pytestmark = pytest.mark.gpu

SHAPES = [(16, 2, 128), (12, 4, 64), (4, 4, 128), (32, 1, 64)]


def run(m, wanted, slopes=None, softcap=0.0, **masks):
    c = context(m.heads, m.kv_heads, m.dim, m.num_blocks, max_batch=len(m.ctx))
    kvp, qp, kvi = gpu(m.kv_indptr), gpu(m.q_indptr), gpu(m.kv_indices)
    as_i32 = lambda x: None if x is None else gpu(np.asarray(x, dtype=np.int32))  # noqa: E731
    plan = torch.empty(c.nsd_chunk_plan_bytes(m.rows), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, m.rows, qp, as_i32(m.ctx), kvp, window=masks.get("window", 0), prefix_len=as_i32(masks.get("prefix_len")),
                     row_first=as_i32(masks.get("row_first")))
    o, lse = torch.empty((m.rows, m.heads, m.dim), dtype=torch.bfloat16, device=DEV), torch.empty((m.rows, m.heads), device=DEV)
    for q in m.queries(wanted):
        o.fill_(7.0)
        c.nsd_chunk_attn(plan, m.rows, m.pool, q, o, lse, kvi, softcap=softcap, alibi_slopes=None if slopes is None else gpu(slopes, torch.float32))
        check_attn(o, lse, m.reference(q, softcap=softcap, slopes=slopes, **masks))
    assert c.nsd_get_status() == (0, -1)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("ctx", [3000, 5000, 20011])
def test_every_tile_edge_of_a_single_token(shape, ctx):
    """One request: each CTA has a tile or two, so nearly every tile edge is a cut."""
    marks = edges(ctx, 128) + [ctx - 1, ctx]
    run(Marked([ctx], [1], *shape, marks, seed=ctx, device=DEV), lambda p: marks)


@pytest.mark.parametrize("shape", SHAPES[:2])
def test_every_block_edge_of_a_few_tiles(shape):
    marks = edges(700, 16)
    run(Marked([700, 650, 690], [1, 3, 1], *shape, marks, seed=1, device=DEV), lambda p: marks)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("window", [1, 100, 1000, 1024])
def test_window_edges(shape, window):
    ctx, new = [3000, 1500, 0], [33, 1, 150]
    near = (-window - 1, -window, 1 - window, 2 - window, -1, 0, 1)
    marks = [p + d for c, n in zip(ctx, new) for p in range(c, c + n) for d in near]
    run(Marked(ctx, new, *shape, marks, seed=window, device=DEV), lambda p: [p + d for d in near], window=window)


@pytest.mark.parametrize("shape", SHAPES)
def test_the_diagonal_of_a_prompt(shape):
    marks = range(600)
    run(Marked([0, 90], [600, 300], *shape, marks, seed=2, device=DEV), lambda p: (p, p + 1, 0, p // 128 * 128, p // 128 * 128 - 1, p - 1, p // 16 * 16))


@pytest.mark.parametrize("shape", SHAPES[:2])
def test_edges_of_documents_and_prefixes(shape):
    ctx, new = [0, 200, 700], [500, 260, 90]
    starts = (0, 37, 128, 200, 333, 384, 401, 700, 731)
    first = [max(s for s in starts if s <= p) for c, n in zip(ctx, new) for p in range(c, c + n)]
    prefix = [60, 340, 0]
    wanted = lambda p: [x for s in starts if abs(p - s) < 200 for x in (s - 1, s)] + [p, p + 1, 59, 60, 339, 340]  # noqa: E731
    marks = sorted({x for c, n in zip(ctx, new) for p in range(c, c + n) for x in wanted(p)})
    m = Marked(ctx, new, *shape, marks, seed=3, device=DEV)
    run(m, wanted, row_first=first)
    run(m, wanted, row_first=first, prefix_len=prefix)


@pytest.mark.parametrize("shape", SHAPES)
def test_cap_and_bias_together_at_either_head_size(shape):
    slopes = [(-1.0) ** h * 0.002 / (h + 1) for h in range(shape[0])]
    marks = edges(1500, 128) + list(range(1400, 1580))
    run(Marked([1450, 1400], [1, 150], *shape, marks, seed=4, device=DEV), lambda p: edges(1500, 128) + [p, p + 1, p - 500, p - 499],
        slopes=slopes, softcap=60.0, window=500)


@pytest.mark.parametrize("shape", SHAPES[:2])
def test_buffers_far_larger_than_the_batch(shape):
    """What a captured step has: room for many more rows than the batch brings."""
    Batch([300, 0, 2000], [1, 70, 5], heads=shape[0], kv_heads=shape[1], dim=shape[2], pad_rows=20000, seed=5).run()
    Batch([0], [1], heads=shape[0], kv_heads=shape[1], dim=shape[2], pad_rows=5000, seed=6).run(window=5)
