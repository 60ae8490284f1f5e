"""Chunk operators given what does not fit or does not belong: the damage stays where the documentation says."""
import math

import numpy as np
import pytest
import torch

from chunk_testlib import BS, DEV, Batch, attn_ref, blocks_of, check_attn, context, gpu, tables_ref, visible
from test_gpu_chunk_prep import Tables

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- tables that do not fit
def _overflowed(ctx, new, held, n_held, free, begin, max_entries):
    """The definition: tables cut at max_entries, nothing taken behind the cut, slots of blocks that are the request's."""
    need = [blocks_of(c + n) for c, n in zip(ctx, new)]
    at, kvp, kvi, slots, held, n_new = 0, [0], [], [], [list(map(int, h)) for h in held], [int(x) for x in n_held]
    for r, (c, n) in enumerate(zip(ctx, new)):
        for k in range(need[r]):
            if at + k < max_entries:
                if k >= n_new[r]:
                    held[r][k] = int(free[begin])
                    n_new[r], begin = k + 1, begin + 1
                kvi.append(held[r][k])
        at += need[r]
        kvp.append(min(at, max_entries))
        slots += [held[r][t // BS] * BS + t % BS if t // BS < n_new[r] else -1 for t in range(c, c + n)]
    return held, n_new, kvp, kvi, slots, begin


@pytest.mark.parametrize("short", [1, 2, 3, 7, 8, 9, 30])
@pytest.mark.parametrize("extra", [0, 2])
def test_lists_agree_when_tables_do_not_fit(short, extra):
    """What is counted as held is recorded, what is not recorded is not taken and given no slot, and the offsets stay inside."""
    t = Tables([20, 30, 0, 90, 5], [5, 60, 16, 50, 3], seed=6 + extra, extra=extra, begin=2, spare_entries=0)
    m = max(0, t.entries - short)
    t.call(kv_indices=t.t["kv_indices"][:m])
    assert t.c.nsd_get_status()[0] == 6
    held, n_new, kvp, kvi, slots, end = _overflowed(t.ctx.tolist(), t.new.tolist(), t.held, t.n_held, t.free, t.begin, m)
    assert t.t["kv_indptr"].tolist() == kvp
    assert t.t["kv_indices"].tolist() == kvi + [-9] * (t.entries - m)
    assert t.t["n_held_new"].tolist() == n_new and t.t["free_end"].item() == end
    assert t.t["held"].tolist() == held
    assert t.t["slot_map"][:t.rows].tolist() == slots
    # the next step, with room again, takes up where this one stopped
    after = dict(held=t.t["held"], n_held=t.t["n_held_new"].clone(), free_begin=t.t["free_end"].clone())
    t.call(**after)
    assert t.c.nsd_get_status() == (0, -1)
    want = tables_ref(t.ctx, t.new, held, n_new, t.free, end)
    assert t.t["held"].tolist() == want[0] and t.t["kv_indices"].tolist() == want[3]
    assert t.t["slot_map"][:t.rows].tolist() == want[5] and t.t["free_end"].item() == want[8]


def test_a_bad_id_of_the_free_list_is_recorded_where_it_counts():
    t = Tables([0, 30], [20, 40], seed=8)                      # two blocks, then three beside the two held
    bad = t.num_blocks + 7
    t.t["free_blocks"][1] = bad
    t.call()
    assert t.c.nsd_get_status() == (6, 0)
    assert t.t["held"][0].tolist()[:2] == [int(t.free[0]), bad] and t.t["n_held_new"][0].item() == 2
    t.call(held=t.t["held"], n_held=t.t["n_held_new"].clone(), free_begin=t.t["free_end"].clone())
    assert t.c.nsd_get_status() == (6, 0)                      # known to the next step too
    assert t.t["slot_map"][16:20].tolist() == [-1] * 4


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


# --------------------------------------------------------------------------- slots that no row sees
def _padded_documents(ctx, new, pads, seed):
    """Documents of random lengths with runs of padding rows (which see nothing) between them."""
    rng = np.random.default_rng(seed)
    out = []
    for c, n in zip(ctx, new):
        rows, start = [], 0
        while len(rows) < n:
            rows += [start] * int(rng.integers(1, 60))
            rows += [10 ** 6] * int(rng.integers(1, pads + 1))
            start = c + len(rows)
        out += rows[:n]
    return out


def _poison(b, **masks):
    """NaN in every slot that no row of its request sees."""
    seen, row = visible(b.ctx, b.new, **masks), 0
    hidden = 0
    for r, (c, n) in enumerate(zip(b.ctx, b.new)):
        used = np.zeros(c + n, dtype=bool)
        for first, stop in seen[row:row + n]:
            used[first:stop] = True
        row += n
        for t in np.flatnonzero(~used):
            b.pool[0, int(b.kv_indices[int(b.kv_indptr[r]) + t // BS]), :, :, t % BS] = math.nan
        hidden += int((~used).sum())
    return hidden


@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64), (4, 4, 128), (28, 4, 128)])
@pytest.mark.parametrize("pads", [1, 5, 40, 300])
def test_slots_between_documents_may_hold_anything(shape, pads):
    """Padding rows inside a request leave keys that no row sees between keys that some do."""
    ctx, new = [0, 300, 5, 70], [400, 150, 1, 700]
    docs = _padded_documents(ctx, new, pads, pads)
    b = Batch(ctx, new, heads=shape[0], kv_heads=shape[1], dim=shape[2], seed=41)
    assert _poison(b, row_first=docs) > 0
    b.run(row_first=docs)


@pytest.mark.parametrize("window,prefix", [(0, [90, 310, 0, 100]), (20, None), (33, [90, 310, 0, 100])])
def test_slots_between_documents_with_windows_and_prefixes(window, prefix):
    ctx, new = [0, 300, 5, 70], [400, 150, 1, 700]
    masks = dict(row_first=_padded_documents(ctx, new, 30, 42), window=window, prefix_len=prefix)
    b = Batch(ctx, new, heads=8, kv_heads=2, dim=128, seed=42)
    assert _poison(b, **masks) > 0
    b.run(softcap=20.0, **masks)


# --------------------------------------------------------------------------- NaN among what a row sees
@pytest.mark.parametrize("mode", [{}, dict(softcap=20.0), dict(slopes=[2.0 ** -(h + 1) for h in range(8)]),
                                  dict(softcap=20.0, slopes=[2.0 ** -(h + 1) for h in range(8)])])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_nan_is_not_taken_for_an_empty_row(mode, dim):
    """In a single tile, in alternate tiles of two streams, in units of two row tiles and in units cut into pieces.  Rows are
    computed apart from one another, so those that see no NaN keep their bits."""
    ctx, new = [3000, 5, 0, 20000, 900], [1, 200, 40, 1, 2]
    b = Batch(ctx, new, heads=8, kv_heads=2, dim=dim, seed=43)
    c = b.context()
    plan = b.plan(c)
    b.attn(c, plan, **mode)
    o, lse = b.o[0].clone(), b.lse[0].clone()
    # a query of NaN
    q = b.q[0].clone()
    want = torch.zeros((b.rows, 8), dtype=torch.bool, device=DEV)
    for row, h in ((0, 3), (1, 0), (150, 7), (200, 5), (201, 1), (240, 2), (241, 6), (243, 4)):
        b.q[0, row, h * dim + 5] = math.nan
        want[row, h] = True
    b.attn(c, plan, **mode)
    _nan_where(b, want, o, lse)
    b.q[0].copy_(q)
    # a key of NaN, of one kv head
    want.zero_()
    for r, t in ((0, 2999), (0, 17), (1, 100), (2, 39), (3, 11111), (4, 0)):
        b.pool[0, int(b.kv_indices[int(b.kv_indptr[r]) + t // BS]), 0, 1, t % BS, 3] = math.nan
        for i in range(new[r]):
            want[int(b.q_indptr[r]) + i, 4:] |= t <= ctx[r] + i
    b.attn(c, plan, **mode)
    _nan_where(b, want, o, lse)
    assert c.nsd_get_status() == (0, -1)


def _nan_where(b, want, o, lse):
    assert torch.equal(torch.isnan(b.lse[0, :b.rows]), want)
    assert torch.isnan(b.o[0, :b.rows][want]).all()
    assert torch.equal(b.o[0, :b.rows][~want], o[:b.rows][~want]) and torch.equal(b.lse[0, :b.rows][~want], lse[:b.rows][~want])


# --------------------------------------------------------------------------- plans of another layout
@pytest.mark.parametrize("more", [-1, 1, 300])
def test_a_plan_of_a_context_with_another_max_batch_is_reported(more):
    """The parts of the buffer lie elsewhere then; nothing of it may be used."""
    b = Batch([100, 30], [30, 1], seed=44)
    c, other = (context(b.heads, b.kv_heads, b.dim, b.num_blocks, max_batch=n) for n in (3, 3 + more))
    plan = torch.zeros(max(c.nsd_chunk_plan_bytes(31), other.nsd_chunk_plan_bytes(31)), dtype=torch.uint8, device=DEV)
    other.nsd_chunk_plan(plan, 31, b.qp, b.ctx_len, b.kvp)
    b.attn(c, plan)
    assert c.nsd_get_status()[0] == 6 and (b.o == 7.0).all() and (b.lse == 7.0).all()
    b.masks = {}
    c.nsd_chunk_plan(plan, 31, b.qp, b.ctx_len, b.kvp)
    b.attn(c, plan)
    assert c.nsd_get_status() == (0, -1)
    b.check()


# --------------------------------------------------------------------------- large caps
@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64)])
@pytest.mark.parametrize("softcap", [1e3, 1.4e3, 1.5e3, 1e4, 1e5, 1e6, 1e9])
def test_rows_of_small_scores_beside_rows_of_scores_like_the_cap(shape, softcap):
    """Rows are capped 32 at a time; a row whose scores reach a large cap must not cost the others their accuracy."""
    b = Batch([200, 0, 1000], [70, 300, 1], heads=shape[0], kv_heads=shape[1], dim=shape[2], seed=45)
    for row in (3, 40, 69, 75, 130, 200, 340):
        b.q[0, row, :shape[2] * 2] *= softcap
    b.run(softcap=softcap)


# --------------------------------------------------------------------------- huge scores
def _check_one_hot(b, scale, rows=None, heads=None, window=0):
    """Where the largest score stands clear of the second, the output is its V and the log-sum is the score.  A score is a sum
    of dim products that are exact in 32 bits; an addition on the tensor cores may cut off 2^-23 of a partial sum, and none is
    larger than the sum of the products' sizes: off by dim 2^-23 of that sum at most.  Scale, product, and the way from the log2
    domain back round four times, 2^-24 each.  Clear means: by more than both scores' errors and 20 nats (all other weights
    together below 1e4 e^-20).  The weight may be rounded to bf16 where the maximum lags, and the output is: 2 x 2^-8."""
    seen = visible(b.ctx, b.new, window=window)
    clear = total = 0
    for r, (c, n) in enumerate(zip(b.ctx, b.new)):
        row0 = int(b.q_indptr[r])
        table = torch.as_tensor(b.kv_indices[int(b.kv_indptr[r]):int(b.kv_indptr[r]) + blocks_of(c + n)].astype(np.int64), device=DEV)
        kv = torch.nan_to_num(b.pool[0][table].double(), nan=0.0).permute(1, 2, 0, 3, 4).reshape(2, b.kv_heads, -1, b.dim)[:, :, :c + n]
        span = torch.tensor(seen[row0:row0 + n], device=DEV)
        key = torch.arange(c + n, device=DEV)
        see = (key[None] >= span[:, :1]) & (key[None] < span[:, 1:])
        for h in range(b.heads):
            g = h // (b.heads // b.kv_heads)
            q = b.q[0, row0:row0 + n].double().reshape(n, b.heads, b.dim)[:, h]
            s = (q @ kv[0, g].T * scale).masked_fill(~see, -math.inf)
            size = (q.abs() @ kv[0, g].T.abs() * scale).masked_fill(~see, 0).max(1).values
            top = torch.cat([s, torch.full((n, 1), -math.inf, device=DEV, dtype=s.dtype)], 1).topk(2, 1)
            err = size * (b.dim * 2.0 ** -23 + 4 * 2.0 ** -24)
            sure = top.values[:, 0] - top.values[:, 1] > 2 * err + 20
            if rows is not None:
                sure &= torch.isin(torch.arange(row0, row0 + n, device=DEV), torch.tensor(rows, device=DEV)) & (heads is None or h in heads)
            o, lse = b.o[0, row0:row0 + n, h].double(), b.lse[0, row0:row0 + n, h].double()
            assert torch.isfinite(o).all() and torch.isfinite(lse).all()
            v = kv[1, g][top.indices[:, 0].clamp(max=c + n - 1)]
            assert ((o - v).abs() <= 2.0 ** -7 * v.abs() + 1e-4)[sure].all()
            assert ((lse - top.values[:, 0]).abs() <= err + 2.0 ** -10)[sure].all()
            clear, total = clear + int(sure.sum()), total + n
    return clear / total


@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64)])
@pytest.mark.parametrize("scale", [1e6, 1e8, 1e9, 1e10, 1e20, 1e30])
def test_huge_scores_by_scales_up_to_the_documented_one(shape, scale):
    """Scores far beyond what 32 bits hold to a whole number: the largest key has all the weight."""
    b = Batch([200, 0, 3000, 9000], [70, 300, 1, 2], heads=shape[0], kv_heads=shape[1], dim=shape[2], seed=46)
    c = b.context()
    for window in (0, 300):
        plan = b.plan(c, window=window)
        b.attn(c, plan, scale=scale)
        assert c.nsd_get_status() == (0, -1)
        assert _check_one_hot(b, scale, window=window) > 0.9


def test_a_row_of_huge_scores_leaves_its_neighbours_their_bits():
    b = Batch([200, 0, 3000], [70, 300, 1], seed=47)
    c = b.context()
    plan = b.plan(c)
    b.attn(c, plan)
    o = b.o[0].clone()
    rows = [3, 40, 69, 75, 200]
    b.q[0, rows, :128] *= 1e12
    b.attn(c, plan)
    assert c.nsd_get_status() == (0, -1)
    assert _check_one_hot(b, 128 ** -0.5, rows, [0]) > 0
    same = torch.ones((b.rows, 8), dtype=torch.bool, device=DEV)
    same[rows, 0] = False
    assert torch.equal(b.o[0, :b.rows][same], o[:b.rows][same])
