"""Plain 64-bit forms of the chunk operators (block tables, rotary append, attention of a chunk over the pool), on the
host and from the definitions, with the tolerances the GPU tests hold the kernels to."""
from __future__ import annotations

import math

import numpy as np
import torch

BS = 16
DEV = "cuda:0"
HALF_BF16 = 2.0 ** -8          # largest relative error of one rounding to bf16


def context(heads=8, kv_heads=2, dim=128, num_blocks=64, max_batch=16, num_layers=1, num_slabs=None, **kw):
    import paper_2609_29364_b200 as nsd

    return nsd.VerifyContext(num_layers=num_layers, num_slabs=num_slabs, num_q_heads=heads, num_kv_heads=kv_heads, head_dim=dim,
                             block_size=BS, num_blocks=num_blocks, region_b_begin=0, max_batch=max_batch, max_gamma=1,
                             vocab_size=2, max_table_entries=num_blocks, **kw)


def offsets(sizes):
    return np.concatenate([[0], np.cumsum(np.asarray(sizes, dtype=np.int64))]).astype(np.int64)


def blocks_of(tokens):
    return (int(tokens) + BS - 1) // BS


def gpu(a, dtype=None):
    t = torch.as_tensor(np.asarray(a)) if not torch.is_tensor(a) else a
    return (t if dtype is None else t.to(dtype)).to(DEV)


# --------------------------------------------------------------------------- block tables
def tables_ref(ctx, new, held, n_held, free, begin):
    """Returns (held, n_held, kv_indptr, kv_indices, q_indptr, slots, positions, owners, next free entry)."""
    held = [list(map(int, row)) for row in held]
    n_held = [int(x) for x in n_held]
    indices, slots, positions, owners = [], [], [], []
    for r, (c, n) in enumerate(zip(map(int, ctx), map(int, new))):
        need = blocks_of(c + n)
        while n_held[r] < need:
            held[r][n_held[r]] = int(free[begin])
            n_held[r] += 1
            begin += 1
        indices += held[r][:need]
        for t in range(c, c + n):
            slots.append(held[r][t // BS] * BS + t % BS)
            positions.append(t)
            owners.append(r)
    need = [blocks_of(int(c) + int(n)) for c, n in zip(ctx, new)]
    return held, n_held, offsets(need), indices, offsets(new), slots, positions, owners, begin


# --------------------------------------------------------------------------- rotary positions
def axis_of_pair(sections, cycled):
    if not cycled:
        return [a for a, s in enumerate(sections) for _ in range(s)]
    n = len(sections)
    return [p % n if p // n < sections[p % n] else 0 for p in range(sum(sections))]


def rope_ref(x, positions, sections, inv_freq, adjacent, cycled):
    """x [rows][heads][dim] float64; returns the rotated values and, per value, the bound of the kernel's error before
    the last rounding: the sines are off by at most 2^-21 (64-bit angle, its 32-bit remainder, sincospi), products and
    sum round three times more."""
    pairs = sum(sections)
    axis = axis_of_pair(sections, cycled)
    angle = np.stack([positions[axis[p]].astype(np.float64) * float(inv_freq[p]) for p in range(pairs)], -1)[:, None, :]
    i = np.arange(pairs)
    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + pairs)
    y, slack = x.copy(), np.zeros_like(x)
    y[..., a] = x[..., a] * np.cos(angle) - x[..., b] * np.sin(angle)
    y[..., b] = x[..., b] * np.cos(angle) + x[..., a] * np.sin(angle)
    slack[..., a] = slack[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * 2.0 ** -20
    return y, slack


# --------------------------------------------------------------------------- attention
def visible(ctx, new, window=0, prefix_len=None, row_first=None):
    """[first, stop) of every row, request by request."""
    out, row = [], 0
    for r, (c, n) in enumerate(zip(map(int, ctx), map(int, new))):
        for i in range(n):
            t = c + i
            stop = t + 1 if prefix_len is None else max(t + 1, min(int(prefix_len[r]), c + n))
            first = max(0, t + 1 - window) if window else 0
            if row_first is not None:
                first = max(first, int(row_first[row]))
            out.append((first, stop))
            row += 1
    return out


def attn_ref(q, pool, ctx, new, kv_indptr, kv_indices, scale=None, softcap=0.0, slopes=None, **masks):
    """q [rows][Hq][D], pool [blocks][2][Hkv][16][D], both float64 tensors.  Returns o, lse and A = sum of weight x |v|,
    which bounds what the rounding of the weights can move."""
    rows, hq, d = q.shape
    hkv = pool.shape[2]
    g = hq // hkv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    seen = visible(ctx, new, **masks)
    o, mag, lse = torch.zeros_like(q), torch.zeros_like(q), torch.full((rows, hq), -math.inf, dtype=torch.float64, device=q.device)
    row = 0
    for r, (c, n) in enumerate(zip(map(int, ctx), map(int, new))):
        if not n:
            continue
        total = c + n
        table = torch.as_tensor(np.asarray(kv_indices[int(kv_indptr[r]):int(kv_indptr[r]) + blocks_of(total)]).astype(np.int64), device=q.device)
        span = torch.tensor(seen[row:row + n], device=q.device)
        key = torch.arange(total, device=q.device)
        see = (key[None] >= span[:, :1]) & (key[None] < span[:, 1:])
        used = see.any(0)
        kv = pool[table.clamp(0, pool.shape[0] - 1)].permute(1, 2, 0, 3, 4).reshape(2, hkv, -1, d)[:, :, :total]
        kv = torch.where(used[None, None, :, None], kv, torch.zeros_like(kv))            # nothing but visible keys takes part
        pos = c + torch.arange(n, device=q.device)
        for h in range(hq):
            s = q[row:row + n, h] @ kv[0, h // g].T * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            if slopes is not None:
                s = s + float(slopes[h]) * (key[None] - pos[:, None])
            s = s.masked_fill(~see, -math.inf)
            top = s.max(1, keepdim=True).values
            p = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
            total_p = p.sum(1, keepdim=True)
            w = p / torch.where(total_p > 0, total_p, torch.ones_like(total_p))
            o[row:row + n, h] = w @ kv[1, h // g]
            mag[row:row + n, h] = w @ kv[1, h // g].abs()
            lse[row:row + n, h] = (top + total_p.log()).squeeze(1)
        row += n
    return o, lse, mag


def check_attn(o, lse, ref):
    """The weights are rounded to bf16 for the product with V: each is off by at most 2^-8 of itself, so a row's sum by
    at most 2^-8 A; the result is rounded once more: 2^-8 |o|.  Scores in 32 bits (an error of 2^-24 per term: with 64 or
    128 terms and the sizes tested here below 2^-12) and the exponentials (2^-12) move a weight and the row's sum by
    less than 2^-10 of themselves together: a quarter of 2^-8 A more.  The log-sum moves by as much as a weight."""
    o_ref, lse_ref, mag = (t.cpu() for t in ref)
    o = o.double().cpu().reshape(o_ref.shape)
    assert torch.isfinite(o).all(), "non-finite output"
    bad = (o - o_ref).abs() > HALF_BF16 * (1.25 * mag + o_ref.abs()) + 1e-30
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, worst {(o - o_ref).abs().max():.3g}"
    if lse is not None:
        lse = lse.double().cpu().reshape(lse_ref.shape)
        empty = torch.isinf(lse_ref)
        assert torch.equal(torch.isinf(lse) & (lse < 0), empty), "empty rows"
        assert (lse - lse_ref)[~empty].abs().le(2.0 ** -10 + 2.0 ** -20 * lse_ref[~empty].abs()).all(), "lse"


class Batch:
    """A batch in a scattered pool whose unused blocks and tail slots hold NaN."""

    def __init__(self, ctx, new, heads=8, kv_heads=2, dim=128, layers=1, seed=0, q_scale=1.0, v_scale=1.0, pad_rows=0, slack_blocks=3,
                 q_stride=None):
        g = torch.Generator().manual_seed(seed)
        self.ctx, self.new, self.heads, self.kv_heads, self.dim = list(ctx), list(new), heads, kv_heads, dim
        need = [blocks_of(c + n) for c, n in zip(ctx, new)]
        self.kv_indptr = offsets(need)
        self.num_blocks = int(self.kv_indptr[-1]) + slack_blocks
        self.kv_indices = torch.randperm(self.num_blocks, generator=g)[:int(self.kv_indptr[-1])].numpy().astype(np.int32)
        self.q_indptr = offsets(new)
        self.rows = int(self.q_indptr[-1])
        self.max_rows = self.rows + pad_rows
        pool = torch.full((layers, self.num_blocks, 2, kv_heads, BS, dim), math.nan)
        for r, (c, n) in enumerate(zip(ctx, new)):
            for j in range(need[r]):
                fill = min(BS, c + n - j * BS)
                vals = torch.randn((layers, 2, kv_heads, fill, dim), generator=g)
                vals[:, 1] *= v_scale
                pool[:, int(self.kv_indices[int(self.kv_indptr[r]) + j]), :, :, :fill] = vals
        self.pool = pool.to(torch.bfloat16).to(DEV)
        width = heads * dim
        self.q_all = torch.zeros((layers, max(1, self.max_rows), q_stride or width), dtype=torch.bfloat16)
        self.q_all[:, :, :width] = (q_scale * torch.randn((layers, max(1, self.max_rows), width), generator=g)).to(torch.bfloat16)
        self.q_all = self.q_all.to(DEV)
        self.q = self.q_all[:, :, :width]
        self.o = torch.full((layers, max(1, self.max_rows), heads, dim), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((layers, max(1, self.max_rows), heads), 7.0, device=DEV)
        self.ctx_len = gpu(np.asarray(ctx, dtype=np.int32))
        self.kvp, self.kvi, self.qp = gpu(self.kv_indptr), gpu(self.kv_indices), gpu(self.q_indptr)

    def context(self, **kw):
        return context(self.heads, self.kv_heads, self.dim, self.num_blocks, max_batch=max(1, len(self.ctx)),
                       num_layers=self.pool.shape[0], **kw)

    def plan(self, c, **masks):
        self.masks = masks
        plan = torch.empty(c.nsd_chunk_plan_bytes(self.max_rows), dtype=torch.uint8, device=DEV)
        c.nsd_chunk_plan(plan, self.max_rows, self.qp, self.ctx_len, self.kvp, window=masks.get("window", 0),
                         prefix_len=None if masks.get("prefix_len") is None else gpu(np.asarray(masks["prefix_len"], dtype=np.int32)),
                         row_first=None if masks.get("row_first") is None else gpu(np.asarray(list(masks["row_first"]) + [0] * (self.max_rows - self.rows), dtype=np.int32)))
        return plan

    def attn(self, c, plan, layer=0, slopes=None, **kw):
        c.nsd_chunk_attn(plan, self.max_rows, self.pool, self.q[layer], self.o[layer], self.lse[layer], self.kvi, layer=layer,
                         alibi_slopes=None if slopes is None else gpu(slopes, torch.float32), **kw)

    def reference(self, layer=0, slopes=None, scale=None, softcap=0.0):
        q = self.q[layer, :self.rows].double().reshape(self.rows, self.heads, self.dim)
        pool = torch.nan_to_num(self.pool[layer].double(), nan=0.0)
        return attn_ref(q, pool, self.ctx, self.new, self.kv_indptr, self.kv_indices, scale=scale, softcap=softcap, slopes=slopes, **self.masks)

    def check(self, layer=0, slopes=None, **kw):
        check_attn(self.o[layer, :self.rows], self.lse[layer, :self.rows], self.reference(layer, slopes, **kw))
        assert (self.o[layer, self.rows:] == 7.0).all() and (self.lse[layer, self.rows:] == 7.0).all(), "padding rows were written"

    def run(self, slopes=None, scale=None, softcap=0.0, **masks):
        c = self.context()
        plan = self.plan(c, **masks)
        for layer in range(self.pool.shape[0]):
            self.attn(c, plan, layer, slopes, softcap=softcap, scale=scale or 0.0)
        assert c.nsd_get_status() == (0, -1)
        for layer in range(self.pool.shape[0]):
            self.check(layer, slopes, scale=scale, softcap=softcap)
        return self
