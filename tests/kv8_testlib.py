"""Plain 64-bit forms of the 8-bit cache's operators, from the definitions, with the tolerances of the GPU tests."""
from __future__ import annotations

import math

import numpy as np
import torch

import chunk_testlib as T
from chunk_testlib import BS, DEV, blocks_of, gpu, offsets

NAN_CODE = 0x7F


# --------------------------------------------------------------------------- the format
def grid():
    """The value of every e4m3 code: sign, four bits of exponent with bias 7, three of mantissa; 0x7f and 0xff are NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where(c & 0x80, -v, v)
    v[[0x7F, 0xFF]] = np.nan
    return v


def exponent(top):
    """The least integer e >= -126 with top <= 448 * 2^e."""
    top = np.asarray(top, dtype=np.float64)
    e = np.full(top.shape, -126)
    for _ in range(300):
        small = top > 448.0 * 2.0 ** e.astype(np.float64)
        if not small.any():
            break
        e[small] += 1
    return e


def nearest(y):
    """The e4m3 value next to each y (|y| <= 448), ties to the even code, by search in the whole grid."""
    pos = grid()[:127]                                     # 0 .. 448, codes in order of value
    a = np.abs(y)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = pos[hi] - a, a - pos[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.copysign(pos[code], y)


def quantise(x):
    """x [...][D] float64 -> (values of the codes, exponents); NaN and infinities become NaN."""
    finite = np.isfinite(x)
    e = exponent(np.where(finite, np.abs(x), 0.0).max(-1))
    y = np.where(finite, x, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    return np.where(finite, nearest(y), np.nan), e


def code_values(codes):
    return grid()[codes.view(torch.uint8).cpu().numpy() if torch.is_tensor(codes) else codes]


def random_cache(shape, generator, device="cpu"):
    """Codes and scales of blocks [...][blocks][2][hkv][16][D] as quantising normal rows of unlike size leaves them, and
    the values they stand for (float64)."""
    x = torch.randn(shape, generator=generator, dtype=torch.float64)
    x *= torch.exp2(torch.randint(-3, 4, shape[:-1] + (1,), generator=generator).double())
    values, e = quantise(x.numpy())
    codes = torch.from_numpy(values).to(torch.float8_e4m3fn)
    scales = torch.from_numpy((e + 127).astype(np.uint8)).transpose(-3, -2).contiguous()     # [block][hkv][K|V][slot]
    return codes, scales, torch.from_numpy(values * 2.0 ** e[..., None])


# --------------------------------------------------------------------------- attention
class Batch8(T.Batch):
    """A batch over an 8-bit cache whose unused blocks and tail slots hold NaN codes and scales that are not numbers."""

    def __init__(self, ctx, new, heads=8, kv_heads=2, dim=128, layers=1, seed=0, q_scale=1.0, pad_rows=0, slack_blocks=3, q_stride=None):
        super().__init__(ctx, new, heads, kv_heads, dim, layers, seed, q_scale, 1.0, pad_rows, slack_blocks, q_stride)
        g = torch.Generator().manual_seed(seed + 1)
        codes, scales, values = random_cache((layers, self.num_blocks, 2, kv_heads, BS, dim), g)
        held = ~torch.isnan(self.pool.float().cpu()).any(-1)                                 # [layer][block][K|V][hkv][slot]
        self.kv8 = torch.where(held[..., None], codes.view(torch.uint8), torch.tensor(NAN_CODE, dtype=torch.uint8)).to(DEV)
        self.scales = torch.where(held.transpose(2, 3), scales, torch.tensor(255, dtype=torch.uint8)).contiguous().to(DEV)
        self.values = torch.where(held[..., None], values, torch.tensor(0.0, dtype=torch.float64)).to(DEV)
        del self.pool

    def set_rows(self, layer, kv, token_values, request=0):
        """Writes K (kv = 0) or V of every token of a request: token_values [tokens][hkv][D] float64."""
        values, e = quantise(np.asarray(token_values, dtype=np.float64))
        codes = torch.from_numpy(values).to(torch.float8_e4m3fn).view(torch.uint8).to(DEV)
        for t in range(len(values)):
            b, s = int(self.kv_indices[int(self.kv_indptr[request]) + t // BS]), t % BS
            self.kv8[layer, b, kv, :, s] = codes[t]
            self.scales[layer, b, :, kv, s] = torch.from_numpy((e[t] + 127).astype(np.uint8)).to(DEV)
            self.values[layer, b, kv, :, s] = torch.from_numpy(values[t] * 2.0 ** e[t][:, None]).to(DEV)

    def context(self, **kw):
        return T.context(self.heads, self.kv_heads, self.dim, self.num_blocks, max_batch=max(1, len(self.ctx)), num_layers=self.kv8.shape[0], **kw)

    def plan(self, c, **masks):
        self.masks = masks
        plan = torch.empty(c.nsd_kv8_plan_bytes(self.max_rows), dtype=torch.uint8, device=DEV)
        c.nsd_kv8_plan(plan, self.max_rows, self.qp, self.ctx_len, self.kvp, window=masks.get("window", 0),
                       prefix_len=None if masks.get("prefix_len") is None else gpu(np.asarray(masks["prefix_len"], dtype=np.int32)),
                       row_first=None if masks.get("row_first") is None else gpu(np.asarray(list(masks["row_first"]) + [0] * (self.max_rows - self.rows), dtype=np.int32)))
        return plan

    def attn(self, c, plan, layer=0, **kw):
        c.nsd_kv8_attn(plan, self.max_rows, self.kv8, self.scales, self.q[layer], self.o[layer], self.lse[layer], self.kvi, layer=layer, **kw)

    def reference(self, layer=0, scale=None):
        q = self.q[layer, :self.rows].double().reshape(self.rows, self.heads, self.dim)
        return T.attn_ref(q, self.values[layer], self.ctx, self.new, self.kv_indptr, self.kv_indices, scale=scale, **self.masks)

    def check(self, layer=0, **kw):
        longest = max([c + n for c, n in zip(self.ctx, self.new)], default=0)
        check_attn8(self.o[layer, :self.rows], self.lse[layer, :self.rows], self.reference(layer, **kw), longest, self.values[layer, :, 1].abs().max())
        assert (self.o[layer, self.rows:] == 7.0).all() and (self.lse[layer, self.rows:] == 7.0).all(), "padding rows were written"

    def run(self, scale=None, **masks):
        c = self.context()
        plan = self.plan(c, **masks)
        for layer in range(self.kv8.shape[0]):
            self.attn(c, plan, layer, scale=scale or 0.0)
        assert c.nsd_get_status() == (0, -1)
        for layer in range(self.kv8.shape[0]):
            self.check(layer, scale=scale)
        return self


def check_attn8(o, lse, ref, keys, v_max):
    """q and the cache's values are multiplied exactly, sums and scores are held in 32 bits: as in the 16-bit form a weight
    and a row's sum move by less than 2^-10 of themselves.  The weights are rounded to 11 bits (half a step: 2^-11 of the
    weight) and, where they are small, to multiples: off by at most 2^-25 as 16-bit floats and 2^-24 in the third term, where
    a row's largest weight is 2^4 at least and V's power of two at most twice the largest |v|'s.  So each weight is off by less
    than 2^-24 of the largest one, which is at most 1, against the largest |v|.  The result is rounded to bf16: 2^-8 |o|."""
    o_ref, lse_ref, mag = (t.cpu() for t in ref)
    o = o.double().cpu().reshape(o_ref.shape)
    assert torch.isfinite(o).all(), "non-finite output"
    limit = T.HALF_BF16 * o_ref.abs() + (2.0 ** -10 + 2.0 ** -11) * mag + 2.0 ** -24 * keys * float(v_max) + 1e-30
    bad = (o - o_ref).abs() > limit
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, worst {(o - o_ref).abs().max():.3g}"
    lse = lse.double().cpu().reshape(lse_ref.shape)
    empty = torch.isinf(lse_ref)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty), "empty rows"
    assert (lse - lse_ref)[~empty].abs().le(2.0 ** -10 + 2.0 ** -20 * lse_ref[~empty].abs()).all(), "lse"


class K8Run:
    """Three requests that grow by a few tokens per step, through block tables, append, plan and attention."""

    def __init__(self, steps=((20, 5, 130), (1, 4, 3), (2, 1, 5)), heads=8, kv_heads=2, dim=128, seed=1):
        self.steps, self.heads, self.kv_heads, self.dim = steps, heads, kv_heads, dim
        self.g = torch.Generator().manual_seed(seed)

    def check(self):
        h, hkv, d, batch, blocks = self.heads, self.kv_heads, self.dim, len(self.steps[0]), 64
        c = T.context(h, hkv, d, num_blocks=blocks, max_batch=batch)
        kv8 = torch.full((1, blocks, 2, hkv, BS, d), NAN_CODE, dtype=torch.uint8, device=DEV)
        scales = torch.full((1, blocks, hkv, 2, BS), 255, dtype=torch.uint8, device=DEV)
        pool = torch.full((1, blocks, 2, hkv, BS, d), math.nan, dtype=torch.bfloat16, device=DEV)
        held = torch.full((batch, 16), -1, dtype=torch.int32, device=DEV)
        n_held, free = torch.zeros(batch, dtype=torch.int32, device=DEV), torch.randperm(blocks, generator=self.g).to(torch.int32).to(DEV)
        begin = torch.zeros(1, dtype=torch.int64, device=DEV)
        ctx = torch.zeros(batch, dtype=torch.int32, device=DEV)
        values = torch.zeros((blocks, 2, hkv, BS, d), dtype=torch.float64, device=DEV)
        for new in self.steps:
            rows = sum(new)
            i64, i32 = dict(dtype=torch.int64, device=DEV), dict(dtype=torch.int32, device=DEV)
            kvp, kvi, qp, slots = torch.zeros(batch + 1, **i64), torch.zeros(blocks, **i32), torch.zeros(batch + 1, **i64), torch.zeros(rows, **i64)
            n_new, end = torch.zeros(batch, **i32), torch.zeros(1, **i64)
            new_len = torch.tensor(new, **i32)
            c.nsd_block_tables(ctx, new_len, held, n_held, free, begin, kvp, kvi, qp, slots, None, None, n_new, end)
            k, v = (torch.randn((rows, hkv, d), generator=self.g).to(torch.bfloat16).to(DEV) for _ in range(2))
            q = torch.randn((rows, h, d), generator=self.g).to(torch.bfloat16).to(DEV)
            c.nsd_kv8_append(kv8, scales, 0, None, k, v, None, slots)
            pool[0, slots // BS, 0, :, slots % BS] = k
            pool[0, slots // BS, 1, :, slots % BS] = v
            plan = torch.empty(c.nsd_kv8_plan_bytes(rows), dtype=torch.uint8, device=DEV)
            c.nsd_kv8_plan(plan, rows, qp, ctx, kvp)
            outs = []
            packed = torch.zeros_like(kv8), torch.zeros_like(scales)
            ids = torch.arange(blocks, **i32)
            c.nsd_kv8_pack(torch.nan_to_num(pool), *packed, ids, ids)
            for cache in ((kv8, scales), packed):
                o, lse = torch.zeros((rows, h, d), dtype=torch.bfloat16, device=DEV), torch.zeros((rows, h), device=DEV)
                c.nsd_kv8_attn(plan, rows, *cache, q, o, lse, kvi)
                outs.append((o, lse))
            assert c.nsd_get_status() == (0, -1)
            assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
            for j, x in enumerate((k, v)):
                got, e = quantise(x.double().cpu().numpy())
                values[slots // BS, j, :, slots % BS] = torch.from_numpy(got * 2.0 ** e[..., None]).to(DEV)
            ref = T.attn_ref(q.double(), values, ctx.tolist(), list(new), kvp.tolist(), kvi.cpu().numpy())
            check_attn8(*outs[0], ref, int((ctx + new_len).max()), values[:, 1].abs().max())
            ctx, n_held, begin = ctx + new_len, n_new, end
