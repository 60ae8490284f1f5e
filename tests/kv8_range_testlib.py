"""Batches over the 8-bit cache whose rows of V differ by any power of two, and a limit of each output from its own row."""
from __future__ import annotations

import math

import numpy as np
import torch

import chunk_testlib as T
from chunk_testlib import BS, DEV
from kv8_testlib import Batch8

LEAST = 2.0 ** -133                                    # a step of bf16's smallest numbers


class Range8(Batch8):
    """Every query has 8 in its first dim and every key 0 there, so that `point` sets the score of one key for all rows: any
    number of half steps of 8 c / sqrt(dim), apart from the others' scores of order one."""

    def __init__(self, ctx, new, **kw):
        super().__init__(ctx, new, **kw)
        self.q.view(*self.q.shape[:2], self.heads, self.dim)[..., 0] = 8.0
        held = self.kv8[:, :, 0, :, :, 0] != 0x7F
        self.kv8[:, :, 0, :, :, 0] = torch.where(held, 0, 0x7F).to(torch.uint8)
        self.values[:, :, 0, :, :, 0] = 0.0

    def place(self, request, token):
        return int(self.kv_indices[int(self.kv_indptr[request]) + token // BS]), token % BS

    def places(self, request, tokens=None):
        t = np.arange(self.ctx[request] + self.new[request]) if tokens is None else np.asarray(tokens)
        blocks = self.kv_indices[int(self.kv_indptr[request]) + t // BS]
        return torch.from_numpy(blocks.astype(np.int64)).to(DEV), torch.from_numpy(t % BS).to(DEV)

    def shift_v(self, request, by, tokens=None, layer=0):
        """Rows of V times 2^by (a number, or one per token)."""
        b, s = self.places(request, tokens)
        by = torch.as_tensor(np.broadcast_to(np.asarray(by), (len(b),)).copy(), device=DEV)
        byte = self.scales[layer, b, :, 1, s].long() + by[:, None]
        assert int(byte.min()) >= 0 and int(byte.max()) <= 247
        self.scales[layer, b, :, 1, s] = byte.to(torch.uint8)
        self.values[layer, b, 1, :, s] *= torch.exp2(by.double())[:, None, None]

    def clear_v(self, request, tokens=None, layer=0):
        b, s = self.places(request, tokens)
        self.kv8[layer, b, 1, :, s] = 0
        self.scales[layer, b, :, 1, s] = 1             # what a row of zeros is stored as
        self.values[layer, b, 1, :, s] = 0.0

    def point(self, request, token, score, layer=0):
        """The key of one token has this score (to the next e4m3 number) in every row: the code in its first dim, and nothing else."""
        c = torch.tensor([score * math.sqrt(self.dim) / 8.0]).clamp(-448, 448).to(torch.float8_e4m3fn)
        b, s = self.place(request, token)
        self.kv8[layer, b, 0, :, s] = 0
        self.kv8[layer, b, 0, :, s, 0] = c.view(torch.uint8).to(DEV)
        self.scales[layer, b, :, 0, s] = 127
        self.values[layer, b, 0, :, s] = 0.0
        self.values[layer, b, 0, :, s, 0] = c.double().to(DEV)

    def close(self, layer=0, scale=None, rows=None, **masks):
        """Whether the outputs of `rows` (all) are right to close8's limit."""
        q = self.q[layer, :self.rows].double().reshape(self.rows, self.heads, self.dim)
        ref = T.attn_ref(q, self.values[layer], self.ctx, self.new, self.kv_indptr, self.kv_indices, scale=scale, **masks)
        part = largest(q, self.values[layer], self.ctx, self.new, self.kv_indptr, self.kv_indices, ref[1], scale, **masks)
        longest = max(c + n for c, n in zip(self.ctx, self.new))
        at = list(range(self.rows)) if rows is None else list(rows)
        close8(self.o[layer, at], self.lse[layer, at], [t[at] for t in ref], part[at], longest)

    def run_close(self, scale=None, **masks):
        c = self.context()
        plan = self.plan(c, **masks)
        self.attn(c, plan, scale=scale or 0.0)
        assert c.nsd_get_status() == (0, -1)
        self.close(scale=scale, **masks)
        return self


def largest(q, values, ctx, new, kv_indptr, kv_indices, lse, scale, **masks):
    """[rows][heads]: the largest product of a key's weight and its largest |v| that each row sees."""
    rows, hq, d = q.shape
    hkv = values.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    seen = T.visible(ctx, new, **masks)
    out, row = torch.zeros((rows, hq), dtype=torch.float64, device=q.device), 0
    for r, (c, n) in enumerate(zip(map(int, ctx), map(int, new))):
        if not n:
            continue
        at = int(kv_indptr[r])
        table = torch.as_tensor(np.asarray(kv_indices[at:at + T.blocks_of(c + n)]).astype(np.int64), device=q.device)
        kv = values[table].permute(1, 2, 0, 3, 4).reshape(2, hkv, -1, d)[:, :, :c + n]
        span, key = torch.tensor(seen[row:row + n], device=q.device), torch.arange(c + n, device=q.device)
        see = (key[None] >= span[:, :1]) & (key[None] < span[:, 1:])
        for h in range(hq):
            s = q[row:row + n, h] @ kv[0, h * hkv // hq].T * scale
            w = torch.exp(torch.where(see, s - lse[row:row + n, h, None], torch.tensor(-math.inf, dtype=torch.float64, device=q.device)))
            out[row:row + n, h] = (w * kv[1, h * hkv // hq].abs().amax(-1)).nan_to_num(0.0).max(1).values
        row += n
    return out


def close8(o, lse, ref, part, keys):
    """Weights and a row's sum move by less than 2^-10 of themselves through scores and exponentials in 32 bits, as in the 16-bit
    form.  A weight times its key's power of two is rounded to 11 bits (half a step: 2^-11 of it) and, where it is small, to
    multiples: off by at most 2^-25 as a 16-bit float and 2^-24 in its third term, 2^-23.4 together, where the row's largest such
    product is 2^3 at least.  A code is 448 at most, and the largest one of a row 224 at least (its power of two is the least
    that holds it), so a key moves an element by less than 2^-23.4 448 / (2^3 224) < 2^-25 of `part`, the largest product of a
    weight and a row's largest |v|.  The result is rounded to bf16: 2^-8 |o|, or a step of its smallest numbers."""
    o_ref, lse_ref, mag = (t.cpu() for t in ref)
    o, lse = o.double().cpu().reshape(o_ref.shape), lse.double().cpu().reshape(lse_ref.shape)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all(), "non-finite output"
    limit = T.HALF_BF16 * o_ref.abs() + (2.0 ** -10 + 2.0 ** -11) * mag + 2.0 ** -25 * keys * part.cpu()[..., None] + LEAST
    off = (o - o_ref).abs() / limit
    assert (off <= 1).all(), f"{int((off > 1).sum())} of {off.numel()} outside, worst {off.max():.3g} of the limit"
    assert ((lse - lse_ref).abs() <= 2.0 ** -10 + 2.0 ** -20 * lse_ref.abs()).all(), "lse"
