"""Contexts in which single keys decide the result: each row's query points at one marked key, whose score stands 24 nats
above the rest, so the row's output is that key's V, or, where the mask hides it, a mean that it would drown.  One key too few or
too many then moves an output by its whole size, however long the context is."""
from __future__ import annotations

import numpy as np
import torch

from chunk_testlib import BS, attn_ref, blocks_of, offsets

NATS = 24.0


class Marked:
    """Requests that share one sequence: request r has its first ctx[r] + new[r] tokens.  marks: positions of marked keys."""

    def __init__(self, ctx, new, heads, kv_heads, dim, marks, seed=0, device="cpu"):
        g = torch.Generator().manual_seed(seed)
        self.ctx, self.new, self.heads, self.kv_heads, self.dim, self.device = list(ctx), list(new), heads, kv_heads, dim, device
        total = max(c + n for c, n in zip(ctx, new))
        self.marks = sorted({int(t) for t in marks if 0 <= t < total})
        size = (NATS / dim ** 0.5) ** 0.5              # q . k / sqrt(dim) = size^2 sqrt(dim) for a query that points at the key
        self.point = (size * (2 * torch.randint(0, 2, (len(self.marks), dim), generator=g) - 1)).to(torch.bfloat16)
        blocks = blocks_of(total)
        k, v = torch.randn((2, blocks * BS, kv_heads, dim), generator=g)
        k[self.marks] = self.point.float()[:, None]
        kv = torch.stack([k, v]).view(2, blocks, BS, kv_heads, dim).permute(1, 0, 3, 2, 4)
        self.num_blocks = blocks + 2
        table = torch.randperm(self.num_blocks, generator=g)[:blocks]
        pool = torch.full((1, self.num_blocks, 2, kv_heads, BS, dim), float("nan"))
        pool[0, table] = kv
        self.pool = pool.to(torch.bfloat16).to(device)
        need = [blocks_of(c + n) for c, n in zip(ctx, new)]
        self.kv_indptr, self.q_indptr = offsets(need), offsets(new)
        self.kv_indices = np.concatenate([table[:n].numpy() for n in need]).astype(np.int32)
        self.rows = int(self.q_indptr[-1])
        self.pos = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)])

    def queries(self, wanted):
        """wanted(position of the row) = marked keys; turn by turn over rows and heads.  Yields q until each had its turn with
        every head."""
        at = {t: i for i, t in enumerate(self.marks)}
        lists = [[at[t] for t in dict.fromkeys(int(x) for x in wanted(int(p))) if t in at] or [0] for p in self.pos]
        for turn in range(max(len(x) for x in lists)):
            pick = torch.tensor([[x[(turn + h + i) % len(x)] for h in range(self.heads)] for i, x in enumerate(lists)])
            yield self.point[pick].to(self.device)

    def reference(self, q, **kw):
        pool = torch.nan_to_num(self.pool[0].double(), nan=0.0)
        return attn_ref(q.double(), pool, self.ctx, self.new, self.kv_indptr, self.kv_indices, **kw)


def edges(total, step):
    return [t for e in range(0, total + step, step) for t in (e - 1, e)]
