"""Attention for groups of requests that share a prefix, against the 64-bit definition over every request's whole table."""
import numpy as np
import pytest
import torch

import chunk_testlib as T
from chunk_testlib import BS, DEV, blocks_of, gpu, offsets

pytestmark = pytest.mark.gpu


class Groups(T.Batch):
    """members: requests of each group; shared: common tokens; own / new: committed tokens behind them and new ones, request by
    request.  Full blocks of a prefix are the same ids for all members (or, with `same` false, other ids in the tables of all
    but the first member with rows: entries that are not to be read); its last, partial block is copied."""

    def __init__(self, members, shared, own, new, heads=8, kv_heads=2, dim=128, layers=1, seed=0, same=True, **kw):
        ctx = [p + o for p, o in zip(np.repeat(shared, members).tolist(), own)]
        super().__init__(ctx, new, heads, kv_heads, dim, layers, seed, **kw)
        self.members, self.shared = list(members), list(shared)
        begin = offsets(members)
        self.true_indices = self.kv_indices.copy()
        for k, p in enumerate(shared):
            a, b = int(begin[k]), int(begin[k + 1])
            lead = next((r for r in range(a, b) if new[r]), a)
            n = p // BS
            src = self.kv_indices[int(self.kv_indptr[lead]):]
            for r in range(a, b):
                if r == lead or not new[r]:
                    continue
                at = int(self.kv_indptr[r])
                self.true_indices[at:at + n] = src[:n]
                if same or b - a < 2:
                    self.kv_indices[at:at + n] = src[:n]
                else:                                  # copies in other blocks, spoilt so that a reader would show
                    self.pool[:, torch.as_tensor(self.kv_indices[at:at + n].astype(np.int64), device=DEV)] = float("nan")
                if p % BS:
                    to, frm = int(self.kv_indices[at + n]), int(src[n])
                    self.pool[:, to, :, :, :p % BS] = self.pool[:, frm, :, :, :p % BS]
        self.kvi = gpu(self.kv_indices)
        self.gp, self.prefix = gpu(begin), gpu(np.asarray(shared, dtype=np.int32))

    def plan(self, c):
        self.masks = {}
        plan = torch.empty(c.nsd_prefix_plan_bytes(self.max_rows), dtype=torch.uint8, device=DEV)
        c.nsd_prefix_plan(plan, self.max_rows, self.gp, self.prefix, self.qp, self.ctx_len, self.kvp)
        return plan

    def attn(self, c, plan, layer=0, slopes=None, **kw):
        c.nsd_prefix_attn(plan, self.max_rows, self.pool, self.q[layer], self.o[layer], self.lse[layer], self.kvi, layer=layer,
                          alibi_slopes=None if slopes is None else gpu(slopes, torch.float32), **kw)

    def reference(self, layer=0, slopes=None, scale=None, softcap=0.0):
        q = self.q[layer, :self.rows].double().reshape(self.rows, self.heads, self.dim)
        return T.attn_ref(q, torch.nan_to_num(self.pool[layer].double(), nan=0.0), self.ctx, self.new, self.kv_indptr, self.true_indices, scale=scale,
                          softcap=softcap, slopes=slopes)


SHAPES = [(8, 2, 128), (8, 2, 64), (4, 4, 128), (5, 1, 64), (28, 4, 128), (12, 4, 64), (32, 1, 128), (32, 8, 128)]


def small(shape):
    return dict(heads=shape[0], kv_heads=shape[1], dim=shape[2])


@pytest.mark.parametrize("shape", SHAPES)
def test_groups_of_every_kind(shape):
    """Groups of one and many, prefixes of nothing, within a block, at and around the edges of blocks and key tiles; requests
    with nothing of their own, without new tokens, and with many."""
    members = [1, 3, 2, 5, 2, 4, 1, 6]
    shared = [40, 0, 5, 128, 127, 400, 0, 16]
    own = [3, 0, 17, 1, 0, 30, 0, 128, 5, 0, 31, 0, 1, 200, 0, 16, 15, 50, 0, 7, 129, 0, 300, 2]
    new = [1, 1, 5, 0, 2, 1, 1, 0, 33, 1, 4, 3, 1, 1, 0, 2, 70, 1, 5, 1, 0, 1, 3, 2]
    Groups(members, shared, own, new, pad_rows=5, seed=1, **small(shape)).run()


@pytest.mark.parametrize("p", [1, 15, 16, 17, 127, 128, 129, 1000])
def test_prefix_lengths(p):
    Groups([4], [p], [0, 5, 40, 200], [1, 2, 1, 3], seed=p).run()


@pytest.mark.parametrize("members", [2, 31, 33, 64, 150])
def test_many_members(members):
    rng = np.random.default_rng(members)
    Groups([members], [700], rng.integers(0, 60, members).tolist(), rng.integers(0, 4, members).tolist(), heads=4, kv_heads=1, dim=64, seed=2).run()


def test_long_prefix_split_over_many_ctas():
    Groups([3], [20011], [10, 0, 300], [1, 2, 1], seed=3).run()


def test_long_prefix_and_many_rows():
    rng = np.random.default_rng(4)
    Groups([40], [5003], rng.integers(0, 400, 40).tolist(), rng.integers(1, 6, 40).tolist(), heads=32, kv_heads=8, seed=4).run()


def test_layers_share_a_plan():
    Groups([5, 2], [300, 100], [1, 20, 3, 0, 70, 2, 2], [1, 1, 2, 1, 1, 3, 1], layers=3, seed=5).run()


def test_only_the_first_member_s_prefix_is_read():
    """The other members' entries for the shared blocks name blocks of NaN; the first member has no rows in one group."""
    Groups([3, 4], [200, 64], [5, 40, 0, 9, 1, 0, 33], [1, 2, 1, 0, 1, 1, 5], seed=6, same=False).run()


@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64)])
def test_caps_biases_and_scale(shape):
    slopes = [2.0 ** (-8.0 * (h + 1) / shape[0]) for h in range(shape[0])]
    args = ([3, 2], [250, 33], [5, 0, 100, 40, 1], [1, 2, 3, 1, 40])
    Groups(*args, seed=7, q_scale=6.0, **small(shape)).run(softcap=20.0)
    Groups(*args, seed=8, **small(shape)).run(slopes=slopes)
    Groups(*args, seed=9, **small(shape)).run(slopes=slopes, softcap=5.0, scale=0.3)


def test_the_outcome_is_that_of_the_chunk_attention():
    b = Groups([6], [513], [5, 0, 100, 40, 1, 7], [1, 2, 3, 1, 4, 0], seed=10).run()
    o, lse = b.o.clone(), b.lse.clone()
    c = b.context()
    b.masks = {}
    plan = torch.empty(c.nsd_chunk_plan_bytes(b.max_rows), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, b.max_rows, b.qp, b.ctx_len, b.kvp)
    c.nsd_chunk_attn(plan, b.max_rows, b.pool, b.q[0], b.o[0], b.lse[0], b.kvi)
    # both within a bf16 step of the 64-bit result, plus what the rounding of the weights moves either
    assert (o.double() - b.o.double()).abs().max() <= 2 * 2.0 ** -8 * (1.25 * 4.0 + 4.0)
    assert (lse - b.lse).abs().max() <= 2 * (2.0 ** -10 + 2.0 ** -20 * 20)


def test_nan_in_a_query_stays_in_its_row():
    b = Groups([3], [300], [5, 0, 100], [1, 2, 1], seed=11)
    b.q[0, 2, 128 * 5] = float("nan")
    c = b.context()
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (0, -1)
    bad = torch.zeros((4, 8), dtype=torch.bool, device=DEV)
    bad[2, 5] = True
    assert torch.equal(torch.isnan(b.lse[0, :4]), bad) and torch.equal(torch.isnan(b.o[0, :4]).any(-1), bad)


def test_same_bits_every_time_and_in_a_graph():
    b = Groups([5, 1, 3], [9000, 50, 300], [5, 0, 100, 40, 1, 7, 0, 3, 20], [1, 2, 3, 1, 4, 1, 1, 0, 5], seed=12, pad_rows=3)
    c = b.context()
    plan = b.plan(c)
    b.attn(c, plan)
    o, lse = b.o.clone(), b.lse.clone()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            c.nsd_prefix_plan(plan, b.max_rows, b.gp, b.prefix, b.qp, b.ctx_len, b.kvp, stream=s)
            c.nsd_prefix_attn(plan, b.max_rows, b.pool, b.q[0], b.o[0], b.lse[0], b.kvi, stream=s)
    for _ in range(2):
        b.o.fill_(7.0), b.lse.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, b.o) and torch.equal(lse, b.lse)
    # the captured step with other lengths and groups, within the same buffers
    b2 = Groups([4, 3, 2], [100, 30, 0], [5, 0, 10, 4, 1, 7, 0, 3, 20], [1, 2, 0, 1, 4, 1, 1, 1, 3], seed=13)
    for dst, src in ((b.gp, b2.gp), (b.prefix, b2.prefix), (b.qp, b2.qp), (b.ctx_len, b2.ctx_len), (b.kvp, b2.kvp), (b.q[0, :b2.rows], b2.q[0, :b2.rows])):
        dst.copy_(src)
    b.kvi[:b2.kvi.numel()] = b2.kvi
    b.pool[:, :b2.pool.shape[1]] = b2.pool
    b.o.fill_(7.0), b.lse.fill_(7.0)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert c.nsd_get_status() == (0, -1)
    b2.masks = {}
    T.check_attn(b.o[0, :b2.rows], b.lse[0, :b2.rows], b2.reference())
    assert (b.o[0, b2.rows:] == 7.0).all() and (b.lse[0, b2.rows:] == 7.0).all()
    del graph


def test_malformed_groups_are_reported_and_nothing_is_written():
    i64 = torch.int64
    for groups, prefix in (([0, 2, 4], [10, 10]), ([1, 2, 5], [10, 10]), ([0, 3, 3, 5], [10, 10, 10]), ([0, 4, 2, 5], [10, 10, 10]), ([0, 2, 6], [10, 10]),
                           ([0, 2, 5], [-1, 10]), ([0, 2, 5], [10, 31]), ([-1, 2, 5], [10, 10])):
        b = Groups([2, 3], [10, 10], [5, 30, 20, 21, 60], [1, 1, 1, 2, 1], seed=14)
        b.gp, b.prefix = gpu(torch.tensor(groups, dtype=i64)), gpu(torch.tensor(prefix, dtype=torch.int32))
        c = b.context()
        b.attn(c, b.plan(c))
        assert c.nsd_get_status()[0] == 6, (groups, prefix)
        assert (b.o == 7.0).all() and (b.lse == 7.0).all()
        assert c.nsd_get_status() == (0, -1)


def test_a_request_without_rows_may_be_shorter_than_the_prefix():
    b = Groups([3], [64], [5, 30, 20], [1, 0, 2], seed=15)
    b.ctx_len[1] = 3
    c = b.context()
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (0, -1)
    b.check()


def test_plans_of_other_kinds_are_refused_on_the_device():
    b = Groups([2], [64], [5, 30], [1, 1], seed=16)
    c = b.context()
    plan = torch.empty(c.nsd_prefix_plan_bytes(2), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, 2, b.qp, b.ctx_len, b.kvp)
    b.attn(c, plan)
    assert c.nsd_get_status()[0] == 6 and (b.o == 7.0).all()
    plan = b.plan(c)
    c.nsd_chunk_attn(plan, 2, b.pool, b.q[0], b.o[0], b.lse[0], b.kvi)
    assert c.nsd_get_status()[0] == 6 and (b.o == 7.0).all()


def test_an_empty_batch():
    b = Groups([2], [64], [5, 30], [0, 0], seed=17, pad_rows=3).run()
    assert (b.o == 7.0).all()
    c = b.context()
    plan = torch.empty(c.nsd_prefix_plan_bytes(3), dtype=torch.uint8, device=DEV)
    none = torch.zeros(1, dtype=torch.int64, device=DEV)
    c.nsd_prefix_plan(plan, 3, none, none[:0].int(), none, none[:0].int(), none)
    b.attn(c, plan)
    assert c.nsd_get_status() == (0, -1) and (b.o == 7.0).all()
