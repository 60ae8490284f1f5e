"""Block tables from request lengths, rotary positions fused with the append, and the whole step they belong to."""
import numpy as np
import pytest
import torch

from chunk_testlib import BS, DEV, HALF_BF16, attn_ref, blocks_of, check_attn, context, gpu, offsets, rope_ref, tables_ref

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- block tables
class Tables:
    def __init__(self, ctx, new, seed=0, extra=0, begin=0, pad_rows=5, spare_entries=6, stride=None, max_batch=None):
        rng = np.random.default_rng(seed)
        self.ctx, self.new = np.asarray(ctx, dtype=np.int32), np.asarray(new, dtype=np.int32)
        n = len(self.ctx)
        n_held = np.asarray([blocks_of(c) + (int(rng.integers(0, extra + 1))) for c in self.ctx], dtype=np.int32)
        need = [blocks_of(int(c) + int(m)) for c, m in zip(self.ctx, self.new)]
        self.stride = stride or max([1] + need + n_held.tolist()) + 2
        take = sum(max(0, a - int(b)) for a, b in zip(need, n_held))
        self.num_blocks = int(n_held.sum()) + take + begin + 10
        ids = rng.permutation(self.num_blocks).astype(np.int32)
        self.held = np.full((max(n, 1), self.stride), -5, dtype=np.int32)
        at = 0
        for r in range(n):
            self.held[r, :n_held[r]] = ids[at:at + n_held[r]]
            at += int(n_held[r])
        self.n_held, self.free, self.begin = n_held, ids[at:], begin
        self.entries, self.rows = int(sum(need)), int(self.new.sum())
        self.t = dict(ctx_len=gpu(self.ctx), new_len=gpu(self.new), held=gpu(self.held), n_held=gpu(n_held), free_blocks=gpu(self.free),
                      free_begin=gpu(np.asarray([begin], dtype=np.int64)),
                      kv_indptr=torch.full((n + 1,), -9, dtype=torch.int64, device=DEV),
                      kv_indices=torch.full((self.entries + spare_entries,), -9, dtype=torch.int32, device=DEV),
                      q_indptr=torch.full((n + 1,), -9, dtype=torch.int64, device=DEV),
                      slot_map=torch.full((self.rows + pad_rows,), -9, dtype=torch.int64, device=DEV),
                      positions=torch.full((self.rows + pad_rows,), -9, dtype=torch.int32, device=DEV),
                      row_req=torch.full((self.rows + pad_rows,), -9, dtype=torch.int32, device=DEV),
                      n_held_new=torch.full((max(n, 1),), -9, dtype=torch.int32, device=DEV),
                      free_end=torch.full((1,), -9, dtype=torch.int64, device=DEV))
        self.c = context(8, 2, 64, self.num_blocks, max_batch=max_batch or max(1, n))

    def call(self, **over):
        self.c.nsd_block_tables(**{**self.t, **over})

    def check(self):
        held, n_held, kvp, kvi, qp, slots, pos, owner, end = tables_ref(self.ctx, self.new, self.held[:len(self.ctx)], self.n_held, self.free, self.begin)
        got = {k: v.cpu().numpy() for k, v in self.t.items()}
        assert np.array_equal(got["kv_indptr"], kvp) and np.array_equal(got["q_indptr"], qp)
        assert got["kv_indices"][:self.entries].tolist() == kvi and (got["kv_indices"][self.entries:] == -9).all()
        assert got["slot_map"][:self.rows].tolist() == slots and (got["slot_map"][self.rows:] == -1).all()
        assert got["positions"][:self.rows].tolist() == pos and (got["positions"][self.rows:] == 0).all()
        assert got["row_req"][:self.rows].tolist() == owner and (got["row_req"][self.rows:] == -1).all()
        if len(self.ctx):
            assert got["held"].tolist() == held and got["n_held_new"].tolist() == n_held
        assert got["free_end"][0] == end


@pytest.mark.parametrize("batch", [0, 1, 2, 31, 255, 256, 257, 700])
def test_tables_of_many_batches(batch):
    rng = np.random.default_rng(batch)
    t = Tables(rng.integers(0, 100, batch), rng.integers(0, 40, batch), seed=batch, extra=2, begin=3)
    t.call()
    assert t.c.nsd_get_status() == (0, -1)
    t.check()


@pytest.mark.parametrize("ctx,new", [([0], [1]), ([0], [0]), ([15, 16, 17], [1, 1, 1]), ([0, 0, 0, 9], [0, 5000, 0, 1]), ([70000], [1]),
                                     ([3] * 20 + [0] + [3] * 20, [1] * 20 + [40000] + [0] * 20)])
def test_tables_of_unequal_requests(ctx, new):
    t = Tables(ctx, new, seed=1, extra=1)
    t.call()
    assert t.c.nsd_get_status() == (0, -1)
    t.check()


def test_row_outputs_may_be_left_out():
    t = Tables([5, 40], [3, 20], seed=2)
    t.call(slot_map=None, positions=None, row_req=None)
    assert t.c.nsd_get_status() == (0, -1)
    for k in ("slot_map", "positions", "row_req"):
        t.t[k].fill_(0)
    t.call(positions=None)
    assert (t.t["positions"] == 0).all()
    t.call(free_begin=None)
    assert t.c.nsd_get_status() == (0, -1)


def test_a_free_list_that_runs_out():
    t = Tables([0, 0, 0], [20, 40, 33], seed=3)                # 2, 3 and 3 blocks
    t.call(free_blocks=t.t["free_blocks"][:4].contiguous())
    assert t.c.nsd_get_status() == (6, 1)
    free = t.free.tolist()
    assert t.t["kv_indices"][:8].tolist() == free[:4] + [-1] * 4
    assert t.t["n_held_new"].tolist() == [2, 2, 0] and t.t["free_end"].item() == 4
    slots = t.t["slot_map"].tolist()
    assert slots[20:52] == [free[2 + i // 16] * BS + i % 16 for i in range(32)] and all(s == -1 for s in slots[52:])
    assert t.t["held"][1].tolist()[2:] == [-5] * (t.stride - 2)


@pytest.mark.parametrize("what", ["context", "new", "stride", "held"])
def test_a_malformed_request_counts_as_empty(what):
    t = Tables([20, 30, 40], [5, 6, 7], seed=4)
    over = {}
    if what == "context":
        over["ctx_len"] = gpu(np.asarray([20, -1, 40], dtype=np.int32))
    elif what == "new":
        over["new_len"] = gpu(np.asarray([5, -6, 7], dtype=np.int32))
    elif what == "stride":
        over["new_len"] = gpu(np.asarray([5, 16 * t.stride, 7], dtype=np.int32))
    else:
        over["n_held"] = gpu(np.asarray([2, 1, 3], dtype=np.int32))
    t.call(**over)
    assert t.c.nsd_get_status() == (6, 1)
    assert t.t["q_indptr"].tolist() == [0, 5, 5, 12]
    assert t.t["kv_indptr"].tolist() == [0, 2, 2, 5]
    assert t.t["positions"][:12].tolist() == list(range(20, 25)) + list(range(40, 47))


def test_a_bad_block_id_gives_no_slot():
    t = Tables([20, 30], [5, 6], seed=5)
    t.t["held"][1, 1] = t.num_blocks
    t.call()
    assert t.c.nsd_get_status() == (6, 1)
    assert t.t["slot_map"][5:7].tolist() == [-1, -1] and (t.t["slot_map"][7:11] >= 0).all()     # positions 30, 31 | 32 ..


def test_outputs_that_are_too_small_are_not_overrun():
    t = Tables([20, 30], [5, 60], seed=6)
    t.call(kv_indices=t.t["kv_indices"][:4], slot_map=t.t["slot_map"][:10], positions=t.t["positions"][:10], row_req=t.t["row_req"][:10])
    assert t.c.nsd_get_status()[0] == 6
    assert (t.t["kv_indices"][4:] == -9).all() and (t.t["slot_map"][10:] == -9).all() and (t.t["positions"][10:] == -9).all()
    assert (t.t["row_req"][10:] == -9).all()


def test_tables_refusals():
    import paper_2609_29364_b200 as nsd

    t = Tables([20, 30], [5, 6], seed=7)
    small = context(8, 2, 64, 64, max_batch=1)

    def refused(code, f):
        with pytest.raises(nsd.NsdError) as e:
            f()
        assert e.value.code == code

    refused(2, lambda: small.nsd_block_tables(**t.t))
    refused(1, lambda: t.call(n_held_new=t.t["n_held"]))
    refused(1, lambda: t.call(free_end=t.t["free_begin"]))
    refused(1, lambda: t.call(kv_indptr=None))
    with pytest.raises(TypeError):
        t.call(ctx_len=t.t["ctx_len"].long())
    with pytest.raises(ValueError):
        t.call(slot_map=t.t["slot_map"][:3])
    with pytest.raises(ValueError):
        t.call(q_indptr=t.t["q_indptr"][:1])


# --------------------------------------------------------------------------- rotary positions
class Rope:
    def __init__(self, rows, heads=8, kv_heads=2, dim=128, dtype=torch.bfloat16, axes=1, far=4096, pad=0, seed=0, offset=0, tail=0):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.heads, self.kv_heads, self.dim, self.axes, self.pad = rows, heads, kv_heads, dim, axes, pad
        width = (heads + 2 * kv_heads) * dim
        n = rows + pad
        flat = torch.randn(n * (width + tail) + offset, generator=g).to(dtype).to(DEV)
        self.qkv = flat[offset:].view(n, width + tail)
        nq, nk = heads * dim, kv_heads * dim
        self.q, self.k, self.v = self.qkv[:, :nq], self.qkv[:, nq:nq + nk], self.qkv[:, nq + nk:nq + 2 * nk]
        self.positions = torch.randint(0, far, (axes, n), generator=g, dtype=torch.int32).to(DEV)
        self.num_blocks = blocks_of(rows + 3) + 2
        ids = torch.randperm(self.num_blocks, generator=g)
        at = torch.arange(rows) + 3
        slots = torch.full((n,), -1, dtype=torch.int64)
        real = torch.randperm(n, generator=g)[:rows].sort().values if pad else torch.arange(rows)
        slots[real] = ids[at // BS] * BS + at % BS
        self.real, self.slots = real, slots.to(DEV)
        self.pool = torch.randn((2, self.num_blocks, 2, kv_heads, BS, dim), generator=g).to(torch.bfloat16).to(DEV)
        self.q_out = torch.full((n, heads, dim), 3.0, dtype=torch.bfloat16, device=DEV)
        self.c = context(heads, kv_heads, dim, self.num_blocks, num_layers=2)

    def run_and_check(self, sections, adjacent=False, cycled=False, layer=1, inv_freq=None, with_q=True, with_kv=True, in_place=False):
        pairs = sum(sections)
        inv_freq = inv_freq if inv_freq is not None else (1e4 ** (-np.arange(pairs) / pairs)).astype(np.float32)
        before = self.qkv.double().cpu().numpy()
        pool0 = self.pool.clone()
        q_out = self.q if in_place else self.q_out
        q_before = q_out.clone()
        self.c.nsd_rope_append(self.pool, layer, self.q if with_q else None, self.k if with_kv else None, self.v if with_kv else None,
                               q_out if with_q else None, self.positions, sections, gpu(inv_freq), self.slots, adjacent=adjacent, cycled=cycled)
        assert self.c.nsd_get_status() == (0, -1)
        n, h, hk, d = before.shape[0], self.heads, self.kv_heads, self.dim
        heads = before[:, :(h + 2 * hk) * d].reshape(n, h + 2 * hk, d)
        y, slack = rope_ref(heads[:, :h + hk], self.positions.cpu().numpy(), sections, inv_freq, adjacent, cycled)
        real, slots = self.real.numpy(), self.slots.cpu().numpy()
        turned = np.abs(y - heads[:, :h + hk]).max() > 0

        def near(got, want, more):
            assert (np.abs(got - want) <= HALF_BF16 * np.abs(want) + 1.01 * more).all()
            assert turned

        if with_q:
            got = q_out.double().cpu().numpy().reshape(n, h, d)
            near(got[real], y[real, :h], slack[real, :h])
            rest = np.setdiff1d(np.arange(n), real)
            assert torch.equal(q_out.reshape(n, -1)[rest], q_before.reshape(n, -1)[rest]), "padding rows were written"
        want = pool0.clone()
        if with_kv:
            b, t = self.slots[self.real.to(DEV)] // BS, self.slots[self.real.to(DEV)] % BS
            got = self.pool[layer][b, 0, :, t].double().cpu().numpy()
            near(got, y[real, h:], slack[real, h:])
            want[layer][b, 0, :, t] = self.pool[layer][b, 0, :, t]
            want[layer][b, 1, :, t] = torch.from_numpy(heads[real, h + hk:]).to(DEV).float().to(torch.bfloat16)
        assert torch.equal(self.pool.view(torch.int16), want.view(torch.int16)), "values, other slots or the other layer differ"
        assert slots.shape[0] == n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dim,pairs", [(128, 64), (128, 32), (128, 8), (128, 29), (128, 1), (64, 32), (64, 16), (64, 5), (64, 24)])
def test_rope_pairs_and_types(dim, pairs, adjacent, dtype):
    Rope(37, dim=dim, dtype=dtype, seed=pairs).run_and_check([pairs], adjacent)


@pytest.mark.parametrize("rows", [1, 2, 7, 64, 1000, 3000])
@pytest.mark.parametrize("shape", [(32, 8, 128), (28, 4, 128), (5, 1, 64), (12, 4, 64)])
def test_rope_rows_and_heads(rows, shape):
    Rope(rows, shape[0], shape[1], shape[2], seed=rows, pad=rows % 5).run_and_check([shape[2] // 2])


@pytest.mark.parametrize("sections,cycled", [([16, 24, 24], False), ([24, 20, 20], True), ([0, 64, 0], False), ([22, 21, 21], True),
                                             ([16, 16, 16, 16], True), ([1, 2, 3, 4], False), ([40, 8, 0], True), ([5, 5], True)])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rope_axes(sections, cycled, adjacent):
    Rope(50, axes=len(sections), seed=sum(sections)).run_and_check(sections, adjacent, cycled)


@pytest.mark.parametrize("dim", [64, 128])
def test_rope_far_positions(dim):
    r = Rope(60, dim=dim, far=2 ** 31 - 1, seed=1)
    r.positions[0, :4] = torch.tensor([0, 1, 2 ** 31 - 1, 2 ** 24 + 1], dtype=torch.int32)
    # products of a 31-bit position and a 24-bit frequency fit 64 bits' 53: the reference's own angle is exact to 2^-53 of
    # itself, so up to 2^31 * 2^-53 = 2^-22 rad, which the slack of 2^-20 covers
    r.run_and_check([dim // 2])


def test_rope_negative_positions_turn_back():
    r = Rope(20, seed=2)
    r.positions.neg_()
    r.run_and_check([64])


@pytest.mark.parametrize("offset,tail", [(0, 64), (0, 4), (1, 0), (3, 5)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_strides_and_alignment(offset, tail, dtype):
    Rope(33, dtype=dtype, offset=offset, tail=tail, seed=3).run_and_check([64])


@pytest.mark.parametrize("pairs,adjacent", [(64, False), (64, True), (20, False)])
def test_rope_in_place(pairs, adjacent):
    Rope(70, pad=6, seed=4).run_and_check([pairs], adjacent, in_place=True)


def test_rope_of_q_or_k_alone():
    Rope(40, seed=5).run_and_check([64], with_kv=False)
    Rope(40, seed=6, pad=3).run_and_check([64], with_q=False)


def test_rope_without_slots_turns_every_row():
    r = Rope(40, seed=7)
    r.c.nsd_rope_append(r.pool, 0, r.q, None, None, r.q_out, r.positions, [64], gpu(np.ones(64, dtype=np.float32)))
    assert r.c.nsd_get_status() == (0, -1)
    y, slack = rope_ref(r.q.double().cpu().numpy().reshape(40, 8, 128), r.positions.cpu().numpy(), [64], np.ones(64), False, False)
    assert (np.abs(r.q_out.double().cpu().numpy() - y) <= HALF_BF16 * np.abs(y) + 1.01 * slack).all()


def test_rope_slot_beyond_the_pool_is_reported():
    r = Rope(40, seed=8)
    keep = r.pool.clone()
    r.slots[11] = r.num_blocks * BS
    r.c.nsd_rope_append(r.pool, 0, r.q, r.k, r.v, r.q_out, r.positions, [64], gpu(np.ones(64, dtype=np.float32)), r.slots)
    assert r.c.nsd_get_status() == (6, 11)
    assert (r.q_out != 3.0).any(-1).all()                          # its query is turned all the same
    assert torch.equal(r.pool[1], keep[1])


def test_rope_dims_that_do_not_turn_keep_infinities():
    r = Rope(10, seed=9)
    r.q[:, 100] = float("inf")
    r.q[:, 101] = float("nan")
    for adjacent in (False, True):
        r.c.nsd_rope_append(r.pool, 0, r.q, r.k, r.v, r.q_out, r.positions, [48], gpu(np.ones(48, dtype=np.float32)), r.slots, adjacent=adjacent)
        assert torch.isinf(r.q_out[:, 0, 100]).all() and torch.isnan(r.q_out[:, 0, 101]).all()
        assert torch.isfinite(r.q_out[:, 0, :100]).all() and torch.isfinite(r.q_out[:, 0, 102:]).all()


def test_rope_refusals():
    import paper_2609_29364_b200 as nsd

    r = Rope(10, axes=3, seed=10)
    f = gpu(np.ones(64, dtype=np.float32))
    args = lambda **k: {**dict(kv_pool=r.pool, layer=0, q=r.q, k=r.k, v=r.v, q_out=r.q_out, positions=r.positions, sections=[16, 24, 24],  # noqa: E731
                               inv_freq=f, slot_map=r.slots), **k}

    def refused(code, **k):
        with pytest.raises(nsd.NsdError) as e:
            r.c.nsd_rope_append(**args(**k))
        assert e.value.code == code

    refused(2, layer=2)
    refused(2, sections=[0, 0, 0])
    refused(2, sections=[-1, 24, 24])
    refused(1, sections=[4, 30, 30], cycled=True)                  # axis 1's 30th pair would be pair 88
    refused(1, slot_map=None)
    refused(4, q=r.q.half(), k=r.k.half(), v=r.v.half())
    with pytest.raises(ValueError):
        r.c.nsd_rope_append(**args(v=None))
    with pytest.raises(ValueError):
        r.c.nsd_rope_append(**args(sections=[32, 32]))
    with pytest.raises(ValueError):
        r.c.nsd_rope_append(**args(q=r.q[:, :-8]))
    with pytest.raises(TypeError):
        r.c.nsd_rope_append(**args(q_out=r.q_out.float()))
    big = gpu(np.ones(80, dtype=np.float32))
    refused(2, sections=[30, 25, 25], inv_freq=big)


# --------------------------------------------------------------------------- the step
def _step_buffers(batch, max_rows, entries, heads, dim, layers):
    z = lambda *s, dtype: torch.zeros(s, dtype=dtype, device=DEV)  # noqa: E731
    return dict(kv_indptr=z(batch + 1, dtype=torch.int64), kv_indices=z(entries, dtype=torch.int32), q_indptr=z(batch + 1, dtype=torch.int64),
                slot_map=z(max_rows, dtype=torch.int64), positions=z(max_rows, dtype=torch.int32), row_req=z(max_rows, dtype=torch.int32),
                n_held_new=z(batch, dtype=torch.int32), free_end=z(1, dtype=torch.int64))


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (12, 4, 64)])
def test_a_prompt_in_pieces_then_single_tokens(heads, kv_heads, dim):
    """Three requests over five steps -- pieces of prompts of odd lengths beside single tokens -- each step tables, plan,
    then append and attention per layer, captured once and replayed with the lengths and blocks of the next step.  Every
    step's attention is compared with the whole sequence computed at once in 64 bits."""
    layers, max_rows, stride, num_blocks, batch = 2, 160, 24, 80, 3
    steps = [[70, 0, 33], [50, 100, 1], [1, 20, 1], [0, 1, 1], [130, 1, 16]]
    total = [sum(s[r] for s in steps) for r in range(batch)]
    g = torch.Generator().manual_seed(11)
    c = context(heads, kv_heads, dim, num_blocks, max_batch=batch, num_layers=layers)
    width = (heads + 2 * kv_heads) * dim
    sequence = [torch.randn((layers, t, width), generator=g).to(torch.bfloat16) for t in total]
    pool = torch.full((layers, num_blocks, 2, kv_heads, BS, dim), float("nan"), dtype=torch.bfloat16, device=DEV)
    inv_freq = gpu((1e6 ** (-np.arange(dim // 2) / (dim // 2))).astype(np.float32))
    ctx_len, new_len = torch.zeros(batch, dtype=torch.int32, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
    held, n_held = torch.full((batch, stride), -1, dtype=torch.int32, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
    free, begin = torch.randperm(num_blocks, generator=g).to(torch.int32).to(DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    out = _step_buffers(batch, max_rows, batch * stride, heads, dim, layers)
    qkv = torch.zeros((layers, max_rows, width), dtype=torch.bfloat16, device=DEV)
    q_rot = torch.zeros((layers, max_rows, heads, dim), dtype=torch.bfloat16, device=DEV)
    o, lse = torch.zeros_like(q_rot), torch.zeros((layers, max_rows, heads), device=DEV)
    plan = torch.empty(c.nsd_chunk_plan_bytes(max_rows), dtype=torch.uint8, device=DEV)
    nq, nk = heads * dim, kv_heads * dim

    def step():
        c.nsd_block_tables(ctx_len, new_len, held, n_held, free, begin, **out)
        c.nsd_chunk_plan(plan, max_rows, out["q_indptr"], ctx_len, out["kv_indptr"])
        for l in range(layers):
            c.nsd_rope_append(pool, l, qkv[l, :, :nq], qkv[l, :, nq:nq + nk], qkv[l, :, nq + nk:], q_rot[l], out["positions"][None],
                              [dim // 2], inv_freq, out["slot_map"])
            c.nsd_chunk_attn(plan, max_rows, pool, q_rot[l], o[l], lse[l], out["kv_indices"], layer=l)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()                                                     # every request empty: nothing happens
    torch.cuda.synchronize()
    assert c.nsd_get_status() == (0, -1) and (o == 0).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    done = [0] * batch
    for new in steps:
        ctx_len.copy_(gpu(np.asarray(done, dtype=np.int32)))
        new_len.copy_(gpu(np.asarray(new, dtype=np.int32)))
        rows = sum(new)
        qkv.fill_(float("nan"))                                    # padding rows of the projection hold anything
        qkv[:, :rows] = torch.cat([sequence[r][:, done[r]:done[r] + new[r]] for r in range(batch)], 1).to(DEV)
        o.fill_(7.0)
        graph.replay()
        assert c.nsd_get_status() == (0, -1)
        n_held.copy_(out["n_held_new"])
        begin.copy_(out["free_end"])
        kvp, kvi = out["kv_indptr"].cpu().numpy(), out["kv_indices"].cpu().numpy()
        assert kvp.tolist() == offsets([blocks_of(d + n) for d, n in zip(done, new)]).tolist()
        assert out["q_indptr"].tolist() == offsets(new).tolist()
        for l in range(layers):
            ref_q, ref_pool = [], torch.zeros((num_blocks, 2, kv_heads, BS, dim), dtype=torch.float64)
            for r in range(batch):
                n = done[r] + new[r]
                x = sequence[r][l, :n].double().numpy().reshape(n, heads + 2 * kv_heads, dim)
                y, _ = rope_ref(x[:, :heads + kv_heads], np.arange(n)[None], [dim // 2], inv_freq.cpu().numpy(), False, False)
                y = torch.from_numpy(y).to(torch.bfloat16).double()
                ref_q.append(y[done[r]:, :heads])
                for t in range(n):
                    b = int(kvi[kvp[r] + t // BS])
                    ref_pool[b, 0, :, t % BS] = y[t, heads:]
                    ref_pool[b, 1, :, t % BS] = torch.from_numpy(x[t, heads + kv_heads:])
            # the kernel's q and k may round the other way where the exact value is next to a tie: attention is compared on
            # the values it was given, the rotation by itself
            got_pool = torch.nan_to_num(pool[l].double().cpu(), nan=0.0)
            assert (got_pool - ref_pool).abs().le(2 * HALF_BF16 * ref_pool.abs() + 2.0 ** -17).all()
            got_q = q_rot[l, :rows].double().cpu()
            want_q = torch.cat(ref_q, 0)
            assert (got_q - want_q).abs().le(2 * HALF_BF16 * want_q.abs() + 2.0 ** -17).all()
            check_attn(o[l, :rows], lse[l, :rows], attn_ref(got_q, got_pool, done, new, kvp, kvi))
            assert (o[l, rows:] == 7.0).all()
        done = [d + n for d, n in zip(done, new)]
