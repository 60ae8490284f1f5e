"""Attention over the 8-bit cache, against the 64-bit definition."""
import numpy as np
import pytest
import torch

from chunk_testlib import DEV, gpu
from kv8_testlib import Batch8

pytestmark = pytest.mark.gpu

SHAPES = [(8, 2, 128), (8, 2, 64), (4, 4, 128), (5, 1, 64), (28, 4, 128), (12, 4, 64), (32, 1, 128), (32, 8, 128), (24, 1, 64)]


def small(shape):
    return dict(heads=shape[0], kv_heads=shape[1], dim=shape[2])


@pytest.mark.parametrize("shape", SHAPES)
def test_lengths_around_every_edge(shape):
    Batch8([0, 0, 1, 15, 16, 17, 127, 128, 129, 255, 300, 0, 1000], [1, 0, 1, 1, 16, 3, 1, 1, 128, 33, 70, 200, 5], pad_rows=7, **small(shape)).run()


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 33])
def test_one_request_of_n_tokens(n):
    Batch8([130], [n], seed=n).run()


@pytest.mark.parametrize("shape", [(8, 2, 128), (8, 2, 64), (6, 6, 64)])
@pytest.mark.parametrize("ctx", [0, 5000, 20011])
def test_single_tokens_over_long_contexts(shape, ctx):
    Batch8([ctx, 3, ctx // 2], [1, 1, 1], seed=ctx, **small(shape)).run()


def test_a_verification_round():
    """Anchors with 0 to 4 drafted tokens, the shape and lengths of the smaller benchmark batches."""
    rng = np.random.default_rng(1)
    Batch8(rng.integers(50, 900, 40).tolist(), rng.integers(1, 6, 40).tolist(), heads=32, kv_heads=8, layers=2, seed=1).run()


def test_many_requests_of_one_token():
    rng = np.random.default_rng(5)
    Batch8(rng.integers(0, 700, 150).tolist(), [1] * 150, heads=4, kv_heads=2, dim=64, seed=5).run()


def test_a_prompt_and_a_chunk():
    Batch8([0, 2001], [500, 301], seed=4).run()


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 1000, 100000])
@pytest.mark.parametrize("dim", [64, 128])
def test_window(window, dim):
    Batch8([0, 700, 129, 2000], [60, 45, 1, 5], dim=dim, seed=window).run(window=window)


def test_prefix_sees_itself_both_ways():
    Batch8([0, 100, 40, 0], [60, 40, 1, 29], seed=7).run(prefix_len=[37, 120, 41, 100000])


@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64)])
def test_documents_and_rows_that_see_nothing(shape):
    ctx, new = [0, 300, 5], [100, 50, 1]
    rng = np.random.default_rng(8)
    first = [10 ** 6 if i % 7 == 0 else int(rng.integers(0, 60)) for i in range(151)]
    Batch8(ctx, new, seed=8, **small(shape)).run(row_first=first)


def test_every_row_sees_nothing():
    b = Batch8([100, 3], [5, 1], seed=9).run(row_first=[10 ** 6] * 6)
    assert (b.o[0, :6] == 0).all() and torch.isinf(b.lse[0, :6]).all()


def test_scale_and_row_stride():
    Batch8([200, 0], [7, 30], q_stride=8 * 128 + 64, seed=14).run(scale=0.02)


@pytest.mark.parametrize("dim", [64, 128])
def test_the_running_maximum_moves_late_and_often(dim):
    """Keys that grow along the context, and ones that grow towards its start, up to scores in the hundreds; also single
    keys that stand out by far, late and early."""
    tokens = 1505
    rng = np.random.default_rng(15)
    base = rng.standard_normal((tokens, 2, dim))
    ramp = np.linspace(0.05, 8.0, tokens)[:, None, None]
    spikes = np.ones((tokens, 1, 1))
    spikes[[3, 200, 700, 1100, 1499]] = 30.0
    for factor in (ramp, ramp[::-1], spikes):
        b = Batch8([1500], [5], dim=dim, seed=15)
        b.set_rows(0, 0, base * factor)
        b.run()


@pytest.mark.parametrize("dim", [64, 128])
def test_values_of_unlike_size(dim):
    """Rows of V whose powers of two rise, fall and jump along the context, over sixty binades; keys likewise small."""
    tokens = 1203
    rng = np.random.default_rng(16)
    base = rng.standard_normal((tokens, 2, dim))
    for steps in (np.linspace(-30, 30, tokens), np.linspace(30, -30, tokens), rng.integers(-30, 31, tokens)):
        b = Batch8([1200], [3], dim=dim, seed=16)
        b.set_rows(0, 1, base * np.exp2(np.round(steps))[:, None, None])
        b.run()


def test_one_large_weight_before_many_small_ones():
    """A key that holds most of a row's weight, before thousands whose weights are 2^-13 of it each but together as much:
    they are not lost in the rounding of the weights."""
    tokens, dim = 8001, 128
    b = Batch8([8000], [1], heads=2, kv_heads=1, seed=17)
    k = np.zeros((tokens, 1, dim))
    q = torch.zeros((1, 1, 256), dtype=torch.bfloat16)
    q[..., 0], q[..., 128] = 1.0, 1.0
    k[0, 0, 0] = 13.0 * np.log(2.0) * np.sqrt(dim) // 1
    b.q.copy_(q)
    b.set_rows(0, 0, k)
    v = np.full((tokens, 1, dim), 1.0)
    v[0] = -1.0
    b.set_rows(0, 1, v)
    b.run()


def test_q_rows_of_unlike_size():
    """Heads whose queries differ by many binades, and rows with an element that stands out."""
    b = Batch8([300, 40], [5, 1], heads=16, kv_heads=2, seed=18)
    s = torch.exp2(torch.linspace(-20, 4, 16)).repeat_interleave(128).to(DEV)
    b.q.mul_(s.to(torch.bfloat16))
    b.q[..., 5] *= 64.0
    b.run()


def test_extreme_scales_and_queries():
    """Keys near the format's least and largest rows against queries that bring the scores back to order one."""
    for e, f in ((2.0 ** -100, 2.0 ** 100), (2.0 ** 100, 2.0 ** -100), (2.0 ** -126, 2.0 ** 60)):
        b = Batch8([140], [3], heads=2, kv_heads=1, seed=19)
        b.set_rows(0, 0, np.random.default_rng(19).standard_normal((143, 1, 128)) * e)
        b.q.mul_(f)
        b.run()


def test_equal_scores_give_the_mean():
    b = Batch8([100], [30], seed=16)
    b.q_all.zero_()
    b.run()


def test_what_is_not_a_number_stays_with_the_rows_that_see_it():
    b = Batch8([100, 50, 60, 70], [3, 1, 2, 1], seed=20)
    nan = float("nan")
    b.q[0, 1, 128 * 3 + 5] = nan                                        # row 1 of request 0, head 3
    b.q[0, 3, 128 * 2] = float("inf")                                   # request 1, head 2
    kv = b.kvi.tolist()
    b.kv8[0, kv[int(b.kv_indptr[2]) + 1], 0, 1, 4, 77] = 0x7F           # a key of request 2, kv head 1
    b.scales[0, kv[int(b.kv_indptr[3])], 0, 1, 9] = 255                 # a scale of V of request 3, kv head 0
    b.values[0, kv[int(b.kv_indptr[3])], 1, 0, 9] = 0.0
    c = b.context()
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (0, -1)
    bad = torch.zeros((7, 8), dtype=torch.bool, device=DEV)
    bad[1, 3] = bad[3, 2] = True
    bad[4:6, 4:] = True
    bad[6, :4] = True
    assert torch.equal(torch.isnan(b.lse[0, :7]), bad)
    assert torch.equal(torch.isnan(b.o[0, :7]).all(-1), bad) and torch.equal(torch.isnan(b.o[0, :7]).any(-1), bad)
    b.q.copy_(torch.nan_to_num(b.q, nan=0.0, posinf=0.0))
    o_ref, lse_ref, mag = b.reference()
    good = ~bad.cpu()
    assert ((b.o[0, :7].double().cpu() - o_ref.cpu()).abs() <= 2.0 ** -8 * o_ref.cpu().abs() + 2.0 ** -9 * mag.cpu() + 1e-3)[good].all()


@pytest.mark.parametrize("tokens", [1, 3, 6, 9])
@pytest.mark.parametrize("dim", [64, 128])
def test_queries_that_are_no_numbers_leave_the_other_rows(dim, tokens):
    """Rows with a NaN or an infinity among up to 36 stacked ones, beside rows of every size: these are right to the same limit
    as without them (the limit of check_attn8, whose first two terms are below 2^-8 |o| + 2^-9 of the weighted |v|)."""
    b = Batch8([100, 300], [tokens, tokens], heads=8, kv_heads=2, dim=dim, seed=30 + tokens)
    b.q *= torch.exp2(torch.arange(-6, 2, device=DEV).float())[None, None, :].repeat_interleave(dim, -1).to(torch.bfloat16)
    bad = torch.zeros((2 * tokens, 8), dtype=torch.bool, device=DEV)
    for i, x in enumerate((float("nan"), float("inf"), float("-inf"))):
        row, head, at = (i * 5 + 1) % (2 * tokens), (3 * i + 2) % 8, (i * 37 + dim - 1) % dim
        b.q[0, row, head * dim + at] = x
        bad[row, head] = True
    b.q[0, tokens, 7 * dim:] = float("nan")                             # a whole row
    bad[tokens, 7] = True
    c = b.context()
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (0, -1)
    assert torch.equal(torch.isnan(b.lse[0, :2 * tokens]), bad)
    assert torch.equal(torch.isnan(b.o[0, :2 * tokens]).all(-1), bad) and torch.equal(torch.isnan(b.o[0, :2 * tokens]).any(-1), bad)
    b.q.copy_(torch.nan_to_num(b.q, nan=0.0, posinf=0.0, neginf=0.0))
    o_ref, lse_ref, mag = (t.cpu() for t in b.reference())
    good = ~bad.cpu()
    limit = 2.0 ** -8 * o_ref.abs() + 2.0 ** -9 * mag + 2.0 ** -24 * (300 + tokens) * float(b.values[0, :, 1].abs().max())
    assert ((b.o[0, :2 * tokens].double().cpu() - o_ref).abs() <= limit)[good].all()
    assert ((b.lse[0, :2 * tokens].double().cpu() - lse_ref).abs() <= 2.0 ** -10 + 2.0 ** -20 * lse_ref.abs())[good].all()


def test_bad_blocks_and_short_tables_are_reported():
    b = Batch8([100, 50], [1, 1], seed=21)
    c = b.context()
    plan = b.plan(c)
    b.kvi[2] = b.num_blocks
    b.attn(c, plan)
    assert c.nsd_get_status() == (6, 0)
    assert torch.isfinite(b.o[0]).all()
    b.kvi[2] = -1
    b.attn(c, plan)
    assert c.nsd_get_status() == (6, 0)
    short = b.kvp.clone()
    short[2] -= 1
    b2 = Batch8([100, 50], [1, 1], seed=21)
    b2.kvp = short
    b2.attn(c, b2.plan(c))
    assert c.nsd_get_status() == (6, 1)


def test_a_plan_of_the_other_kind_is_refused_on_the_device():
    b = Batch8([100], [2], seed=22)
    c = b.context()
    plan = torch.empty(max(c.nsd_chunk_plan_bytes(2), c.nsd_kv8_plan_bytes(2)), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, 2, b.qp, b.ctx_len, b.kvp)
    b.attn(c, plan)
    assert c.nsd_get_status()[0] == 6 and (b.o == 7.0).all() and (b.lse == 7.0).all()
    plan.zero_()
    b.attn(c, plan)
    assert c.nsd_get_status()[0] == 6 and (b.o == 7.0).all()


def test_bad_lengths_leave_an_empty_plan():
    b = Batch8([100, 20], [2, 1], seed=23)
    c = b.context()
    b.ctx_len[1] = -1
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (6, 1) and (b.o == 7.0).all()


def test_captured_and_replayed_with_other_lengths():
    """One graph of plan and attention serves any lengths that its buffers hold."""
    from kv8_testlib import T

    big = Batch8([900, 700, 300], [5, 5, 5], seed=24, pad_rows=4)
    c = big.context()
    plan = big.plan(c)
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            c.nsd_kv8_plan(plan, big.max_rows, big.qp, big.ctx_len, big.kvp, stream=s)
            c.nsd_kv8_attn(plan, big.max_rows, big.kv8, big.scales, big.q[0], big.o[0], big.lse[0], big.kvi, stream=s)
    for ctx, new in (([900, 700, 300], [5, 5, 5]), ([17, 0, 300], [1, 5, 0]), ([128, 400, 1], [5, 2, 1])):
        big.ctx, big.new = ctx, new
        big.ctx_len.copy_(gpu(np.asarray(ctx, dtype=np.int32)))
        big.qp.copy_(gpu(T.offsets(new)))
        big.rows = int(sum(new))
        big.o.fill_(7.0), big.lse.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert c.nsd_get_status() == (0, -1)
        big.check()
    del graph


def test_same_bits_every_time():
    b = Batch8([30000, 500], [3, 1], seed=25)
    c = b.context()
    plan = b.plan(c)
    b.attn(c, plan)
    o, lse = b.o.clone(), b.lse.clone()
    for _ in range(3):
        b.o.zero_(), b.lse.zero_()
        b.attn(c, plan)
        assert torch.equal(o, b.o) and torch.equal(lse, b.lse)


def test_without_lse_and_on_another_stream():
    b = Batch8([300, 20], [2, 1], seed=26)
    c = b.context()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        plan = b.plan(c)
        c.nsd_kv8_attn(plan, b.max_rows, b.kv8, b.scales, b.q[0], b.o[0], None, b.kvi)
    s.synchronize()
    assert (b.lse == 7.0).all()
    b.attn(c, plan)
    o = b.o.clone()
    torch.cuda.synchronize()
    assert torch.equal(o, b.o)
    b.check()


def test_append_plan_attend_together():
    """A decoding run: rows appended to the 8-bit cache step by step, attention over it each time, and the same tokens
    packed from a 16-bit pool give the same outputs."""
    from kv8_testlib import K8Run

    K8Run().check()


def test_refusals_launch_nothing():
    import paper_2609_29364_b200 as nsd

    b = Batch8([100], [2], seed=30)
    c = b.context()
    plan = b.plan(c)
    before = c.nsd_launch_count()

    def code(call):
        with pytest.raises(nsd.NsdError) as e:
            call()
        return e.value.code

    args = dict(plan=plan, max_rows=2, kv8=b.kv8, scales=b.scales, q=b.q[0], o=b.o[0], lse=b.lse[0], kv_indices=b.kvi)
    assert code(lambda: c.nsd_kv8_attn(**args, layer=1)) == 2
    assert code(lambda: c.nsd_kv8_attn(**args, layer=-1)) == 2
    assert code(lambda: c.nsd_kv8_attn(**args, scale=float("nan"))) == 1
    assert code(lambda: c.nsd_kv8_attn(**args, scale=-1.0)) == 1
    assert code(lambda: c.nsd_kv8_attn(**{**args, "plan": plan[:-256]})) == 3
    assert code(lambda: c.nsd_kv8_attn(**{**args, "plan": plan[16:]})) == 1
    assert code(lambda: c.nsd_kv8_attn(**{**args, "kv8": b.kv8.data_ptr() + 8})) == 1
    wide = torch.zeros((2, 8 * 128 + 4), dtype=torch.bfloat16, device=DEV)
    assert code(lambda: c.nsd_kv8_attn(**{**args, "q": wide[:, :1024]})) == 1
    assert code(lambda: c.nsd_kv8_plan(plan[:256], 2, b.qp, b.ctx_len, b.kvp)) == 3
    assert code(lambda: c.nsd_kv8_plan(plan, 2, b.qp, b.ctx_len, b.kvp, window=-1)) == 1
    many = torch.zeros(5, dtype=torch.int64, device=DEV)
    assert code(lambda: c.nsd_kv8_plan(plan, 2, many, torch.zeros(2, dtype=torch.int32, device=DEV), many)) == 2
    assert c.nsd_launch_count() == before and (b.o == 7.0).all()


def test_an_empty_batch_and_requests_without_rows():
    b = Batch8([100, 20], [0, 0], seed=31, pad_rows=3).run()
    assert (b.o == 7.0).all()


def test_blocks_shared_by_requests_and_named_twice():
    b = Batch8([64, 64, 100], [1, 2, 3], seed=32)
    t = b.kv_indices
    a0, a1, a2 = (int(x) for x in b.kv_indptr[:3])
    t[a1:a1 + 4] = t[a0:a0 + 4]                                          # four full blocks in common
    t[a2 + 2] = t[a2 + 1]                                                # and one twice in a row
    b.kvi = gpu(t)
    b.run()


def test_blocks_before_the_window_may_be_gone():
    b = Batch8([700, 300], [5, 1], seed=33)
    for r, c in ((0, 700), (1, 300)):
        at, gone = int(b.kv_indptr[r]), (c + 1 - 100) // 16
        b.kv_indices[at:at + gone] = -1
    b.kvi = gpu(b.kv_indices)
    b.run(window=100)


def test_offsets_beyond_32_bits():
    """Blocks whose codes lie more than 2^32 bytes into the cache."""
    small = Batch8([300], [2], heads=8, kv_heads=8, dim=128, seed=34)
    blocks = 140000
    big = torch.zeros((1, blocks, 2, 8, 16, 128), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((1, blocks, 8, 2, 16), dtype=torch.uint8, device=DEV)
    shift = blocks - small.num_blocks
    big[0, shift:], scales[0, shift:] = small.kv8[0], small.scales[0]
    from kv8_testlib import T

    c = T.context(8, 8, 128, blocks, max_batch=1)
    plan = small.plan(c)
    c.nsd_kv8_attn(plan, small.max_rows, big, scales, small.q[0], small.o[0], small.lse[0], small.kvi + shift)
    assert c.nsd_get_status() == (0, -1)
    small.check()


def test_waits_that_run_out_end_the_call_and_nothing_else():
    """With one poll per wait, calls give up wherever a copy or a product is not there at once: they end, say so or are right,
    and the next context works on the same memory."""
    b = Batch8([3000, 200, 17], [5, 1, 2], seed=35)
    c = b.context(wait_budget=1)
    gave_up = 0
    for _ in range(5):
        b.attn(c, b.plan(c))
        rc, _ = c.nsd_get_status()
        assert rc in (0, 8)
        gave_up += rc == 8
        if rc == 0:
            b.check()
    assert gave_up > 0
    b.o.fill_(7.0), b.lse.fill_(7.0)
    b.run()


def test_two_plans_at_once_on_two_streams():
    a, b = Batch8([5000, 30], [3, 1], seed=36), Batch8([200, 4000], [1, 4], seed=37)
    ca, cb = a.context(), b.context()
    pa, pb = a.plan(ca), b.plan(cb)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.attn(ca, pa, stream=s)
        b.attn(cb, pb, stream=t)
    torch.cuda.synchronize()
    assert ca.nsd_get_status() == (0, -1) and cb.nsd_get_status() == (0, -1)
    a.check(), b.check()


def test_random_batches():
    rng = np.random.default_rng(38)
    for i in range(12):
        n = int(rng.integers(1, 30))
        heads, hkv, dim = SHAPES[int(rng.integers(0, len(SHAPES)))]
        ctx = np.where(rng.random(n) < 0.5, rng.integers(0, 60, n), rng.integers(0, 3000, n)).tolist()
        new = np.where(rng.random(n) < 0.8, rng.integers(0, 6, n), rng.integers(0, 40, n)).tolist()
        Batch8(ctx, new, heads=heads, kv_heads=hkv, dim=dim, seed=100 + i, pad_rows=2).run(**({"window": int(rng.integers(1, 500))} if i % 3 == 0 else {}))
