"""Attention of a chunk of new tokens over the paged pool, against the 64-bit definition."""
import numpy as np
import pytest
import torch

from chunk_testlib import DEV, Batch, blocks_of, check_attn, gpu, offsets

pytestmark = pytest.mark.gpu

SHAPES = [(8, 2, 128), (8, 2, 64), (4, 4, 128), (5, 1, 64), (28, 4, 128), (12, 4, 64), (32, 1, 128), (32, 8, 128)]


def small(shape):
    return dict(heads=shape[0], kv_heads=shape[1], dim=shape[2])


@pytest.mark.parametrize("shape", SHAPES)
def test_lengths_around_every_edge(shape):
    """Chunks of 0, 1 and many tokens over contexts of 0 and around the edges of blocks and key tiles, in one batch."""
    Batch([0, 0, 1, 15, 16, 17, 127, 128, 129, 255, 300, 0, 1000], [1, 0, 1, 1, 16, 3, 1, 1, 128, 33, 70, 200, 5], pad_rows=7, **small(shape)).run()


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 257])
def test_one_request_of_n_tokens(n):
    Batch([130], [n], seed=n).run()


@pytest.mark.parametrize("shape", [(8, 2, 128), (8, 2, 64)])
@pytest.mark.parametrize("ctx", [0, 5000, 20011])
def test_single_tokens_over_long_contexts(shape, ctx):
    Batch([ctx, 3, ctx // 2], [1, 1, 1], seed=ctx, **small(shape)).run()


def test_a_prompt_from_nothing():
    Batch([0], [1500], seed=3).run()


def test_a_chunk_over_a_long_context():
    Batch([9001], [301], seed=4).run()


def test_many_requests_of_one_token():
    rng = np.random.default_rng(5)
    Batch(rng.integers(0, 700, 150).tolist(), [1] * 150, heads=4, kv_heads=2, dim=64, seed=5).run()


def test_layers_share_a_plan():
    Batch([100, 0, 513], [40, 200, 1], layers=3, seed=6).run()


@pytest.mark.parametrize("window", [1, 2, 16, 100, 128, 1000, 100000])
def test_window(window):
    Batch([0, 700, 129], [300, 45, 1], seed=window).run(window=window)


@pytest.mark.parametrize("dim", [64, 128])
def test_prefix_sees_itself_both_ways(dim):
    Batch([0, 100, 40, 0], [300, 200, 1, 129], dim=dim, seed=7).run(prefix_len=[170, 50, 41, 100000])


def _docs(ctx, new, seed, empty=False):
    rng = np.random.default_rng(seed)
    out = []
    for c, n in zip(ctx, new):
        start = 0
        for i in range(n):
            if rng.random() < 0.02:
                start = c + i
            out.append(start)
    if empty:
        for i in range(0, len(out), 7):
            out[i] = 10 ** 6                       # such a row sees nothing
    return out


@pytest.mark.parametrize("empty", [False, True])
@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64)])
def test_documents_and_rows_that_see_nothing(shape, empty):
    ctx, new = [0, 300, 5], [400, 150, 1]
    Batch(ctx, new, seed=8, **small(shape)).run(row_first=_docs(ctx, new, 8, empty))


def test_every_row_sees_nothing():
    b = Batch([100, 3], [50, 1], seed=9).run(row_first=[10 ** 6] * 51)
    assert (b.o[0, :51] == 0).all() and torch.isinf(b.lse[0, :51]).all()


@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64), (5, 1, 64)])
@pytest.mark.parametrize("softcap,q_scale", [(30.0, 1.0), (30.0, 8.0), (5.0, 3.0), (0.5, 2.0), (1000.0, 1.0)])
def test_capped_scores(shape, softcap, q_scale):
    Batch([200, 0, 1000], [70, 300, 1], q_scale=q_scale, seed=10, **small(shape)).run(softcap=softcap)


def _slopes(heads):
    return [2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)]


@pytest.mark.parametrize("shape", [(8, 2, 128), (12, 4, 64), (5, 1, 64)])
def test_bias_on_distance(shape):
    Batch([200, 0, 3000], [70, 300, 1], seed=11, **small(shape)).run(slopes=_slopes(shape[0]))


def test_bias_of_either_sign_and_none():
    Batch([200, 0, 2000], [70, 300, 1], seed=12).run(slopes=[1.0, -0.25, 0.0, 0.01, -0.001, 2.0, 0.5, -1.0])


def test_everything_at_once():
    ctx, new = [0, 300, 2000, 17], [400, 150, 1, 90]
    Batch(ctx, new, q_scale=4.0, seed=13).run(slopes=_slopes(8), softcap=20.0, window=130, prefix_len=[100, 400, 7, 60],
                                              row_first=_docs(ctx, new, 13, True))


def test_scale():
    Batch([200, 0], [70, 30], seed=14).run(scale=0.02)


def test_the_running_maximum_moves_late_and_often():
    """Keys that grow along the context, and ones that grow towards its start: the reference point of the sums moves in
    most tiles, up to scores in the hundreds."""
    for grow in (1, -1):
        b = Batch([2000, 10], [150, 1], seed=15)
        ramp = torch.linspace(0.05, 8.0, 2150)
        ramp = ramp if grow > 0 else ramp.flip(0)
        for t in range(2150):
            b.pool[0, int(b.kv_indices[t // 16]), 0, :, t % 16] *= float(ramp[t])
        b.run()


def test_equal_scores_give_the_mean():
    b = Batch([100], [30], seed=16)
    b.q_all.zero_()
    b.run()


def test_row_stride_of_q():
    Batch([100, 7], [30, 100], q_stride=8 * 128 + 2 * 2 * 128, seed=17).run()


def test_blocks_before_the_window_may_be_gone():
    """Table entries no row can see may be -1 or repeat a block that holds NaN."""
    b = Batch([1000, 600], [40, 1], seed=18)
    for r, keep in ((0, (1001 - 100) // 16), (1, (601 - 100) // 16)):
        lo = int(b.kv_indptr[r])
        for j in range(keep):
            b.pool[0, int(b.kv_indices[lo + j])] = float("nan")
        b.kvi[lo:lo + keep] = -1
    b.run(window=100)


def test_bad_block_ids_are_reported_and_read_as_zeros():
    b = Batch([100, 200], [30, 1], seed=19)
    c = b.context()
    plan = b.plan(c)
    bad = int(b.kv_indptr[1]) + 3
    for entry in (-1, b.num_blocks, 2 ** 30):
        b.kvi[bad] = entry
        b.attn(c, plan)
        rc, who = c.nsd_get_status()
        assert (rc, who) == (6, 1)
    pool = b.pool.clone()
    b.pool[0, int(b.kv_indices[bad])] = 0
    b.check()
    b.pool.copy_(pool)


def test_a_short_table_is_reported():
    b = Batch([100, 200], [30, 1], seed=20)
    c = b.context()
    b.kvp[2] -= 2                                  # the second request's table ends early
    plan = b.plan(c)
    b.attn(c, plan)
    assert c.nsd_get_status() == (6, 1)


@pytest.mark.parametrize("what", ["rows beyond", "rows decrease", "negative context", "tables decrease", "first row"])
def test_malformed_lengths_leave_an_empty_plan(what):
    b = Batch([100, 200, 5], [30, 1, 4], seed=21)
    c = b.context()
    if what == "rows beyond":
        b.qp[3] = b.max_rows + 1
    elif what == "rows decrease":
        b.qp[2] = 10
    elif what == "negative context":
        b.ctx_len[1] = -1
    elif what == "tables decrease":
        b.kvp[1] = b.kvp[3] + 5
    else:
        b.qp[0] = 3
    plan = b.plan(c)
    b.attn(c, plan)
    assert c.nsd_get_status()[0] == 6
    assert (b.o == 7.0).all() and (b.lse == 7.0).all()


def test_a_buffer_without_a_plan_is_reported():
    b = Batch([100], [30], seed=22)
    c = b.context()
    plan = torch.zeros(c.nsd_chunk_plan_bytes(b.max_rows), dtype=torch.uint8, device=DEV)
    b.attn(c, plan)
    assert c.nsd_get_status()[0] == 6
    assert (b.o == 7.0).all()


def test_empty_batches():
    b = Batch([100, 7], [0, 0], pad_rows=3, seed=23)
    b.masks = {}
    c = b.context()
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (0, -1)
    assert (b.o == 7.0).all()
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    plan = torch.empty(c.nsd_chunk_plan_bytes(3), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, 3, torch.zeros(1, dtype=torch.int64, device=DEV), none, torch.zeros(1, dtype=torch.int64, device=DEV))
    c.nsd_chunk_attn(plan, 3, b.pool, b.q[0], b.o[0], None, b.kvi)
    assert c.nsd_get_status() == (0, -1)
    assert (b.o == 7.0).all()


def test_repeated_calls_give_the_same_bits():
    b = Batch([3000, 0, 77, 9000], [1, 300, 40, 3], seed=24)
    c = b.context()
    plan = b.plan(c)
    b.attn(c, plan)
    first = (b.o.clone(), b.lse.clone())
    for _ in range(3):
        b.o.fill_(7.0)
        b.attn(c, plan)
        assert torch.equal(b.o, first[0]) and torch.equal(b.lse, first[1])


def test_two_plans_on_two_streams():
    a, b = Batch([3000, 5], [1, 200], seed=25), Batch([9000], [1], seed=26)
    ca, cb = a.context(), b.context()
    pa, pb = a.plan(ca), b.plan(cb)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        a.attn(ca, pa, stream=sa)
        b.attn(cb, pb, stream=sb)
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_one_context_two_plans_two_streams():
    a = Batch([3000, 5], [1, 200], seed=27)
    c = a.context()
    pa, pb = a.plan(c), a.plan(c)
    o2, lse2 = a.o.clone(), a.lse.clone()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        a.attn(c, pa, stream=sa)
        c.nsd_chunk_attn(pb, a.max_rows, a.pool, a.q[0], o2[0], lse2[0], a.kvi, stream=sb)
    torch.cuda.synchronize()
    a.check()
    assert torch.equal(a.o, o2) and torch.equal(a.lse, lse2)


def test_agrees_with_the_verification_attention():
    """The rows of a verification round are a chunk of gamma + 1 tokens: the two entry points agree within the roundings
    of both."""
    b = Batch([100, 37, 900], [2, 2, 2], seed=28)
    c = b.context()
    b.attn(c, b.plan(c))
    o2, lse2 = torch.empty_like(b.o[0]), torch.empty_like(b.lse[0])
    c.nsd_verify_plan(np.asarray(b.ctx, dtype=np.int32), b.kv_indptr, None, 1)
    c.nsd_verify_attn(b.pool, b.q[0].contiguous(), o2, lse2, 3, 1, b.ctx_len, b.kvp, b.kvi)
    assert c.nsd_get_status() == (0, -1)
    b.check()
    check_attn(o2, lse2, b.reference())


def test_captured_call_serves_other_lengths():
    """Plan and attention in one graph; the replay sees new lengths written into the same buffers."""
    b = Batch([500, 40, 0], [60, 1, 130], pad_rows=50, seed=29)
    c = b.context()
    plan = torch.empty(c.nsd_chunk_plan_bytes(b.max_rows), dtype=torch.uint8, device=DEV)

    def step():
        c.nsd_chunk_plan(plan, b.max_rows, b.qp, b.ctx_len, b.kvp)
        b.attn(c, plan)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    b.masks = {}
    for ctx, new in (([500, 40, 0], [60, 1, 130]), ([520, 3, 100], [1, 38, 5]), ([0, 41, 129], [100, 0, 1])):
        b.ctx, b.new = ctx, new
        b.ctx_len.copy_(gpu(np.asarray(ctx, dtype=np.int32)))
        b.q_indptr = offsets(new)
        b.rows = int(b.q_indptr[-1])
        b.qp.copy_(gpu(b.q_indptr))
        b.o.fill_(7.0)
        b.lse.fill_(7.0)
        # every key of these lengths has to hold a token
        b.pool.nan_to_num_(nan=0.25)
        graph.replay()
        assert c.nsd_get_status() == (0, -1)
        b.check()
        assert all(blocks_of(x + y) <= int(b.kv_indptr[r + 1] - b.kv_indptr[r]) for r, (x, y) in enumerate(zip(ctx, new)))


def test_refusals():
    import paper_2609_29364_b200 as nsd

    b = Batch([100], [30], seed=30)
    c = b.context()
    plan = b.plan(c)

    def refused(code, f, *a, **k):
        with pytest.raises(nsd.NsdError) as e:
            f(*a, **k)
        assert e.value.code == code

    refused(1, b.attn, c, plan, scale=-1.0)
    refused(1, b.attn, c, plan, scale=float("nan"))
    refused(1, b.attn, c, plan, softcap=-1.0)
    refused(1, b.attn, c, plan, softcap=float("inf"))
    for layer in (1, -1):
        refused(2, c.nsd_chunk_attn, plan, 30, b.pool, b.q[0], b.o[0], None, b.kvi, layer=layer)
    refused(3, b.attn, c, plan[:-256])
    refused(1, b.attn, c, plan[8:])
    refused(1, c.nsd_chunk_plan, plan, b.max_rows, b.qp, b.ctx_len, b.kvp, window=-1)
    refused(3, c.nsd_chunk_plan, plan, b.max_rows + 100000, b.qp, b.ctx_len, b.kvp)
    refused(2, c.nsd_chunk_plan, plan, b.max_rows, torch.zeros(3, dtype=torch.int64, device=DEV),
            torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV))
    odd = torch.zeros((30, 8 * 128 + 4), dtype=torch.bfloat16, device=DEV)
    refused(1, c.nsd_chunk_attn, plan, 30, b.pool, odd[:, :1024], b.o[0], None, b.kvi)          # row stride not a multiple of 8
    off = torch.zeros(30 * 1024 + 8, dtype=torch.bfloat16, device=DEV)[1:30 * 1024 + 1].view(30, 1024)
    refused(1, c.nsd_chunk_attn, plan, 30, b.pool, off, b.o[0], None, b.kvi)                    # q not on 16 bytes
    with pytest.raises(TypeError):
        c.nsd_chunk_attn(plan, 30, b.pool, b.q[0].float(), b.o[0], None, b.kvi)
    with pytest.raises(ValueError):
        c.nsd_chunk_attn(plan, 30, b.pool, b.q[0], b.o[0], b.lse[0, :3], b.kvi)
    assert c.nsd_chunk_plan_bytes(-1) == 0
    assert (b.o == 7.0).all()


@pytest.mark.parametrize("softcap", [1e-30, 1e-7, 2e30, 3e38, float("nan")])
def test_caps_beyond_32_bits_are_refused(softcap):
    import paper_2609_29364_b200 as nsd

    b = Batch([100], [30], seed=30)
    c = b.context()
    plan = b.plan(c)
    with pytest.raises(nsd.NsdError) as e:
        b.attn(c, plan, softcap=softcap)
    assert e.value.code == 1
    with pytest.raises(nsd.NsdError) as e:
        b.attn(c, plan, scale=2e30)
    assert e.value.code == 1
    assert (b.o == 7.0).all()


@pytest.mark.parametrize("shape", [(32, 8, 128), (12, 4, 64)])
def test_the_smallest_and_largest_caps(shape):
    """A cap far above every score changes none of them; one far below makes all weights equal to within it."""
    Batch([700, 0], [40, 300], seed=32, **small(shape)).run(softcap=1e30)
    Batch([700, 0], [40, 300], seed=32, **small(shape)).run(softcap=1e-6)


@pytest.mark.parametrize("shape", [(32, 8, 128), (12, 4, 64)])
def test_requests_that_share_blocks_and_a_block_twice_in_a_table(shape):
    """A common prefix is stored once, and nothing forbids a table that names a block again: only reads meet."""
    b = Batch([640, 640, 320], [1, 33, 1], seed=34, **small(shape))
    first, second, third = (int(b.kv_indptr[r]) for r in range(3))
    b.kv_indices[second:second + 20] = b.kv_indices[first:first + 20]
    b.kv_indices[third + 7] = b.kv_indices[third + 3]
    b.kvi.copy_(torch.from_numpy(b.kv_indices))
    b.run()


def test_a_plan_of_another_shape_is_reported():
    b = Batch([100, 30], [30, 1], heads=8, kv_heads=2, seed=31)
    c, other = b.context(), Batch([100, 30], [30, 1], heads=8, kv_heads=4, seed=31).context()
    plan = torch.empty(max(c.nsd_chunk_plan_bytes(31), other.nsd_chunk_plan_bytes(31)), dtype=torch.uint8, device=DEV)
    other.nsd_chunk_plan(plan, 31, b.qp, b.ctx_len, b.kvp)
    b.attn(c, plan)
    assert c.nsd_get_status()[0] == 6 and (b.o == 7.0).all()


@pytest.mark.parametrize("shape", [(32, 8, 128), (12, 4, 64)])
@pytest.mark.parametrize("softcap", [0.0, 25.0])
def test_short_units_of_two_row_tiles_among_single_tokens(shape, softcap):
    """Many pieces per CTA, of one to three key tiles, that change between one and two row tiles: a Q buffer is filled anew right
    behind its last use, while the two streams' progress differs.  Repeated, since what can go wrong here is a matter of timing."""
    tokens = 128 // (shape[0] // shape[1])
    rng = np.random.default_rng(7)
    n = 400
    ctx = rng.integers(0, 300, n)
    new = np.where(rng.random(n) < 0.5, 1, rng.integers(tokens + 1, 2 * tokens + 1, n))
    batch = Batch(ctx.tolist(), new.tolist(), seed=1, **small(shape))
    c = batch.context()
    plan = batch.plan(c)
    for _ in range(50):
        batch.attn(c, plan, softcap=softcap)
    status = c.nsd_get_status()
    assert status == (0, -1), status
    batch.check(softcap=softcap)


@pytest.mark.parametrize("shape", [(32, 8, 128), (12, 4, 64)])
@pytest.mark.parametrize("seed", range(4))
def test_random_batches(shape, seed):
    """Single tokens, short and long chunks of any length beside one another: every way a CTA's share can begin, end and
    change between units of one and two row tiles, with odd and even numbers of key tiles."""
    rng = np.random.default_rng(100 + seed)
    n = 24
    ctx = np.where(rng.random(n) < 0.3, rng.integers(0, 40, n), rng.integers(0, 4000, n))
    new = np.where(rng.random(n) < 0.6, 1, rng.integers(0, 400, n))
    masks = [{}, dict(window=700), dict(prefix_len=rng.integers(0, 500, n).tolist()), {}][seed]
    Batch(ctx.tolist(), new.tolist(), seed=seed, **small(shape)).run(softcap=25.0 if seed == 3 else 0.0, **masks)


def test_long_single_tokens_from_scattered_blocks_again_and_again():
    """Many long pieces of alternate key tiles, odd in number, out of a pool far larger than the cache: copies land in any
    order, and an issuer must not take one in flight for landed.  The same bits each time, and the right ones."""
    rng = np.random.default_rng(32)
    ctx = (128 * (2 * rng.integers(10, 90, 40) + 1) - 1 - rng.integers(0, 3, 40)).tolist()
    b = Batch(ctx, [1] * 40, heads=32, kv_heads=8, seed=32)
    c = b.context()
    plan = b.plan(c)
    b.attn(c, plan)
    first = b.o.clone()
    for _ in range(50):
        b.attn(c, plan)
        assert torch.equal(b.o, first)
    assert c.nsd_get_status() == (0, -1)
    b.check()


def test_more_units_than_the_split_keeps_in_shared_memory():
    n, heads, dim = 13000, 2, 64
    from chunk_testlib import context

    g = torch.Generator().manual_seed(33)
    pool = torch.randn((n, 2, 1, 16, dim), generator=g).to(torch.bfloat16).to(DEV)
    q = torch.randn((n, heads, dim), generator=g).to(torch.bfloat16).to(DEV)
    c = context(heads, 1, dim, n, max_batch=n)
    kvi = torch.randperm(n, generator=g).to(torch.int32).to(DEV)
    ramp = torch.arange(n + 1, dtype=torch.int64, device=DEV)
    o, lse = torch.empty_like(q), torch.empty((n, heads), device=DEV)
    plan = torch.empty(c.nsd_chunk_plan_bytes(n), dtype=torch.uint8, device=DEV)
    c.nsd_chunk_plan(plan, n, ramp, torch.full((n,), 3, dtype=torch.int32, device=DEV), ramp)
    c.nsd_chunk_attn(plan, n, pool, q, o, lse, kvi)
    assert c.nsd_get_status() == (0, -1)
    kv = pool[kvi.long()].double()[:, :, 0, :4]                      # four keys each
    s = torch.einsum("nhd,nkd->nhk", q.double(), kv[:, 0]) / dim ** 0.5
    w = torch.softmax(s, -1)
    check_attn(o, lse, (torch.einsum("nhk,nkd->nhd", w, kv[:, 1]), torch.logsumexp(s, -1), torch.einsum("nhk,nkd->nhd", w, kv[:, 1].abs())))
