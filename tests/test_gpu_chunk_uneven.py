"""Plans of batches whose rows lie in few of their requests: every unit is found, whatever the request it belongs to."""
import numpy as np
import pytest
import torch

from chunk_testlib import DEV, Batch, context, gpu, offsets
from kv8_testlib import Batch8

pytestmark = pytest.mark.gpu


def uneven(n, long, at, seed):
    """n requests of 0 to 2 new tokens, and `long` of them where `at` says."""
    rng = np.random.default_rng(seed)
    new = rng.integers(0, 3, n)
    new[at] = long
    return rng.integers(0, 40, n).tolist(), new.tolist()


@pytest.mark.parametrize("at", [0, 31, 32, 150, 299])
def test_one_long_request_among_many(at):
    ctx, new = uneven(300, 700, at, at)
    Batch8(ctx, new, heads=4, kv_heads=2, dim=64, seed=at, pad_rows=3).run()
    Batch(ctx, new, heads=4, kv_heads=2, dim=64, seed=at, pad_rows=3).run()


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 1024, 1025])
def test_as_many_requests_as_a_search_can_miss(n):
    """Numbers of requests around the widths of the search, most of them without rows."""
    new = [0] * n
    for r in {0, n // 2, n - 1}:
        new[r] = 3 + r % 50
    Batch8([5] * n, new, heads=4, kv_heads=2, dim=64, seed=n, pad_rows=130).run()


def test_many_more_rows_held_than_used():
    ctx, new = uneven(40, 65, 7, 1)
    Batch8(ctx, new, heads=4, kv_heads=2, dim=64, seed=3, pad_rows=60000).run()


@pytest.mark.parametrize("bad", [0, 17, 39])
def test_a_malformed_request_is_named(bad):
    ctx, new = uneven(40, 65, 20, 2)
    b = Batch8(ctx, new, heads=4, kv_heads=2, dim=64, seed=4)
    c = b.context()
    b.ctx_len[bad] = -1
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (6, bad) and (b.o == 7.0).all()


@pytest.mark.parametrize("seed", range(3))
def test_offsets_of_any_value_are_refused(seed):
    """Offsets that fall, are negative or lie beyond the buffer: an empty plan, nothing written.  (That nothing is read or written
    out of place was checked beforehand on the host: every slot's request, rows and place in the plan are clamped or compared.)"""
    rng = np.random.default_rng(seed)
    ctx, new = uneven(60, 200, 30, seed)
    b = Batch8(ctx, new, heads=4, kv_heads=2, dim=64, seed=5)
    c = b.context()
    wrong = b.qp.clone()
    for at in rng.integers(1, 61, 5):
        wrong[int(at)] = int(rng.choice([-1, -2 ** 62, 2 ** 62, b.max_rows + 1, 0]))
    wrong[60] = int(rng.choice([-5, 2 ** 62, 3]))
    b.qp = wrong
    b.attn(c, b.plan(c))
    assert c.nsd_get_status()[0] == 6 and (b.o == 7.0).all() and (b.lse == 7.0).all()


def plan_time(new):
    """Least device time of eight plans, in microseconds."""
    c = context(32, 8, 128, num_blocks=64, max_batch=len(new))
    rows, zeros = int(np.sum(new)), np.zeros(len(new) + 1, dtype=np.int64)
    qp, kvp, ctx = gpu(offsets(new)), gpu(zeros), torch.zeros(len(new), dtype=torch.int32, device=DEV)
    plan = torch.empty(c.nsd_kv8_plan_bytes(rows), dtype=torch.uint8, device=DEV)
    best = float("inf")
    for _ in range(10):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        a.record()
        for _ in range(8):
            c.nsd_kv8_plan(plan, rows, qp, ctx, kvp)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) / 8 * 1000)
    assert c.nsd_get_status() == (0, -1)
    return best


def test_one_long_request_among_many_takes_no_longer_than_by_itself():
    """As many rows in one request, and in one of 512: the same units, so about the same time (three times as much where each
    request gets its share of the GPU)."""
    assert plan_time([1] * 511 + [100000]) < 2 * plan_time([100511])
