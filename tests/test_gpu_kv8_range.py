"""Attention over the 8-bit cache where rows of V differ by many powers of two, each row held to a limit of its own."""
import numpy as np
import pytest
import torch

from chunk_testlib import DEV
from kv8_range_testlib import Range8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("byte", [248, 250, 254, 255])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_scale_that_is_none_stays_with_the_rows_that_see_it(dim, byte):
    """The power of two of V, or of K, of a drafted token: only the rows from that token on see it."""
    for kv in (0, 1):
        b = Range8([200, 40, 130], [4, 3, 1], dim=dim, seed=byte)
        spoilt = []
        for request, token, first in ((0, 203, 3), (1, 41, 5)):
            block, slot = b.place(request, token)
            b.scales[0, block, 1, kv, slot] = byte
            spoilt += list(range(first, 4 if request == 0 else 7))
        c = b.context()
        b.attn(c, b.plan(c))
        assert c.nsd_get_status() == (0, -1)
        bad = torch.zeros((b.rows, b.heads), dtype=torch.bool, device=DEV)
        bad[spoilt, b.heads // 2:] = True
        assert torch.equal(torch.isnan(b.o[0]).all(-1), bad) and torch.equal(torch.isnan(b.o[0]).any(-1), bad)
        assert torch.equal(torch.isnan(b.lse[0]), bad)
        b.o[0][bad], b.lse[0][bad] = 0.0, 0.0
        good = [r for r in range(b.rows) if r not in spoilt]
        b.close(rows=good)


@pytest.mark.parametrize("by", [117, 100, 60, -60, -100, -115])
@pytest.mark.parametrize("dim", [64, 128])
def test_large_and_small_v_in_pieces_as_in_whole_units(dim, by):
    """A context that many CTAs share, whose pieces are joined, and requests that each have one to themselves."""
    b = Range8([20000], [2], dim=dim, heads=4, kv_heads=1, seed=by % 97)
    b.shift_v(0, by)
    b.run_close()
    b = Range8([300] * 300, [1] * 300, dim=dim, heads=4, kv_heads=1, seed=by % 89)
    for r in range(300):
        b.shift_v(r, by)
    b.run_close()


@pytest.mark.parametrize("dim", [64, 128])
def test_small_queries_with_large_keys(dim):
    """Queries near the least numbers against keys near the largest, under a small scale."""
    b = Range8([300, 20, 140], [3, 1, 2], dim=dim, heads=8, kv_heads=2, seed=5)
    b.q.mul_(2.0 ** -118)
    held = b.scales != 255
    b.scales[0, :, :, 0] = torch.where(held[0, :, :, 0], b.scales[0, :, :, 0] + 118, 255).to(torch.uint8)
    b.values[0, :, 0] *= 2.0 ** 118
    for scale in (0.1, 2.0 ** -9):
        if scale < 0.01:
            b.scales[0, :, :, 0] = torch.where(held[0, :, :, 0], b.scales[0, :, :, 0] + 5, 255).to(torch.uint8)
            b.values[0, :, 0] *= 2.0 ** 5
        b.run_close(scale=scale)


@pytest.mark.parametrize("tokens", [1, 5])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_large_v_with_next_to_no_weight(dim, tokens):
    """One row of V 2^22 to 2^118 larger than the others, of a key whose weight is below 2^-60 of a row's: first, last and in the
    middle of contexts that each have a CTA to themselves."""
    n = 150
    b = Range8([600] * n, [tokens] * n, dim=dim, heads=4, kv_heads=2, seed=11 + tokens)
    for r in range(n):
        token = (0, 599, 300, 130, 127)[r % 5]
        b.point(r, token, -(45.0, 65.0, 100.0)[r // 5 % 3])
        b.shift_v(r, (22, 24, 26, 30, 40, 59, 64, 80, 100, 118)[r // 15], [token])
    b.run_close()


@pytest.mark.parametrize("ctx", [140, 9000])
@pytest.mark.parametrize("by", [22, 30, 45, 90, 118])
def test_a_large_v_with_next_to_no_weight_in_pieces(by, ctx):
    for token in (0, ctx // 2, ctx - 1):
        b = Range8([ctx], [3], heads=8, kv_heads=2, seed=by)
        b.point(0, token, -60.0)
        b.shift_v(0, by, [token])
        b.run_close()


@pytest.mark.parametrize("by", [10, 22, 30, 45, 60, 90, 118, -60, -110])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_large_v_that_only_later_rows_see(dim, by):
    """Drafted tokens whose V differs from the context's by many powers of two: the rows before them do not see it."""
    n = 80
    b = Range8([260] * n, [5] * n, dim=dim, heads=8, kv_heads=2, seed=by % 101)
    for r in range(n):
        b.shift_v(r, by, [(264,), (262,), (261, 264), (263, 260)][r % 4])
    b.run_close()


@pytest.mark.parametrize("dim", [64, 128])
def test_v_of_every_size_alone_and_mixed(dim):
    """Whole requests of one size, rows of random sizes with scores of order one and twenty, sizes that grow and fall along
    the context, and rows of zeros: all of them, a whole tile, single ones with and without all of the weight."""
    rng = np.random.default_rng(21)
    n = 160
    b = Range8([500] * n, [3] * n, dim=dim, heads=4, kv_heads=2, seed=21)
    for r in range(n):
        kind = r % 8
        if kind == 0:
            b.shift_v(r, (-115, -90, -62, -56, -50, -30, 0, 30, 40, 44, 48, 52, 56, 60, 75, 90, 100, 110, 117, 118)[r // 8])
        elif kind == 1:
            b.shift_v(r, rng.integers(-115, 119, 503))
        elif kind == 2:
            b.shift_v(r, np.round(np.linspace(-115, 118, 503)).astype(int)[::1 if r % 16 < 8 else -1])
        elif kind == 3:
            b.clear_v(r) if r % 3 == 0 else b.clear_v(r, np.arange(128 if r % 3 == 1 else 300))
        elif kind == 4:
            b.clear_v(r, [int(rng.integers(0, 500))])
            b.point(r, 5 + r, 60.0)
            b.clear_v(r, [5 + r])
        elif kind == 5:
            b.point(r, 200 + r, 90.0)
            b.shift_v(r, -int(rng.integers(0, 115)), [200 + r])
        elif kind == 6:
            for t in rng.integers(0, 500, 40):
                b.point(r, int(t), float(rng.normal() * 20))
            b.shift_v(r, rng.integers(-115, 119, 503))
        else:
            b.shift_v(r, rng.integers(-30, 31, 503))
    b.run_close()
    b.run_close(window=200)


@pytest.mark.parametrize("seed", range(6))
def test_random_sizes_in_random_batches(seed):
    rng = np.random.default_rng(seed)
    heads, hkv, dim = [(8, 2, 128), (4, 4, 64), (5, 1, 64), (32, 1, 128), (28, 4, 128), (12, 4, 64)][seed]
    n = int(rng.integers(1, 30))
    ctx, new = rng.integers(0, 1500, n).tolist(), rng.integers(1, 12, n).tolist()
    b = Range8(ctx, new, heads=heads, kv_heads=hkv, dim=dim, seed=seed)
    for r in range(n):
        total = ctx[r] + new[r]
        b.shift_v(r, rng.integers(-115, 119, total) if rng.random() < 0.5 else rng.integers(-40, 41, total))
        for t in rng.integers(0, total, total // 8):
            b.point(r, int(t), float(rng.normal() * 30))
    b.run_close()
    b.run_close(row_first=[int(rng.integers(0, 400)) if rng.random() < 0.5 else 0 for _ in range(b.rows)]) if min(ctx) > 500 else None


@pytest.mark.parametrize("tokens", [1, 5])
@pytest.mark.parametrize("dim", [64, 128])
def test_equal_scores_beyond_2_24_weigh_the_same(dim, tokens):
    """Two keys with one score that no other comes near, the first where the row's reference moves: the mean of their rows of V.
    The scores, 2^26 and up in steps of some 2^8, are exact sums of two products."""
    n = 40
    b = Range8([700] * n, [tokens] * n, dim=dim, heads=8, kv_heads=2, seed=3)
    b.q.zero_()
    q = b.q.view(1, b.rows, b.heads, dim)
    q[..., 0], q[..., 1] = 2.0 ** 18, 1.0
    b.kv8[0, :, 0], b.values[0, :, 0] = torch.where(b.kv8[0, :, 0] == 0x7F, 0x7F, 0).to(torch.uint8), 0.0

    def key(request, token, first, second):
        block, slot = b.place(request, token)
        for d, x in ((0, first), (1, second)):
            b.kv8[0, block, 0, :, slot, d] = torch.tensor([x]).to(torch.float8_e4m3fn).view(torch.uint8).to(DEV)
            b.values[0, block, 0, :, slot, d] = x
        b.scales[0, block, :, 0, slot] = 127
    for r in range(n):
        key(r, 5 + r, 256.0, 0.0)                      # 2^26
        key(r, 300 + r, 256.0, 128.0 + 16 * (r % 16))  # more by 128 to 368
        key(r, 500 + r, 256.0, 128.0 + 16 * (r % 16))  # the same again, in a later tile
    b.run_close(scale=1.0)


@pytest.mark.parametrize("dim", [64, 128])
def test_queries_of_zeros_beside_ones_whose_scores_overflow(dim):
    """One head's scores are beyond 32 bits; the other's are all 0, and its rows the mean of V."""
    b = Range8([200, 30], [3, 1], dim=dim, heads=2, kv_heads=1, seed=7)
    q = b.q.view(1, b.rows, 2, dim)
    q[0, :, 0], q[0, :, 1] = 0.0, 2.0 ** 126
    held = b.scales[0, :, :, 0] != 255
    b.scales[0, :, :, 0] = torch.where(held, b.scales[0, :, :, 0] + 100, 255).to(torch.uint8)
    b.values[0, :, 0] *= 2.0 ** 100
    c = b.context()
    b.attn(c, b.plan(c))
    assert c.nsd_get_status() == (0, -1)
    o_ref = torch.stack([b.values[0, b.places(r)[0], 1, 0, b.places(r)[1]][: b.ctx[r] + i + 1].mean(0) for r in range(2) for i in range(b.new[r])])
    mag = torch.stack([b.values[0, b.places(r)[0], 1, 0, b.places(r)[1]][: b.ctx[r] + i + 1].abs().mean(0) for r in range(2) for i in range(b.new[r])])
    keys = torch.tensor([float(b.ctx[r] + i + 1) for r in range(2) for i in range(b.new[r])], dtype=torch.float64, device=DEV)
    assert ((b.o[0, :, 0].double() - o_ref).abs() <= 2.0 ** -8 * o_ref.abs() + 2.0 ** -9 * mag).all()
    assert ((b.lse[0, :, 0].double() - keys.log()).abs() <= 2.0 ** -10).all()
