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
