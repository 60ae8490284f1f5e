"""The marked contexts notice single keys: mistakes planted in the definition, on the CPU."""
import numpy as np
import pytest

from chunk_marked import Marked
from chunk_testlib import check_attn


def _flagged(right, wrong):
    try:
        check_attn(wrong[0], wrong[1], right)
    except AssertionError:
        return True
    return False


@pytest.mark.parametrize("kw", [{}, dict(softcap=50.0), dict(softcap=50.0, slopes=[-0.0005, 0.001, 0.0, 0.0002])])
@pytest.mark.parametrize("window", [999, 1001])
def test_a_window_off_by_one_is_noticed(window, kw):
    w = 1000
    m = Marked([3000], [9], 4, 2, 64, [p + d for p in range(3000, 3009) for d in (-w, 1 - w, 0, 1)], seed=1)
    seen = 0
    for q in m.queries(lambda p: (p - w, p - w + 1, p)):
        right = m.reference(q, window=w, **kw)
        assert not _flagged(right, right)
        seen += _flagged(right, m.reference(q, window=window, **kw))
    assert seen == 3                                   # in every turn some row points at the key that differs


def test_a_lost_block_is_noticed():
    m = Marked([5000], [1], 4, 2, 64, [2 * 16, 3 * 16 - 1, 200 * 16], seed=2)
    table = m.kv_indices.copy()
    for q in m.queries(lambda p: m.marks):
        right = m.reference(q)
        for lost in (2, 200):
            m.kv_indices = table.copy()
            m.kv_indices[lost] = table[lost + 1]
            assert _flagged(right, m.reference(q))
        m.kv_indices = table


def test_every_marked_key_has_its_turn():
    m = Marked([100], [3], 4, 2, 64, [5, 50, 90, 101], seed=3)
    want = {(h, t) for h in range(4) for t in (5, 50, 90)}
    point = m.point.float().numpy()
    got = set()
    for q in m.queries(lambda p: (5, 50, 90)):
        for row in q.float().numpy():
            for h in range(4):
                got.add((h, m.marks[int(np.flatnonzero((point == row[h]).all(1))[0])]))
    assert got == want
