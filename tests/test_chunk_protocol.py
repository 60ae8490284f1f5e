"""The barrier protocol of the chunk attention in random walks (chunk_protocol_model.py)."""
import random

import numpy as np
import pytest

from chunk_protocol_model import Cta, walks
from test_chunk_host import _starts, _units


def test_nothing_gets_stuck_or_takes_a_tile_in_flight_for_landed():
    assert walks(1, 1200) == {"ok": 1200}


def _pieces(units, start, end, hkv):
    out, at = [], start
    while at != end:
        u, h, k0 = at
        cut = (u, h) == end[:2]
        out.append(((end[2] if cut else units[u][2]) - k0, units[u][1]))
        if cut:
            break
        at = (u + 1, h, 0) if u < units[u][4] else ((units[u][3], h + 1, 0) if h + 1 < hkv else (units[u][4] + 1, 0, 0))
    return out


@pytest.mark.parametrize("heads,hkv,dim", [(32, 8, 128), (12, 4, 64)])
def test_the_walks_of_a_mixed_batch(heads, hkv, dim):
    rng, rnd = np.random.default_rng(5), random.Random(5)
    ctx = np.where(rng.random(24) < 0.3, rng.integers(0, 40, 24), rng.integers(0, 4000, 24))
    new = np.where(rng.random(24) < 0.6, 1, rng.integers(0, 400, 24))
    t = 128 // (heads // hkv)
    units = _units(ctx.tolist(), new.tolist(), t)
    starts = _starts(units, t, hkv, 148)
    for c in range(148):
        pieces = [(n, tokens > t) for n, tokens in _pieces(units, starts[c], starts[c + 1], hkv)]
        assert Cta(pieces, dim, rnd).run() == "ok"


def test_both_issuers_have_to_release_the_q_buffers_of_a_pair():
    """Released by its owner alone, a buffer can be filled twice between two looks of the other issuer, whose wait then never
    passes."""
    assert walks(1, 300, pairs_release_q=False).get("stuck", 0) > 0


def test_who_gives_up_leaves_nothing_in_flight():
    got = walks(2, 3000, give_up=0.002)
    assert set(got) == {"ok", "gave up"} and got["gave up"] > 1000


def test_a_tile_counts_as_soon_as_its_copies_are_sent():
    """Counted at the end of its turn instead, a tile whose turn ends in a wait that runs out is not waited for."""
    assert walks(2, 1500, give_up=0.002, counted_when_sent=False).get("in flight", 0) > 0


def test_the_flag_is_read_when_it_is_final():
    """Read by each actor as it ends, one that ends before another gives up leaves behind what it has in flight."""
    assert walks(2, 4000, give_up=0.002, flag_is_final=False).get("in flight", 0) > 0
