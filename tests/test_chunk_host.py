"""What of the chunk operators needs no GPU: refusals, constants and structures of the binding, the 64-bit forms the GPU
tests compare with, and the arithmetic of the work split."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import chunk_testlib as T
import paper_2609_29364_b200 as nsd
import paper_2609_29364_b200.api as api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    text = open(os.path.join(ROOT, "include", "nsd.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_entry_points_refuse_a_missing_context():
    lib = nsd.load_library()
    one = ctypes.c_void_p(256)
    assert lib.nsd_block_tables(None, 0, one, one, one, 1, one, one, 1, None, 0, 0, one, one, one, None, None, None, one, one, None) == 1
    assert lib.nsd_rope_append(None, one, 0, 1, 1, one, 8, one, 8, one, 8, one, 8, one, 1, one, one, 0, one, None) == 1
    assert lib.nsd_chunk_plan_bytes(None, 5) == 0
    assert lib.nsd_chunk_plan(None, one, 1, 0, 0, None, None, None, None, None) == 1
    assert lib.nsd_chunk_attn(None, one, 1, one, one, 8, one, None, 1, one, 0, 0.0, 0.0, None, None) == 1


def test_rope_flags_and_masks_match_the_header():
    header = {n: 1 << int(s) for n, s in re.findall(r"\b(NSD_ROPE_[A-Z]+)\s*=\s*1\s*<<\s*(\d+)", _header())}
    assert header == {n: getattr(nsd, n) for n in dir(nsd) if n.startswith("NSD_ROPE_")} and len(header) == 2
    body = re.search(r"typedef struct \{([^}]*)\} nsd_chunk_masks;", _header()).group(1)
    fields = re.findall(r"(\w+);", body)
    assert fields == [n for n, _ in api.ChunkMasks._fields_]
    assert ctypes.sizeof(api.ChunkMasks) == 4 + 4 + 8 + 8


class _Lib:
    def __getattr__(self, name):
        def reached(*args):
            raise AssertionError(f"{name} was reached with arguments that the binding has to refuse")
        return reached


def _context(heads=8, kv_heads=2, dim=64):
    c = api.VerifyContext.__new__(api.VerifyContext)
    c.lib, c._h, c.cfg = _Lib(), None, api.NsdConfig(num_layers=1, num_q_heads=heads, num_kv_heads=kv_heads, head_dim=dim)
    c._i32, c._i64, c._f32, c._bf16 = torch.int32, torch.int64, torch.float32, torch.bfloat16
    c._raw_stream, c._device_index = (lambda index: 0), 0
    return c


def test_binding_refuses_wrong_tables():
    i32, i64 = torch.int32, torch.int64
    good = dict(ctx_len=torch.zeros(2, dtype=i32), new_len=torch.zeros(2, dtype=i32), held=torch.zeros((2, 4), dtype=i32),
                n_held=torch.zeros(2, dtype=i32), free_blocks=torch.zeros(3, dtype=i32), free_begin=None,
                kv_indptr=torch.zeros(3, dtype=i64), kv_indices=torch.zeros(5, dtype=i32), q_indptr=torch.zeros(3, dtype=i64),
                slot_map=torch.zeros(4, dtype=i64), positions=torch.zeros(4, dtype=i32), row_req=None,
                n_held_new=torch.zeros(2, dtype=i32), free_end=torch.zeros(1, dtype=i64))
    for bad, error in ((dict(ctx_len=torch.zeros(2, dtype=i64)), TypeError), (dict(new_len=torch.zeros(1, dtype=i32)), ValueError),
                       (dict(held=torch.zeros(8, dtype=i32)), ValueError), (dict(held=torch.zeros((1, 4), dtype=i32)), ValueError),
                       (dict(held=torch.zeros((4, 2), dtype=i32).t()), ValueError), (dict(kv_indptr=torch.zeros(2, dtype=i64)), ValueError),
                       (dict(positions=torch.zeros(3, dtype=i32)), ValueError), (dict(free_end=torch.zeros(1, dtype=i32)), TypeError)):
        with pytest.raises(error):
            _context().nsd_block_tables(**{**good, **bad})


def test_binding_refuses_wrong_rope_and_attention_arguments():
    c, bf = _context(), torch.bfloat16
    q, k, out = torch.zeros((3, 512), dtype=bf), torch.zeros((3, 128), dtype=bf), torch.zeros((3, 8, 64), dtype=bf)
    pos, f, slots = torch.zeros((1, 3), dtype=torch.int32), torch.ones(32), torch.zeros(3, dtype=torch.int64)
    pool = torch.zeros((1, 4, 2, 2, 16, 64), dtype=bf)
    args = lambda **x: {**dict(kv_pool=pool, layer=0, q=q, k=k, v=k, q_out=out, positions=pos, sections=[32], inv_freq=f, slot_map=slots), **x}  # noqa: E731
    for bad, error in ((dict(k=None), ValueError), (dict(q=None, k=None, v=None), ValueError), (dict(v=k[:2]), ValueError),
                       (dict(k=k.float()), ValueError), (dict(q=q[:, ::2]), ValueError), (dict(q_out=out.float()), TypeError),
                       (dict(positions=pos[0]), ValueError), (dict(sections=[16, 16]), ValueError), (dict(inv_freq=f[:8]), ValueError),
                       (dict(slot_map=slots.int()), TypeError), (dict(positions=pos.long()), TypeError)):
        with pytest.raises(error):
            c.nsd_rope_append(**args(**bad))
    plan, kvi, o, lse = torch.zeros(256, dtype=torch.uint8), torch.zeros(4, dtype=torch.int32), torch.zeros((3, 8, 64), dtype=bf), torch.zeros(24)
    for bad, error in ((dict(q=q.float()), TypeError), (dict(q=q[:2]), TypeError), (dict(o=o[:2]), ValueError), (dict(lse=lse[:5]), ValueError),
                       (dict(kv_indices=kvi.long()), TypeError), (dict(alibi_slopes=torch.ones(3)), ValueError), (dict(q=q[:, :256]), ValueError)):
        with pytest.raises(error):
            c.nsd_chunk_attn(**{**dict(plan=plan, max_rows=3, kv_pool=pool, q=q, o=o, lse=lse, kv_indices=kvi), **bad})
    i = torch.zeros(2, dtype=torch.int64)
    for bad, error in ((dict(q_indptr=i[:1]), ValueError), (dict(ctx_len=torch.zeros(1)), TypeError), (dict(row_first=torch.zeros(2, dtype=torch.int32)), ValueError)):
        with pytest.raises(error):
            c.nsd_chunk_plan(**{**dict(plan=plan, max_rows=3, q_indptr=i, ctx_len=torch.zeros(1, dtype=torch.int32), kv_indptr=i), **bad})


def test_reference_attention_equals_torch():
    """Plain causal attention over a gathered cache, against torch's own in 64 bits."""
    g = torch.Generator().manual_seed(0)
    ctx, new, heads, hkv, d = [5, 0, 33], [7, 20, 1], 6, 2, 8
    need = [T.blocks_of(a + b) for a, b in zip(ctx, new)]
    kvp = T.offsets(need)
    pool = torch.randn((int(kvp[-1]) + 2, 2, hkv, 16, d), generator=g, dtype=torch.float64)
    kvi = torch.randperm(pool.shape[0], generator=g)[:int(kvp[-1])].numpy()
    q = torch.randn((sum(new), heads, d), generator=g, dtype=torch.float64)
    o, lse, mag = T.attn_ref(q, pool, ctx, new, kvp, kvi)
    row = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        kv = pool[kvi[kvp[r]:kvp[r + 1]]].permute(1, 2, 0, 3, 4).reshape(2, hkv, -1, d)[:, :, :c + n].repeat_interleave(heads // hkv, 1)
        mask = torch.arange(c + n)[None] <= c + torch.arange(n)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(q[row:row + n].transpose(0, 1), kv[0], kv[1], attn_mask=mask)
        assert torch.allclose(o[row:row + n].transpose(0, 1), want, atol=1e-12)
        row += n
    assert (mag >= o.abs() - 1e-12).all() and torch.isfinite(lse).all()


def test_visible_keys_by_hand():
    assert T.visible([3], [2], window=2) == [(2, 4), (3, 5)]
    assert T.visible([3], [2], prefix_len=[9]) == [(0, 5), (0, 5)]
    assert T.visible([1], [2], prefix_len=[1], row_first=[0, 2]) == [(0, 2), (2, 3)]
    assert T.visible([0, 2], [1, 1], row_first=[5, 0]) == [(5, 1), (0, 3)]


@pytest.mark.parametrize("adjacent", [False, True])
def test_reference_rotation_keeps_lengths_and_adds_angles(adjacent):
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((4, 3, 16)), rng.random(6)
    a, b = rng.integers(0, 50, (1, 4)), rng.integers(0, 50, (1, 4))
    one, _ = T.rope_ref(x, a, [6], f, adjacent, False)
    two, _ = T.rope_ref(one, b, [6], f, adjacent, False)
    both, _ = T.rope_ref(x, a + b, [6], f, adjacent, False)
    assert np.allclose(two, both, atol=1e-12) and np.allclose(one[..., 12:], x[..., 12:])
    assert np.allclose((one ** 2).sum(-1), (x ** 2).sum(-1))
    assert T.axis_of_pair([3, 2, 2], True) == [0, 1, 2, 0, 1, 2, 0] and T.axis_of_pair([3, 2, 2], False) == [0, 0, 0, 1, 1, 2, 2]


# ---- the split of the work, restated
UNIT_TILES, TILE = 2, 128


def _units(ctx, new, t):
    """(request, tokens, key tiles, first unit, last unit) in the order of the compact list, from the scattered index."""
    tu, qp = 2 * t, T.offsets(new)
    raw = {}
    for r, (c, n) in enumerate(zip(ctx, new)):
        s, e = int(qp[r]), int(qp[r + 1])
        count = -(-n // tu)
        for j in range(1 + e // tu - s // tu):
            at = r + s // tu + j
            assert at not in raw
            raw[at] = None if j >= count else (r, min(tu, n - j * tu), -(-(c + min(n, (j + 1) * tu)) // TILE), j, count)
    assert sorted(raw) == list(range(len(new) + int(qp[-1]) // tu))
    out = []
    for at in sorted(raw):
        if raw[at]:
            r, ntok, tiles, j, count = raw[at]
            out.append((r, ntok, tiles, len(out) - j, len(out) - j + count - 1))
    return out


def _starts(units, t, hkv, ctas):
    weight = [2 if u[1] > t else 1 for u in units]
    cost = T.offsets([(u[2] + UNIT_TILES) * w for u, w in zip(units, weight)])
    out = []
    for c in range(ctas):
        pos = int(cost[-1]) * hkv * c // ctas
        at = max(i for i in range(len(units)) if int(cost[i]) * hkv <= pos)
        first, last = units[at][3], units[at][4]
        head_cost, inside = int(cost[last + 1] - cost[first]), pos - int(cost[first]) * hkv
        head, rem = inside // head_cost, inside % head_cost + int(cost[first])
        u = max(i for i in range(first, last + 1) if int(cost[i]) <= rem)
        out.append((u, head, max(0, (rem - int(cost[u])) // weight[u] - UNIT_TILES)))
    return out + [(len(units), 0, 0)]


@pytest.mark.parametrize("seed", range(12))
def test_every_key_tile_belongs_to_one_piece(seed):
    rng = np.random.default_rng(seed)
    t, hkv, ctas = int(rng.choice([4, 18, 32, 128])), int(rng.integers(1, 9)), int(rng.choice([3, 148]))
    n = int(rng.integers(1, 30))
    ctx = rng.integers(0, 3000, n).tolist()
    new = np.where(rng.random(n) < 0.5, 1, rng.integers(0, 700, n)).tolist()
    units = _units(ctx, new, t)
    if not units:
        return
    starts, seen, slots = _starts(units, t, hkv, ctas), {}, set()
    total = sum((u[2] + UNIT_TILES) * (2 if u[1] > t else 1) for u in units) * hkv
    for c in range(ctas):
        share = 0
        at, end = starts[c], starts[c + 1]
        while at != end:
            u, h, k0 = at
            cut = (u, h) == end[:2]
            k1 = end[2] if cut else units[u][2]
            slot = 2 * c if k0 > 0 else (2 * c + 1 if cut else -1)
            if slot >= 0:
                assert slot not in slots
                slots.add(slot)
            assert (k0, k1) not in seen.setdefault((u, h), []) and k0 < k1
            seen[(u, h)].append((k0, k1))
            share += (k1 - k0) * (2 if units[u][1] > t else 1)
            if cut:
                break
            at = (u + 1, h, 0) if u < units[u][4] else ((units[u][3], h + 1, 0) if h + 1 < hkv else (units[u][4] + 1, 0, 0))
        # no CTA's tiles cost more than its part of the line and a tile at its ends
        assert share <= total / ctas + 3
    assert sorted(seen) == [(u, h) for u in range(len(units)) for h in range(hkv)]
    for (u, _), pieces in seen.items():
        pieces.sort()
        assert pieces[0][0] == 0 and pieces[-1][1] == units[u][2] and all(a[1] == b[0] for a, b in zip(pieces, pieces[1:]))
