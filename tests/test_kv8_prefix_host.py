"""What of the 8-bit cache and of the groups' attention needs no GPU: refusals of the library and of the binding, sizes, the format's
definition, and the tolerances' own checks."""
import ctypes

import numpy as np
import pytest
import torch

import kv8_testlib as K
import paper_2609_29364_b200 as nsd
import paper_2609_29364_b200.api as api
from test_chunk_host import _context


# --------------------------------------------------------------------------- the format
def test_the_grid_is_e4m3():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(K.grid(), codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_nearest_is_torch_s_rounding():
    y = torch.cat([torch.linspace(-448, 448, 20001, dtype=torch.float64), torch.linspace(-0.05, 0.05, 5001, dtype=torch.float64),
                   torch.tensor([2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -10, 17.0, 19.0, 0.0])]).float().double()
    assert np.array_equal(K.nearest(y.numpy()), y.float().to(torch.float8_e4m3fn).double().numpy())


def test_exponents_at_the_edges():
    top = np.array([0.0, 448.0, np.nextafter(448.0, 1e9), 447.0, 896.0, 224.0, 224.0 * (1 + 1e-15), 2.0 ** -149, 448 * 2.0 ** -126, 450 * 2.0 ** -126, 3.4e38])
    assert K.exponent(top).tolist() == [-126, 0, 1, 0, 1, -1, 0, -126, -126, -125, 120]


def test_the_scale_byte_rule_is_the_definition_s():
    """The carry out of the mantissa that the kernels use, in integers, against the least exponent."""
    rng = np.random.default_rng(1)
    bits = np.concatenate([rng.integers(0, 0x7F800000, 20000), (np.arange(0, 255) << 23), (np.arange(0, 255) << 23) | 0x600000,
                           (np.arange(0, 255) << 23) | 0x600001]).astype(np.uint32)
    b = (bits.astype(np.int64) + 0x1FFFFF) >> 23
    byte = np.where(b > 9, b - 8, 1)
    assert np.array_equal(byte - 127, K.exponent(bits.view(np.float32).astype(np.float64)))


def test_quantising_keeps_what_is_not_a_number_and_loses_half_a_step_at_most():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((50, 64)) * np.exp2(rng.integers(-40, 40, (50, 1)))
    x[3, 5], x[4, 6] = np.nan, np.inf
    v, e = K.quantise(x)
    assert np.isnan(v[3, 5]) and np.isnan(v[4, 6]) and np.isnan(v).sum() == 2
    y = v * 2.0 ** e[:, None].astype(float)
    ok = np.isfinite(x)
    assert (np.abs(y - x)[ok] <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** (e[:, None] - 10.0) * np.ones_like(x))[ok]).all()


def test_three_terms_hold_a_query_exactly():
    """A bf16 value times a power of two as three numbers of two mantissa bits: the split of the kernel, in numpy."""
    x = torch.randn(20000, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).float().numpy()
    k = 14 - np.floor(np.log2(np.abs(x).max()))
    h = (x * 2.0 ** k).astype(np.float16)

    def upper(a):
        return ((a.view(np.uint16).astype(np.uint32) + 0x80) & 0xFF00).astype(np.uint16).view(np.float16)

    a0 = upper(h)
    r = h - a0
    a1 = upper(r)
    a2 = upper(r - a1)
    small = np.abs(h.astype(np.float64)) < 2.0 ** -9       # below that the last term may fall under the least step
    total = a0.astype(np.float64) + a1.astype(np.float64) + a2.astype(np.float64)
    assert np.array_equal(total[~small], x.astype(np.float64)[~small] * 2.0 ** k)
    assert (np.abs(total - x.astype(np.float64) * 2.0 ** k) <= 2.0 ** -17).all()


# --------------------------------------------------------------------------- refusals
def test_entry_points_refuse_a_missing_context():
    lib, one = nsd.load_library(), ctypes.c_void_p(256)
    assert lib.nsd_kv8_append(None, one, one, 0, 1, 1, one, 8, one, 8, one, 8, one, 8, None, 0, None, None, 0, one, None) == 1
    assert lib.nsd_kv8_pack(None, one, one, one, 1, one, one, 0, 1, None) == 1
    assert lib.nsd_kv8_unpack(None, one, one, one, 1, one, one, 0, 1, None) == 1
    assert lib.nsd_kv8_plan_bytes(None, 5) == 0 and lib.nsd_prefix_plan_bytes(None, 5) == 0
    assert lib.nsd_kv8_plan(None, one, 1, 0, 0, None, None, None, None, None) == 1
    assert lib.nsd_kv8_attn(None, one, 1, one, one, one, 8, one, None, 1, one, 0, 0.0, None) == 1
    assert lib.nsd_prefix_plan(None, one, 1, 0, 0, 0, None, None, None, None, None, None) == 1
    assert lib.nsd_prefix_attn(None, one, 1, one, one, 8, one, None, 1, one, 0, 0.0, 0.0, None, None) == 1


def test_sizes_of_the_cache():
    lib = nsd.load_library()
    cfg = nsd.NsdConfig(num_layers=3, num_slabs=2, num_q_heads=8, num_kv_heads=2, head_dim=64, block_size=16, num_blocks=10, region_b_begin=0,
                        max_batch=1, max_gamma=1, vocab_size=2, max_table_entries=1)
    assert lib.nsd_kv8_pool_bytes(ctypes.byref(cfg)) == 2 * 10 * 2 * 2 * 16 * 64
    assert lib.nsd_kv8_scale_bytes(ctypes.byref(cfg)) == 2 * 10 * 2 * 2 * 16
    cfg.num_blocks = 0
    assert lib.nsd_kv8_pool_bytes(ctypes.byref(cfg)) == 0 and lib.nsd_kv8_scale_bytes(ctypes.byref(cfg)) == 0


def _with_cache(heads=8, kv_heads=2, dim=64, blocks=4):
    c = _context(heads, kv_heads, dim)
    c._kv8_sizes = (blocks * 2 * kv_heads * 16 * dim, blocks * 2 * kv_heads * 16)
    u8 = torch.uint8
    return c, torch.zeros(c._kv8_sizes[0], dtype=u8), torch.zeros(c._kv8_sizes[1], dtype=u8)


def test_binding_refuses_a_cache_of_another_size_or_type():
    c, kv8, scales = _with_cache()
    k = torch.zeros((3, 128))
    slots = torch.zeros(3, dtype=torch.int64)
    for a, b in ((kv8[:-1], scales), (kv8, scales[:-1]), (kv8.float(), scales), (kv8, scales.to(torch.int32)), (kv8.reshape(2, -1).t(), scales)):
        with pytest.raises(ValueError, match="bytes"):
            c.nsd_kv8_append(a, b, 0, None, k, k, None, slots)
    ids = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="one length"):
        c.nsd_kv8_pack(0, kv8, scales, ids, ids[:1])
    with pytest.raises(TypeError, match="int32"):
        c.nsd_kv8_unpack(kv8, scales, 0, ids.long(), ids)
    with pytest.raises(TypeError, match="bfloat16"):
        c.nsd_kv8_attn(kv8, 3, kv8, scales, torch.zeros((3, 512)), kv8, None, ids)
    with pytest.raises(TypeError, match="bfloat16"):
        c.nsd_prefix_attn(kv8, 3, 0, torch.zeros((3, 512)), kv8, None, ids)


def test_binding_refuses_wrong_rows_and_positions():
    c, kv8, scales = _with_cache()
    k, slots = torch.zeros((3, 128)), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="q, or k and v"):
        c.nsd_kv8_append(kv8, scales, 0, None, None, None, None, slots)
    with pytest.raises(ValueError, match="q, or k and v"):
        c.nsd_kv8_append(kv8, scales, 0, None, k, None, None, slots)
    with pytest.raises(ValueError, match="positions"):
        c.nsd_kv8_append(kv8, scales, 0, None, k, k, None, slots, None, [32], torch.ones(32))
    with pytest.raises(ValueError, match="positions"):
        c.nsd_kv8_append(kv8, scales, 0, None, k, k, None, slots, torch.zeros((1, 2), dtype=torch.int32), [32], torch.ones(32))
    with pytest.raises(ValueError, match="slot_map"):
        c.nsd_kv8_append(kv8, scales, 0, None, k, k, None, slots[:2])
    with pytest.raises(ValueError, match="rows of"):
        c.nsd_kv8_append(kv8, scales, 0, None, k[:, :64], k, None, slots)


def test_binding_refuses_tensors_that_the_device_cannot_read():
    c, kv8, scales = _with_cache()
    i64, i32 = torch.zeros(3, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)
    k, q = torch.zeros((3, 128)), torch.zeros((3, 512), dtype=torch.bfloat16)
    for call in (lambda: c.nsd_kv8_append(kv8, scales, 0, None, k, k, None, i64), lambda: c.nsd_kv8_pack(q, kv8, scales, i32, i32, 0, 1),
                 lambda: c.nsd_kv8_unpack(kv8, scales, q, i32, i32, 0, 1), lambda: c.nsd_kv8_plan(kv8, 3, i64, i32[:2], i64),
                 lambda: c.nsd_kv8_attn(kv8, 3, kv8, scales, q, q, None, i32), lambda: c.nsd_prefix_plan(kv8, 3, i64, i32[:2], i64, i32[:2], i64),
                 lambda: c.nsd_prefix_attn(kv8, 3, q, q, q, None, i32)):
        with pytest.raises(ValueError, match="cuda:0"):
            call()


def test_binding_refuses_groups_of_another_length():
    c, plan, _ = _with_cache()
    i64, i32 = torch.zeros(3, dtype=torch.int64), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="group_indptr"):
        c.nsd_prefix_plan(plan, 3, i64[:2], i32, i64, i32, i64)
    with pytest.raises(TypeError, match="prefix_len"):
        c.nsd_prefix_plan(plan, 3, i64, i32.long(), i64, i32, i64)
    with pytest.raises(ValueError, match="q_indptr"):
        c.nsd_prefix_plan(plan, 3, i64, i32, i64[:2], i32, i64)


# --------------------------------------------------------------------------- the tolerances see a mistake
def _case():
    g = torch.Generator().manual_seed(4)
    o, lse = torch.randn((3, 2, 64), generator=g, dtype=torch.float64), torch.randn((3, 2), generator=g, dtype=torch.float64)
    return o, lse, o.abs() + 0.5


@pytest.mark.parametrize("wrong", ["one element", "lse", "nan", "row"])
def test_a_planted_mistake_is_seen(wrong):
    o, lse, mag = _case()
    K.check_attn8(o.to(torch.bfloat16), lse.float(), (o, lse, mag), 100, 4.0)
    a, b = o.to(torch.bfloat16).clone(), lse.float().clone()
    if wrong == "one element":
        a[1, 1, 7] += 0.05
    elif wrong == "lse":
        b[2, 0] += 0.01
    elif wrong == "nan":
        a[0, 0, 0] = float("nan")
    else:
        a[[0, 1]] = a[[1, 0]]
    with pytest.raises(AssertionError):
        K.check_attn8(a, b, (o, lse, mag), 100, 4.0)
