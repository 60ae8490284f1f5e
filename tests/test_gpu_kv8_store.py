"""Writing the 8-bit cache row by row, packing whole blocks into it and unpacking them, against the format's definition."""
import numpy as np
import pytest
import torch

import chunk_testlib as T
import kv8_testlib as K
from chunk_testlib import BS, DEV, gpu

pytestmark = pytest.mark.gpu

SHAPES = [(8, 2, 128), (8, 2, 64), (5, 5, 64), (28, 4, 128), (24, 1, 128)]


def cache(c, fill=0xA5):
    """An 8-bit cache whose bytes are all `fill`."""
    n, m = c.kv8_bytes()
    cfg = c.cfg
    return (torch.full((cfg.num_slabs, cfg.num_blocks, 2, cfg.num_kv_heads, BS, cfg.head_dim), fill, dtype=torch.uint8, device=DEV),
            torch.full((cfg.num_slabs, cfg.num_blocks, cfg.num_kv_heads, 2, BS), fill, dtype=torch.uint8, device=DEV), (n, m))


def rows_like_a_model(rows, heads, dim, seed, dtype):
    """Rows of unlike size, among them a zero row, rows at the edges of the scale's rule and rows far from 1."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, heads, dim), generator=g, dtype=torch.float64)
    x *= torch.exp2(torch.randint(-12, 13, (rows, heads, 1), generator=g).double())
    if rows > 8:
        x[0] = 0.0
        x[1, :, 0] = 448.0 * 2.0 ** 5                      # exactly the largest code
        x[1, :, 1:] = x[1, :, 1:].clamp(-448, 448)
        x[2] = 1e-30 * x[2]
        x[3] = 1e30 * x[3]
        x[4] = 2.0 ** -131 * torch.sign(x[4])              # below the least scale: subnormal codes or zero
        x[5, :, -1] = 1e4
        x[6, :, :] = torch.where(torch.rand(x[6].shape, generator=g) < 0.5, 1.0625, -17.0).double()     # ties
    return x.to(dtype)


def assert_rows(kv8, scales, want, where):
    """want [n][hkv][D] float64 at [block][slot] pairs `where`, as K or V."""
    values, e = K.quantise(want)
    got = K.code_values(kv8)
    assert np.array_equal(got, values, equal_nan=True), f"{(got != values).sum()} codes differ"
    assert np.array_equal(scales.cpu().numpy(), e + 127), "scales"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("rows", [1, 2, 17, 333])
def test_append_quantises_rows(shape, rows, dtype):
    heads, hkv, dim = shape
    c = T.context(heads, hkv, dim, num_blocks=40, num_layers=2)
    kv8, scales, _ = cache(c)
    k, v = (rows_like_a_model(rows, hkv, dim, s + rows, dtype) for s in (1, 2))
    slots = torch.randperm(40 * BS, generator=torch.Generator().manual_seed(3))[:rows]
    c.nsd_kv8_append(kv8, scales, 1, None, gpu(k).reshape(rows, -1), gpu(v), None, gpu(slots))
    assert c.nsd_get_status() == (0, -1)
    b, s = slots // BS, slots % BS
    for j, x in enumerate((k, v)):
        assert_rows(kv8[1, b, j, :, s], scales[1, b, :, j, s], x.double().numpy(), (b, s))
    mark = torch.ones(40, BS, dtype=torch.bool)
    mark[b, s] = False                                     # slots of no row, and the other layer
    assert (kv8[0] == 0xA5).all() and (scales[0] == 0xA5).all()
    assert (kv8[1].permute(0, 3, 1, 2, 4)[gpu(mark)] == 0xA5).all() and (scales[1].permute(0, 3, 1, 2)[gpu(mark)] == 0xA5).all()


@pytest.mark.parametrize("sections,adjacent,cycled", [([64], False, False), ([32], False, False), ([29], False, False), ([24], True, False),
                                                      ([11, 11, 10], True, True), ([16, 24, 24], False, False)])
@pytest.mark.parametrize("dim", [64, 128])
def test_append_turns_q_and_k_as_the_16_bit_append(dim, sections, adjacent, cycled):
    """The same rows through nsd_rope_append: q_out equal bit for bit, and k's codes those of values that differ from the
    exact ones by the rotation's own error at most (a code may then be its neighbour)."""
    heads, hkv, rows = 8, 2, 70
    sections = [s * dim // 128 for s in sections] if dim == 64 else sections
    if cycled:
        sections = [max(sections)] * len(sections) if dim == 128 else [5, 5, 5]
    c = T.context(heads, hkv, dim, num_blocks=8)
    kv8, scales, _ = cache(c)
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn((rows, (heads + 2 * hkv) * dim), generator=g)
    q, k, v = (gpu(qkv[:, a * dim:b * dim]) for a, b in ((0, heads), (heads, heads + hkv), (heads + hkv, heads + 2 * hkv)))
    qkv = gpu(qkv)
    q, k, v = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + hkv) * dim], qkv[:, (heads + hkv) * dim:]
    pos = torch.randint(0, 100000, (len(sections), rows), generator=g, dtype=torch.int32)
    freq = (1e5 ** -torch.linspace(0, 1, sum(sections), dtype=torch.float64)).float()
    slots = torch.randperm(8 * BS, generator=g)[:rows].clone()
    slots[5] = -1                                          # a padding row
    pool = torch.zeros((1, 8, 2, hkv, BS, dim), dtype=torch.bfloat16, device=DEV)
    outs = [torch.full((rows, heads, dim), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    c.nsd_rope_append(pool, 0, q, k, v, outs[0], gpu(pos), sections, gpu(freq), gpu(slots), adjacent=adjacent, cycled=cycled)
    c.nsd_kv8_append(kv8, scales, 0, q, k, v, outs[1], gpu(slots), gpu(pos), sections, gpu(freq), adjacent=adjacent, cycled=cycled)
    assert c.nsd_get_status() == (0, -1)
    assert torch.equal(outs[0], outs[1]) and (outs[1][5] == 3.0).all()
    keep = slots >= 0
    b, s = slots[keep] // BS, slots[keep] % BS
    turned, slack = T.rope_ref(k.cpu().double().reshape(rows, hkv, dim).numpy()[keep], pos.numpy()[:, keep], sections, freq.numpy(), adjacent, cycled)
    got = K.code_values(kv8[0, b, 0, :, s]) * 2.0 ** (scales[0, b, :, 0, s].cpu().numpy()[..., None].astype(np.float64) - 127)
    e = K.exponent(np.abs(turned).max(-1))[..., None].astype(np.float64)
    # half a step of e4m3: 2^-4 of the value, 2^-10 2^e below the normal numbers; the scale may be the next one at an edge
    assert (np.abs(got - turned) <= np.maximum(2.0 ** -4 * np.abs(turned), 2.0 ** (e - 9)) + slack + 1e-30).all()
    same = np.abs(scales[0, b, :, 0, s].cpu().numpy().astype(int) - 127 - e[..., 0])
    assert (same == 0).mean() > 0.99 and same.max() <= 1
    assert_rows(kv8[0, b, 1, :, s], scales[0, b, :, 1, s], v.cpu().double().reshape(rows, hkv, dim).numpy()[keep], (b, s))


def test_append_keeps_what_is_not_a_number_to_itself():
    """NaN and infinities become NaN codes and do not count towards their row's scale; other rows are as ever."""
    c = T.context(8, 2, 128, num_blocks=4)
    kv8, scales, _ = cache(c)
    k, v = rows_like_a_model(10, 2, 128, 5, torch.float32), rows_like_a_model(10, 2, 128, 6, torch.float32)
    k[7, 0, 3], k[7, 1, 100], v[8, 0, :] = float("nan"), float("inf"), float("-inf")
    slots = torch.arange(10) + 20
    c.nsd_kv8_append(kv8, scales, 0, None, gpu(k), gpu(v), None, gpu(slots))
    for j, x in enumerate((k, v)):
        assert_rows(kv8[0, slots // BS, j, :, slots % BS], scales[0, slots // BS, :, j, slots % BS], x.double().numpy(), None)


def test_append_of_unaligned_rows_and_strides():
    """Rows that start off 16 bytes, and slices of a wider projection, come out as copies of them do."""
    c = T.context(8, 2, 64, num_blocks=8)
    wide = torch.randn((50, 300), generator=torch.Generator().manual_seed(7)).to(torch.bfloat16).to(DEV)
    slots = gpu(torch.randperm(8 * BS, generator=torch.Generator().manual_seed(8))[:50])
    got = []
    for k, v in ((wide[:, 3:131], wide[:, 141:269]), (wide[:, 3:131].contiguous(), wide[:, 141:269].contiguous())):
        kv8, scales, _ = cache(c)
        c.nsd_kv8_append(kv8, scales, 0, None, k, v, None, slots)
        got.append((kv8, scales))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_append_q_alone_and_bad_slots():
    c = T.context(8, 2, 64, num_blocks=3)
    kv8, scales, _ = cache(c)
    x = torch.randn((4, 8 * 64), device=DEV)
    out = torch.zeros((4, 8, 64), dtype=torch.bfloat16, device=DEV)
    c.nsd_kv8_append(kv8, scales, 0, x, None, None, out, None)
    assert torch.equal(out, x.to(torch.bfloat16).reshape(4, 8, 64))                           # nothing turns: q is copied
    k = torch.ones((4, 128), device=DEV)
    c.nsd_kv8_append(kv8, scales, 0, None, k, k, None, gpu(torch.tensor([0, 3 * BS, -1, 47])))
    assert c.nsd_get_status() == (6, 1)
    assert (scales[0] != 0xA5).sum() == 2 * 4 and (kv8[0] != 0xA5).sum() == 2 * 4 * 64


# --------------------------------------------------------------------------- whole blocks
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("blocks", [1, 3, 60])
def test_pack_and_unpack(shape, blocks):
    heads, hkv, dim = shape
    total = blocks + 4
    c = T.context(heads, hkv, dim, num_blocks=total, num_layers=3)
    g = torch.Generator().manual_seed(blocks)
    x = rows_like_a_model(3 * total * 2 * BS, hkv, dim, blocks, torch.bfloat16).reshape(3, total, 2, BS, hkv, dim).transpose(3, 4).contiguous()
    pool = gpu(x)
    src, dst = (torch.randperm(total, generator=g)[:blocks].to(torch.int32) for _ in range(2))
    kv8, scales, _ = cache(c)
    c.nsd_kv8_pack(pool, kv8, scales, gpu(src), gpu(dst), layer_begin=1)
    values, e = K.quantise(x.double().numpy()[1:, src.numpy()])
    assert np.array_equal(K.code_values(kv8[1:, dst.long()]), values, equal_nan=True)
    assert np.array_equal(scales[1:, dst.long()].cpu().numpy(), np.swapaxes(e + 127, 2, 3))
    rest = [b for b in range(total) if b not in dst.tolist()]
    assert (kv8[0] == 0xA5).all() and (scales[0] == 0xA5).all() and (kv8[:, rest] == 0xA5).all() and (scales[:, rest] == 0xA5).all()
    # and back, to other blocks
    back = torch.full_like(pool, 9.0)
    to = torch.randperm(total, generator=g)[:blocks].to(torch.int32)
    c.nsd_kv8_unpack(kv8, scales, back, gpu(dst), gpu(to), layer_begin=1, layer_count=2)
    want = torch.from_numpy(values * 2.0 ** e[..., None].astype(np.float64)).to(torch.bfloat16)
    assert torch.equal(back[1:, to.long()].cpu(), want)
    rest = [b for b in range(total) if b not in to.tolist()]
    assert (back[0] == 9.0).all() and (back[:, rest] == 9.0).all()
    assert c.nsd_get_status() == (0, -1)
    # a second trip is exact: the values are on the grid already
    again = cache(c)
    c.nsd_kv8_pack(back, again[0], again[1], gpu(to), gpu(dst), layer_begin=1)
    c.nsd_kv8_unpack(again[0], again[1], pool, gpu(dst), gpu(to), layer_begin=1)
    assert torch.equal(pool[1:, to.long()].cpu(), want)


@pytest.mark.parametrize("dim", [64, 128])
def test_pack_keeps_what_is_not_a_number_to_itself(dim):
    """NaN and infinities become NaN codes and do not count towards their row's scale; rows beside them in a warp, of zeros, of
    subnormal numbers and of the largest ones are as ever."""
    c = T.context(4, 2, dim, num_blocks=3)
    x = rows_like_a_model(3 * 2 * BS, 2, dim, 9, torch.bfloat16).reshape(1, 3, 2, BS, 2, dim).transpose(3, 4).contiguous()
    nan, inf, most, least = float("nan"), float("inf"), torch.finfo(torch.bfloat16).max, 2.0 ** -133
    x[0, 0, 0, 0, 3, 5], x[0, 0, 0, 0, 3, 6] = nan, most
    x[0, 0, 1, 1, 4, dim - 1] = inf
    x[0, 0, 1, 1, 5] = 0.0
    x[0, 0, 1, 1, 6] *= -0.0
    x[0, 1, 0, 0, 0], x[0, 1, 0, 0, 1], x[0, 1, 0, 0, 2], x[0, 1, 0, 0, 4] = -inf, nan, most, -most
    x[0, 1, 1, 0, 15] = torch.arange(dim).to(torch.bfloat16) * least
    x[0, 1, 1, 0, 14] = least
    x[0, 1, 1, 0, 14, 0] = inf
    kv8, scales, _ = cache(c)
    ids = torch.tensor([0, 1], dtype=torch.int32)
    c.nsd_kv8_pack(gpu(x), kv8, scales, gpu(ids), gpu(ids))
    values, e = K.quantise(x.double().numpy()[:, :2])
    assert np.array_equal(K.code_values(kv8[:, :2]), values, equal_nan=True)
    assert np.array_equal(scales[:, :2].cpu().numpy(), np.swapaxes(e + 127, 2, 3))
    assert c.nsd_get_status() == (0, -1) and (kv8[:, 2] == 0xA5).all()


def test_every_code_and_scale_unpacks_to_its_value():
    c = T.context(2, 2, 128, num_blocks=16)
    codes = torch.arange(256, dtype=torch.uint8).repeat(16 * 2 * 2 * BS * 128 // 256).reshape(1, 16, 2, 2, BS, 128).clone()
    scales = torch.arange(256, dtype=torch.uint8).repeat(16 * 2 * 2 * BS // 256).reshape(1, 16, 2, 2, BS)
    pool = torch.zeros((1, 16, 2, 2, BS, 128), dtype=torch.bfloat16, device=DEV)
    ids = gpu(torch.arange(16, dtype=torch.int32))
    c.nsd_kv8_unpack(gpu(codes), gpu(scales), pool, ids, ids)
    two = np.where(np.arange(256) == 255, np.nan, 2.0 ** (np.arange(256) - 127.0))[scales.numpy()].swapaxes(2, 3)
    want = torch.from_numpy(K.grid()[codes.numpy()] * two[..., None]).to(torch.bfloat16)
    got = pool.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_slabs_wrap_and_bad_blocks_are_reported():
    c = T.context(4, 2, 64, num_blocks=6, num_layers=4, num_slabs=2)
    pool = torch.randn((2, 6, 2, 2, BS, 64), device=DEV).to(torch.bfloat16)
    kv8, scales, _ = cache(c)
    c.nsd_kv8_pack(pool, kv8, scales, gpu(torch.tensor([0, 6, 2, 3], dtype=torch.int32)), gpu(torch.tensor([1, 2, -1, 4], dtype=torch.int32)), layer_begin=3, layer_count=1)
    assert c.nsd_get_status()[0] == 6
    assert c.nsd_get_status() == (0, -1)
    assert (kv8[0] == 0xA5).all() and (kv8[1, [0, 2, 3, 5]] == 0xA5).all()
    values, _ = K.quantise(pool[1, [0, 3]].double().cpu().numpy())
    assert np.array_equal(K.code_values(kv8[1, [1, 4]]), values)
    back = torch.zeros_like(pool)
    c.nsd_kv8_unpack(kv8, scales, back, gpu(torch.tensor([1, 7], dtype=torch.int32)), gpu(torch.tensor([5, 0], dtype=torch.int32)), layer_begin=3, layer_count=1)
    assert c.nsd_get_status() == (6, 1)
    assert (back[0] == 0).all() and (back[1, :5] == 0).all() and (back[1, 5] != 0).any()


def test_a_captured_pack_replays_on_new_contents():
    c = T.context(4, 2, 64, num_blocks=6)
    pool = torch.zeros((1, 6, 2, 2, BS, 64), dtype=torch.bfloat16, device=DEV)
    kv8, scales, _ = cache(c)
    ids = gpu(torch.tensor([0, 1, 2], dtype=torch.int32))
    back, to = torch.zeros_like(pool), gpu(torch.tensor([3, 4, 5], dtype=torch.int32))
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            c.nsd_kv8_pack(pool, kv8, scales, ids, ids, stream=s)
            c.nsd_kv8_unpack(kv8, scales, back, ids, to, stream=s)
    for seed in (1, 2):
        pool.copy_(torch.randn(pool.shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        values, e = K.quantise(pool[0, :3].double().cpu().numpy())
        assert torch.equal(back[0, 3:].cpu(), torch.from_numpy(values * 2.0 ** e[..., None]).to(torch.bfloat16))
    del graph


def test_offsets_beyond_32_bits():
    """Blocks whose codes lie more than 2^32 bytes into the cache."""
    c = T.context(8, 8, 128, num_blocks=140000)
    kv8 = torch.zeros((1, 140000, 2, 8, BS, 128), dtype=torch.uint8, device=DEV)
    scales = torch.zeros((1, 140000, 8, 2, BS), dtype=torch.uint8, device=DEV)
    k = torch.randn((3, 8 * 128), generator=torch.Generator().manual_seed(9)).to(DEV)
    slots = torch.tensor([139999 * BS + 15, 131072 * BS, 5])
    c.nsd_kv8_append(kv8, scales, 0, None, k, -k, None, gpu(slots))
    for i, sl in enumerate(slots.tolist()):
        for j, x in enumerate((k, -k)):
            values, e = K.quantise(x[i].double().cpu().numpy().reshape(8, 128))
            assert np.array_equal(K.code_values(kv8[0, sl // BS, j, :, sl % BS]), values)
            assert np.array_equal(scales[0, sl // BS, :, j, sl % BS].cpu().numpy(), e + 127)
    assert int((scales != 0).sum()) == 3 * 16


def test_refusals_launch_nothing():
    import paper_2609_29364_b200 as nsd

    c = T.context(8, 2, 64, num_blocks=4, num_layers=2)
    kv8, scales, _ = cache(c)
    pool = torch.zeros((2, 4, 2, 2, BS, 64), dtype=torch.bfloat16, device=DEV)
    ids, k, slots = gpu(torch.zeros(2, dtype=torch.int32)), torch.zeros((2, 128), device=DEV), gpu(torch.zeros(2, dtype=torch.int64))
    q, pos, freq = torch.zeros((2, 512), device=DEV), gpu(torch.zeros((5, 2), dtype=torch.int32)), torch.ones(64, device=DEV)
    out = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device=DEV)
    before = c.nsd_launch_count()

    def code(call):
        with pytest.raises(nsd.NsdError) as e:
            call()
        return e.value.code

    assert code(lambda: c.nsd_kv8_pack(pool, kv8, scales, ids, ids, 2, 1)) == 2                   # layers
    assert code(lambda: c.nsd_kv8_pack(pool, kv8, scales, ids, ids, -1, 1)) == 2
    assert code(lambda: c.nsd_kv8_unpack(kv8, scales, pool, ids, ids, 1, 2)) == 2
    assert code(lambda: c.nsd_kv8_unpack(kv8.data_ptr() + 8, scales, pool, ids, ids)) == 1        # alignment
    assert code(lambda: c.nsd_kv8_pack(pool, kv8, scales.data_ptr() + 8, ids, ids)) == 1
    assert code(lambda: c.nsd_kv8_append(kv8, scales, 2, None, k, k, None, slots)) == 2           # layer
    assert code(lambda: c.nsd_kv8_append(kv8, scales, 0, None, k, k, None, None)) == 1            # no slots
    assert code(lambda: c.nsd_kv8_append(kv8, scales, 0, None, k.half(), k.half(), None, slots)) == 4
    assert code(lambda: c.nsd_kv8_append(kv8, scales, 0, q, k, k, out, slots, pos, [8] * 5, freq)) == 2
    assert code(lambda: c.nsd_kv8_append(kv8, scales, 0, q, k, k, out, slots, pos[:1], [33], freq)) == 2
    assert code(lambda: c.nsd_kv8_append(kv8, scales, 0, None, k, k, None, slots, adjacent=True)) == 1
    assert code(lambda: c.nsd_kv8_append(kv8.data_ptr() + 4, scales, 0, None, k, k, None, slots)) == 1
    assert code(lambda: c.nsd_rope_append(pool, 0, q, k, k, out, pos[:0], [], freq, slots)) == 2  # the 16-bit append still wants an axis
    c.nsd_kv8_pack(pool, kv8, scales, ids[:0], ids[:0])
    c.nsd_kv8_pack(pool, kv8, scales, ids, ids, 1, 0)
    c.nsd_kv8_append(kv8, scales, 0, None, k[:0], k[:0], None, slots[:0])
    assert c.nsd_launch_count() == before and (kv8 == 0xA5).all()


def test_pack_and_append_on_another_stream_than_the_current_one():
    c = T.context(8, 2, 64, num_blocks=4)
    kv8, scales, _ = cache(c)
    pool = torch.randn((1, 4, 2, 2, BS, 64), device=DEV).to(torch.bfloat16)
    ids = gpu(torch.arange(4, dtype=torch.int32))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    c.nsd_kv8_pack(pool, kv8, scales, ids, ids, stream=s)
    s.synchronize()
    values, _ = K.quantise(pool.double().cpu().numpy())
    assert np.array_equal(K.code_values(kv8), values)
