// Whole blocks between the bf16 pool and the 8-bit cache: parking a request that leaves the worker in
// half its bytes, and fetching it back (the block moves of Section 3 and Appendix E.2).
#include "kv8_codec.h"
#include "nsd_internal.h"

namespace nsd {
namespace {

// A (layer, pair, K|V, kv head) tile is 16 rows of D values in the pool, 16 x D codes and 16 scale
// bytes in the cache.  A thread holds eight values of a row -- 16 bytes in bf16, 8 in codes -- so
// both sides move in whole lines; the D / 8 lanes of a row find its maximum by shuffles.  Nothing
// is read twice, so HBM bounds it: 3 D + 1 bytes per row.  The grid is (pairs, tiles of a block,
// layers), so that no thread divides to find its place (with one flat index, taken apart by three
// 64-bit divisions, 2048 blocks of 4 layers took 336 and 288 us), and the loads of kAhead tiles are
// under way together (4: 162 and 135 us, 16: 180 and 130).  A CTA takes one pair (16 CTAs per SM
// that take several: 151 and 137).  2048 blocks of 4 layers (8 kv heads of 128) 140 us packed = 5.8
// TB/s (149 with a row's maximum of floats instead of packed bits), 130 unpacked = 6.2 TB/s; 67
// blocks 6.8 and 5.3 us.
constexpr int kBsP = 16;
constexpr int kThreadsP = 256;
constexpr int kAhead = 8;

__device__ __forceinline__ void report(int32_t* status, int64_t j) {
    atomicOr(status, STATUS_BAD_BLOCK);
    atomicCAS(status + 1, 0, (int32_t)j + 1);
}

template <int D, bool PACK>
__global__ void __launch_bounds__(kThreadsP)
kv8_copy_kernel(const __grid_constant__ Kv8Copy c) {
    constexpr int kLanes = D / 8;                      // lanes of a row
    constexpr int kTileThreads = kBsP * kLanes;        // threads of a tile: whole warps, which so agree on what they have
    constexpr int kPerCta = kThreadsP / kTileThreads;
    const int tiles = 2 * c.shape.Hkv, mine = threadIdx.x / kTileThreads;
    const int in = threadIdx.x % kTileThreads, row = in / kLanes, d0 = in % kLanes * 8;
    const uint32_t pair = blockIdx.x;
    const int src = __ldg(c.src + pair), dst = __ldg(c.dst + pair);
    if ((uint32_t)src >= (uint32_t)c.shape.num_blocks || (uint32_t)dst >= (uint32_t)c.shape.num_blocks) {
        if (blockIdx.y == 0 && blockIdx.z == 0 && threadIdx.x == 0) report(c.status, pair);
        return;
    }
    for (int l = blockIdx.z; l < c.layer_count; l += gridDim.z) {
        const int64_t slab = (int64_t)((c.layer_begin + l) % c.num_slabs) * c.shape.num_blocks;
        const int64_t tile16 = (slab + (PACK ? src : dst)) * tiles, tile8 = (slab + (PACK ? dst : src)) * tiles;
        for (int t0 = blockIdx.y * (kPerCta * kAhead) + mine; t0 < tiles; t0 += gridDim.y * (kPerCta * kAhead)) {
            uint16_t* const at16 = c.pool + ((tile16 + t0) * kBsP + row) * D + d0;
            uint8_t* const at8 = c.codes + ((tile8 + t0) * kBsP + row) * D + d0;
            constexpr int kStep = kPerCta * kBsP * D;
            auto scale_at = [&](int i) {           // [kv head][K|V][16]
                const int t = t0 + i * kPerCta, kv = t >= c.shape.Hkv;
                return c.scales + (tile8 + 2 * (t - (kv ? c.shape.Hkv : 0)) + kv) * kBsP + row;
            };
            if constexpr (PACK) {
                uint4 w[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (t0 + i * kPerCta < tiles) w[i] = __ldcs(reinterpret_cast<const uint4*>(at16 + i * kStep));
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (t0 + i * kPerCta >= tiles) break;
                    const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                    // magnitudes order as their bits do, two at a time
                    uint32_t top = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = __vmaxu2(top, v[j] & 0x7fff7fffu);
#pragma unroll
                    for (int s = kLanes / 2; s > 0; s >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, s));
                    top = max(top & 0xffffu, top >> 16);
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(v[j] << 16), x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
                    if (__any_sync(0xffffffffu, top >= 0x7f80u)) {                      // no number in a row of the warp: the largest of the others
                        float m = 0.f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) m = fmaxf(m, kv8_magnitude(x[j])), x[j] = fmaf(x[j], 0.f, x[j]);
#pragma unroll
                        for (int s = kLanes / 2; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
                        top = __float_as_uint(m) >> 16;
                    }
                    const uint32_t byte = kv8_scale_byte(__uint_as_float(top << 16));
                    const float inv = kv8_inverse(byte);
                    uint2 out;
                    out.x = kv8_codes2_finite(x[0], x[1], inv) | kv8_codes2_finite(x[2], x[3], inv) << 16;
                    out.y = kv8_codes2_finite(x[4], x[5], inv) | kv8_codes2_finite(x[6], x[7], inv) << 16;
                    *reinterpret_cast<uint2*>(at8 + i * kStep) = out;
                    if (d0 == 0) *scale_at(i) = (uint8_t)byte;
                }
            } else {
                uint2 w[kAhead];
                uint32_t byte[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i)
                    if (t0 + i * kPerCta < tiles) w[i] = __ldcs(reinterpret_cast<const uint2*>(at8 + i * kStep)), byte[i] = *scale_at(i);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (t0 + i * kPerCta >= tiles) break;
                    const float s = kv8_scale(byte[i]);
                    uint32_t out[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 v = kv8_values2((j < 2 ? w[i].x : w[i].y) >> (16 * (j & 1)));
                        const __nv_bfloat162 b = __floats2bfloat162_rn(v.x * s, v.y * s);
                        out[j] = *reinterpret_cast<const uint32_t*>(&b);
                    }
                    *reinterpret_cast<uint4*>(at16 + i * kStep) = make_uint4(out[0], out[1], out[2], out[3]);
                }
            }
        }
    }
}

template <bool PACK>
cudaError_t launch(const Kv8Copy& c, cudaStream_t stream) {
    if (c.layer_count == 0 || c.n_blocks == 0) return cudaSuccess;
    const int batch = kAhead * (c.shape.D == 128 ? 1 : 2), y = (2 * c.shape.Hkv + batch - 1) / batch, z = c.layer_count < 64 ? c.layer_count : 64;
    const dim3 grid((unsigned)c.n_blocks, (unsigned)(y < 64 ? y : 64), (unsigned)z);
    if (c.shape.D == 128) kv8_copy_kernel<128, PACK><<<grid, kThreadsP, 0, stream>>>(c);
    else kv8_copy_kernel<64, PACK><<<grid, kThreadsP, 0, stream>>>(c);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_pack(const Kv8Copy& c, cudaStream_t stream) { return launch<true>(c, stream); }
cudaError_t launch_kv8_unpack(const Kv8Copy& c, cudaStream_t stream) { return launch<false>(c, stream); }

}  // namespace nsd
