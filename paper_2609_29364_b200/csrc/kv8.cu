// Whole blocks between the bf16 pool and the 8-bit cache: parking a request that leaves the worker in
// half its bytes, and fetching it back (the block moves of Section 3 and Appendix E.2).
#include "kv8_codec.h"
#include "nsd_internal.h"

namespace nsd {
namespace {

// A (layer, pair, K|V, kv head) tile is 16 rows of D values in the pool, 16 x D codes and 16 scale
// bytes in the cache.  A thread holds eight values of a row -- 16 bytes in bf16, 8 in codes -- so
// both sides move in whole lines; the D / 8 lanes of a row find its maximum by shuffles.  Nothing
// is read twice, so HBM bounds it: 3 D + 1 bytes per row.  The loads of kAhead tiles are under way
// together; a thread that had one would leave the memory idle between its load and its stores.
constexpr int kBsP = 16;
constexpr int kThreadsP = 256;
constexpr int kAhead = 4;

__device__ __forceinline__ void report(int32_t* status, int64_t j) {
    atomicOr(status, STATUS_BAD_BLOCK);
    atomicCAS(status + 1, 0, (int32_t)j + 1);
}

// Where a tile lies in the pool and in the cache; pool is -1 for a pair that names a block outside.
struct Tile {
    int64_t pool, code, scale;                         // pool and code in tiles of 16 x D, scale in bytes
};
template <bool PACK>
__device__ __forceinline__ Tile tile_at(const Kv8Copy& c, int64_t t) {
    const int per = 2 * c.shape.Hkv, part = (int)(t % per), kv = part / c.shape.Hkv, head = part % c.shape.Hkv;
    const int64_t pair = t / per % c.n_blocks;
    const int64_t slab = (c.layer_begin + t / per / c.n_blocks) % c.num_slabs * c.shape.num_blocks;
    const int src = c.src[pair], dst = c.dst[pair];
    if ((uint32_t)src >= (uint32_t)c.shape.num_blocks || (uint32_t)dst >= (uint32_t)c.shape.num_blocks) {
        if (part == 0 && threadIdx.x % 32 == 0) report(c.status, pair);
        return Tile{-1, -1, -1};
    }
    const int64_t block16 = slab + (PACK ? src : dst), block8 = slab + (PACK ? dst : src);
    return Tile{block16 * per + part, block8 * per + part, (block8 * per + head * 2 + kv) * kBsP};
}

template <int D, bool PACK>
__global__ void __launch_bounds__(kThreadsP)
kv8_copy_kernel(const __grid_constant__ Kv8Copy c) {
    constexpr int kLanes = D / 8;                      // lanes of a row
    constexpr int kTileThreads = kBsP * kLanes;        // threads of a tile
    constexpr int kPerCta = kThreadsP / kTileThreads;
    const int64_t tiles = (int64_t)c.layer_count * c.n_blocks * 2 * c.shape.Hkv;
    const int in = threadIdx.x % kTileThreads, row = in / kLanes, d0 = in % kLanes * 8;
    const int64_t step = (int64_t)gridDim.x * kPerCta;
    for (int64_t t = blockIdx.x * (int64_t)kPerCta + threadIdx.x / kTileThreads; t < tiles; t += step * kAhead) {
        Tile at[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) at[i] = t + i * step < tiles ? tile_at<PACK>(c, t + i * step) : Tile{-1, -1, -1};
        if constexpr (PACK) {
            uint4 w[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (at[i].pool >= 0) w[i] = __ldcs(reinterpret_cast<const uint4*>(c.pool + (at[i].pool * kBsP + row) * D + d0));
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                // a tile's threads are whole warps, so a warp agrees on what it has
                if (at[i].pool < 0) continue;
                const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                float x[8], top = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[2 * j] = __uint_as_float(v[j] << 16), x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
                    top = fmaxf(top, fmaxf(kv8_magnitude(x[2 * j]), kv8_magnitude(x[2 * j + 1])));
                }
#pragma unroll
                for (int s = kLanes / 2; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
                const uint32_t byte = kv8_scale_byte(top);
                const float inv = kv8_inverse(byte);
                uint2 out;
                out.x = kv8_codes2(x[0], x[1], inv) | kv8_codes2(x[2], x[3], inv) << 16;
                out.y = kv8_codes2(x[4], x[5], inv) | kv8_codes2(x[6], x[7], inv) << 16;
                __stcs(reinterpret_cast<uint2*>(c.codes + (at[i].code * kBsP + row) * D + d0), out);
                if (d0 == 0) c.scales[at[i].scale + row] = (uint8_t)byte;
            }
        } else {
            uint2 w[kAhead];
            uint32_t byte[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (at[i].pool >= 0) {
                    w[i] = __ldcs(reinterpret_cast<const uint2*>(c.codes + (at[i].code * kBsP + row) * D + d0));
                    byte[i] = c.scales[at[i].scale + row];
                }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (at[i].pool < 0) continue;
                const float s = kv8_scale(byte[i]);
                uint32_t out[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 v = kv8_values2((j < 2 ? w[i].x : w[i].y) >> (16 * (j & 1)));
                    const __nv_bfloat162 b = __floats2bfloat162_rn(v.x * s, v.y * s);
                    out[j] = *reinterpret_cast<const uint32_t*>(&b);
                }
                __stcs(reinterpret_cast<uint4*>(c.pool + (at[i].pool * kBsP + row) * D + d0), make_uint4(out[0], out[1], out[2], out[3]));
            }
        }
    }
}

template <bool PACK>
cudaError_t launch(const Kv8Copy& c, cudaStream_t stream) {
    const int64_t tiles = (int64_t)c.layer_count * c.n_blocks * 2 * c.shape.Hkv;
    if (tiles == 0) return cudaSuccess;
    const int per_cta = c.shape.D == 128 ? 1 : 2;
    const int64_t want = (tiles + per_cta - 1) / per_cta, most = 8LL * c.n_sms;
    const unsigned grid = (unsigned)(want < most ? want : most);
    if (c.shape.D == 128) kv8_copy_kernel<128, PACK><<<grid, kThreadsP, 0, stream>>>(c);
    else kv8_copy_kernel<64, PACK><<<grid, kThreadsP, 0, stream>>>(c);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_pack(const Kv8Copy& c, cudaStream_t stream) { return launch<true>(c, stream); }
cudaError_t launch_kv8_unpack(const Kv8Copy& c, cudaStream_t stream) { return launch<false>(c, stream); }

}  // namespace nsd
