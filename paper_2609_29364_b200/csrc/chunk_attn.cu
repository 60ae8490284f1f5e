// Attention of a chunk of new tokens over the paged pool: any number of rows per request, from a
// single token to a whole prompt (Section 3, block maps; Appendix G.2, the target's forward pass).
#include <cuda_bf16.h>

#include "nsd_internal.h"

namespace nsd {
namespace {

constexpr int kTileKeys = 128;
constexpr int kRows = 128;                             // stacked rows of a tile
constexpr uint32_t kMagic = 0x4e534443u;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// What a unit costs beside its key tiles (loading Q, filling the pipeline, writing O), in tiles.
constexpr int kUnitCost = 2;

__device__ __forceinline__ void report(int32_t* status, int32_t bit, int r) {
    atomicOr(status, bit);
    atomicCAS(status + 1, 0, r + 1);
}

// ---- plan -------------------------------------------------------------------------------------
// Two kernels.  The first works on every request's units side by side: the visible keys of each
// row and their hull over the unit.  Unit j of request r sits at r + floor(q_indptr[r] / TU) + j,
// an index that needs no prefix sum and leaves at most one gap per request.  The second, one CTA,
// closes the gaps, sums the costs and cuts the whole work -- units x kv heads x key tiles in one
// line -- into n_ctas equal pieces.
struct PlanArgs {
    ChunkPlan p;
    nsd_chunk_masks masks;
    int32_t batch, T, Hkv, bs;
    const int64_t *q_indptr, *kv_indptr;
    const int32_t* ctx_len;
    int32_t* status;
};
__device__ __forceinline__ bool request_ok(const PlanArgs& a, int r) {
    const int64_t s = a.q_indptr[r], e = a.q_indptr[r + 1], c = a.ctx_len[r];
    return s >= 0 && s <= e && e <= a.p.max_rows && c >= 0 && c + (e - s) <= 0x7fffffffll - kTileKeys && a.kv_indptr[r] >= 0 &&
           a.kv_indptr[r] <= a.kv_indptr[r + 1];
}

__global__ void __launch_bounds__(128)
chunk_units_kernel(const PlanArgs a) {
    pdl_release_dependents();
    const int r = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (!request_ok(a, r)) {
        if (blockIdx.y == 0 && threadIdx.x == 0) report(a.status, STATUS_BAD_TOKEN, r);
        return;
    }
    const int TU = 2 * a.T;
    const int64_t s = a.q_indptr[r], e = a.q_indptr[r + 1];
    const int n = (int)(e - s), ctx = a.ctx_len[r], total = ctx + n;
    const int n_units = (n + TU - 1) / TU;
    const int64_t at = r + s / TU, owned = 1 + e / TU - s / TU;
    int prefix = 0;
    if (a.masks.prefix_len) prefix = min(max(a.masks.prefix_len[r], 0), total);
    const int64_t nblk = a.kv_indptr[r + 1] - a.kv_indptr[r];
    for (int64_t j = blockIdx.y * 4 + warp; j < owned; j += gridDim.y * 4) {
        ChunkUnit u{};
        if (j < n_units) {
            const int i0 = (int)j * TU;
            u.ntok = min(TU, n - i0);
            int lo = 0x7fffffff, hi = 0;
            for (int i = i0 + lane; i < i0 + u.ntok; i += 32) {
                const int pos = ctx + i;
                const int stop = max(pos + 1, prefix);
                int first = a.masks.window > 0 ? max(pos + 1 - a.masks.window, 0) : 0;
                if (a.masks.row_first) first = max(first, a.masks.row_first[s + i]);
                const bool any = first < stop;
                a.p.row_lo[s + i] = any ? first : 0;
                a.p.row_hi[s + i] = any ? stop : 0;
                if (any) lo = min(lo, first), hi = max(hi, stop);
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            u.tbl = a.kv_indptr[r];
            u.nblk = (int32_t)min(nblk, (int64_t)0x7fffffff);
            u.row0 = (int32_t)(s + i0);
            u.req = r;
            u.pos0 = ctx + i0;
            u.key_lo = hi > 0 ? lo : 0;
            u.key_hi = hi;
            u.n_tiles = hi > 0 ? (hi + kTileKeys - 1) / kTileKeys - lo / kTileKeys : 0;
            u.first = (int)j;                          // made absolute by the second kernel
            u.last = n_units - 1;
        }
        if (lane == 0) a.p.raw[at + j] = u;
    }
}

constexpr int kSplitThreads = 1024;
constexpr int kCostSmem = 12288;                       // prefix sums the second kernel keeps in shared memory
__global__ void __launch_bounds__(kSplitThreads)
chunk_split_kernel(const PlanArgs a) {
    extern __shared__ int64_t cost_s[];
    __shared__ int64_t warp_cost[kSplitThreads / 32];
    __shared__ int32_t warp_n[kSplitThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    bool ok = true;
    for (int r = tid; r < a.batch; r += kSplitThreads) ok = ok && request_ok(a, r);
    if (tid == 0 && a.batch > 0 && a.q_indptr[0] != 0) {
        report(a.status, STATUS_BAD_TOKEN, 0);
        ok = false;
    }
    ok = __syncthreads_and(ok);
    pdl_wait();                                        // the units of the kernel before are complete
    const int64_t n_raw = ok && a.batch > 0 ? a.batch + a.q_indptr[a.batch] / (2 * a.T) : 0;
    const int64_t per = (n_raw + kSplitThreads - 1) / kSplitThreads;
    const int64_t i0 = min(tid * per, n_raw), i1 = min(i0 + per, n_raw);
    int n_mine = 0;
    int64_t c_mine = 0;
    for (int64_t i = i0; i < i1; ++i)
        if (a.p.raw[i].ntok > 0) ++n_mine, c_mine += a.p.raw[i].n_tiles + kUnitCost;
    int n_inc = n_mine;
    int64_t c_inc = c_mine;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const int vn = __shfl_up_sync(0xffffffffu, n_inc, s);
        const int64_t vc = __shfl_up_sync(0xffffffffu, c_inc, s);
        if (lane >= s) n_inc += vn, c_inc += vc;
    }
    if (lane == 31) warp_n[warp] = n_inc, warp_cost[warp] = c_inc;
    __syncthreads();
    int n_at = n_inc - n_mine, n_units = 0;
    int64_t c_at = c_inc - c_mine, c_all = 0;
    for (int w = 0; w < kSplitThreads / 32; ++w) {
        if (w < warp) n_at += warp_n[w], c_at += warp_cost[w];
        n_units += warp_n[w], c_all += warp_cost[w];
    }
    int64_t* const cost = n_units < kCostSmem ? cost_s : a.p.cost;
    for (int64_t i = i0; i < i1; ++i) {
        ChunkUnit u = a.p.raw[i];
        if (u.ntok <= 0) continue;
        u.last = n_at - u.first + u.last;
        u.first = n_at - u.first;
        a.p.units[n_at] = u;
        cost[n_at] = c_at;
        ++n_at;
        c_at += u.n_tiles + kUnitCost;
    }
    if (tid == 0) {
        cost[n_units] = c_all;
        *a.p.header = ChunkHeader{kMagic, n_units, a.p.max_rows, a.p.n_ctas, 2 * a.T};
    }
    __syncthreads();
    // the line: request by request, kv head by kv head, unit by unit, tile by tile
    for (int c = tid; c <= a.p.n_ctas; c += kSplitThreads) {
        ChunkStart st{n_units, 0, 0, 0};
        const int64_t pos = c_all * a.Hkv * c / a.p.n_ctas;
        if (c < a.p.n_ctas && n_units > 0) {
            int lo = 0, hi = n_units;                  // Hkv * cost[lo] <= pos
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (cost[mid] * a.Hkv <= pos) lo = mid; else hi = mid;
            }
            const int first = a.p.units[lo].first, last = a.p.units[lo].last;
            const int64_t head_cost = cost[last + 1] - cost[first], in_req = pos - cost[first] * a.Hkv;
            st.head = (int)(in_req / head_cost);
            const int64_t rem = in_req % head_cost + cost[first];
            lo = first, hi = last + 1;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (cost[mid] <= rem) lo = mid; else hi = mid;
            }
            st.unit = lo;
            st.tile = (int)max((int64_t)0, rem - cost[lo] - kUnitCost);
        }
        a.p.starts[c] = st;
    }
}

// ---- attention ----------------------------------------------------------------------------------
struct AttnArgs {
    ChunkPlan p;
    const uint16_t *slab, *q;
    int64_t q_stride;
    uint16_t* o;
    float* lse;
    const int32_t* kv_indices;
    float scale, softcap;
    const float* slopes;
    int32_t* status;
    int32_t Hq, Hkv, num_blocks;
};

// A warp per (row, q head): a lane scores one key at a time, the weights are handed round for the
// sum of values, of which a lane owns D / 32 dims.
template <int D>
__global__ void __launch_bounds__(256)
chunk_attn_rows_kernel(const __grid_constant__ AttnArgs a) {
    __shared__ float q_s[8][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (a.p.header->magic != kMagic || a.p.header->max_rows != a.p.max_rows) {
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) report(a.status, STATUS_BAD_TOKEN, -1);
        return;
    }
    const int n_units = a.p.header->n_units, G = a.Hq / a.Hkv, head = blockIdx.y;
    for (int ui = blockIdx.x; ui < n_units; ui += gridDim.x) {
        const ChunkUnit u = a.p.units[ui];
        for (int m = warp; m < u.ntok * G; m += 8) {
            const int row = u.row0 + m / G, h = head * G + m % G;
            const int lo = a.p.row_lo[row], hi = a.p.row_hi[row];
            const int64_t orow = (int64_t)row * a.Hq + h;
            __syncwarp();
            for (int d = lane; d < D; d += 32)
                q_s[warp][d] = __uint_as_float((uint32_t)a.q[row * a.q_stride + h * D + d] << 16);
            __syncwarp();
            const int pos = u.pos0 + row - u.row0;
            float m_run = -INFINITY, l = 0.f, acc[D / 32] = {};
            for (int k0 = lo; k0 < hi; k0 += 32) {
                const int key = k0 + lane;
                float s = -INFINITY;
                int64_t tile = -1;
                if (key < hi) {
                    const int b = key / 16 < u.nblk ? a.kv_indices[u.tbl + key / 16] : -1;
                    if ((uint32_t)b >= (uint32_t)a.num_blocks) {
                        report(a.status, STATUS_BAD_BLOCK, u.req);
                        s = 0.f;
                    } else {
                        tile = ((int64_t)b * 2 * a.Hkv + head) * 16 + key % 16;
                        const uint4* kp = reinterpret_cast<const uint4*>(a.slab + tile * D);
                        tile += 16 * a.Hkv;
                        float d0 = 0.f;
                        for (int c = 0; c < D / 8; ++c) {
                            const uint4 x = kp[c];
                            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                d0 = fmaf(__uint_as_float(w[i] << 16), q_s[warp][c * 8 + 2 * i], d0);
                                d0 = fmaf(__uint_as_float(w[i] & 0xffff0000u), q_s[warp][c * 8 + 2 * i + 1], d0);
                            }
                        }
                        s = d0;
                    }
                    s *= a.scale;
                    if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
                    if (a.slopes) s += a.slopes[h] * (float)(key - pos);
                }
                float mx = s;
                for (int i = 16; i; i >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, i));
                const float m_new = fmaxf(m_run, mx);
                const float f = m_run == -INFINITY ? 0.f : expf(m_run - m_new);
                const float p = key < hi ? expf(s - m_new) : 0.f;
                m_run = m_new;
                l = l * f + p;
                for (int i = 0; i < D / 32; ++i) acc[i] *= f;
                for (int j = 0; j < 32 && k0 + j < hi; ++j) {
                    const float pj = __shfl_sync(0xffffffffu, p, j);
                    const int64_t t = __shfl_sync(0xffffffffu, tile, j);
                    if (t >= 0)
                        for (int i = 0; i < D / 32; ++i) acc[i] = fmaf(pj, __uint_as_float((uint32_t)a.slab[t * D + lane + 32 * i] << 16), acc[i]);
                }
            }
            for (int i = 16; i; i >>= 1) l += __shfl_xor_sync(0xffffffffu, l, i);
            const float inv = l > 0.f ? 1.f / l : 0.f;
            for (int i = 0; i < D / 32; ++i) {
                const __nv_bfloat16 v = __float2bfloat16(acc[i] * inv);
                a.o[orow * D + lane + 32 * i] = *reinterpret_cast<const uint16_t*>(&v);
            }
            if (a.lse && lane == 0) a.lse[orow] = m_run == -INFINITY ? -INFINITY : m_run + logf(l);
        }
    }
}

}  // namespace

size_t chunk_plan_layout(ChunkPlan* p, void* base, const Shape& s, int32_t max_batch, int64_t max_rows, int32_t n_sms) {
    const int64_t T = kRows / (s.Hq / s.Hkv);
    const int64_t max_units = max_batch + max_rows / (2 * T) + 2;
    size_t off = 0;
    char* const b = static_cast<char*>(base);
    auto part = [&](size_t bytes) {
        char* const at = b + off;
        off = (off + bytes + 255) / 256 * 256;
        return static_cast<void*>(at);
    };
    ChunkPlan q{};
    q.header = static_cast<ChunkHeader*>(part(sizeof(ChunkHeader)));
    q.starts = static_cast<ChunkStart*>(part((n_sms + 1) * sizeof(ChunkStart)));
    q.raw = static_cast<ChunkUnit*>(part(max_units * sizeof(ChunkUnit)));
    q.units = static_cast<ChunkUnit*>(part(max_units * sizeof(ChunkUnit)));
    q.cost = static_cast<int64_t*>(part((max_units + 1) * sizeof(int64_t)));
    q.row_lo = static_cast<int32_t*>(part(max_rows * sizeof(int32_t)));
    q.row_hi = static_cast<int32_t*>(part(max_rows * sizeof(int32_t)));
    q.part_ml = static_cast<float*>(part(2ull * n_sms * 2 * kRows * 2 * sizeof(float)));
    q.part_acc = static_cast<float*>(part(2ull * n_sms * 2 * kRows * s.D * sizeof(float)));
    q.max_rows = max_rows;
    q.max_units = max_units;
    q.n_ctas = n_sms;
    if (p) *p = q;
    return off;
}

cudaError_t chunk_attn_init() {
    return cudaFuncSetAttribute(chunk_split_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kCostSmem * (int)sizeof(int64_t));
}

cudaError_t launch_chunk_plan(const ChunkPlan& p, const Shape& s, int32_t batch, const int64_t* q_indptr, const int32_t* ctx_len,
                              const int64_t* kv_indptr, const nsd_chunk_masks& masks, int32_t* status, cudaStream_t stream) {
    const int T = kRows / (s.Hq / s.Hkv);
    const PlanArgs a{p, masks, batch, T, s.Hkv, s.bs, q_indptr, kv_indptr, ctx_len, status};
    if (batch > 0) {
        // a warp per unit: enough of them for the average request, at most 64 CTAs for the longest
        const int64_t units = p.max_rows / (2 * T) / 4 + 1;
        const unsigned slices = (unsigned)(units < 64 ? units : 64);
        chunk_units_kernel<<<dim3((unsigned)batch, slices), 128, 0, stream>>>(a);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    const int64_t most = p.max_units + 1;
    const size_t smem = (size_t)(most < kCostSmem ? most : kCostSmem) * sizeof(int64_t);
    return launch_kernel(chunk_split_kernel, dim3(1), dim3(kSplitThreads), smem, stream, batch > 0, a);
}

cudaError_t launch_chunk_attn(const ChunkPlan& p, const ChunkAttnLaunch& l, cudaStream_t stream, int* launched) {
    const AttnArgs a{p, l.slab, l.q, l.q_stride, l.o, l.lse, l.kv_indices, l.scale, l.softcap, l.slopes, l.status, l.shape.Hq, l.shape.Hkv, l.shape.num_blocks};
    const dim3 grid((unsigned)(p.max_units < 4096 ? p.max_units : 4096), l.shape.Hkv);
    if (l.shape.D == 128) chunk_attn_rows_kernel<128><<<grid, 256, 0, stream>>>(a);
    else chunk_attn_rows_kernel<64><<<grid, 256, 0, stream>>>(a);
    *launched = 1;
    return cudaGetLastError();
}

}  // namespace nsd
