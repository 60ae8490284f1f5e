// What precedes the attention of a chunk of new tokens: block tables and slot maps from request
// lengths, and rotary positions fused with the append into the paged pool (Section 3, "KV cache
// organization"; the free list of a bank, Appendix E.2).
#include <cuda_bf16.h>

#include "nsd_internal.h"

namespace nsd {
namespace {

// ---- block tables ---------------------------------------------------------------------------
// Every output position is computed on its own: the flat entry e of kv_indices (or the flat row i
// of slot_map) finds its request by a search in the prefix sums and reads the one block id it
// needs.  So the work is spread evenly however unequal the requests are (one prompt of 100 000
// tokens beside 500 single tokens), and no CTA waits for another: each forms the prefix sums of
// the whole batch for itself in shared memory (12 bytes per request read from L2), which costs
// less than a second launch.  What bounds it is latency: launch, lengths, sums, one search, one
// block id, stores.  The grid follows the buffers, whose CTAs behind the batch's last position form
// the sums for nothing: 512 requests in buffers of their size 4.3 us, of 262 144 entries 8.0, of 4 194 304 86.
constexpr int kTablesThreads = 256;
constexpr int kTablesPerCta = 256;                // flat positions per CTA: one per thread (512 requests, 72 000 entries: 4.4 us; two per thread 5.2, four 7.4)
constexpr int kBsT = 16;

struct TablesArgs {
    int32_t batch, num_blocks;
    const int32_t *ctx_len, *new_len, *n_held, *free_blocks;
    int32_t* held;
    int64_t held_stride, n_free;
    const int64_t* free_begin;
    int64_t max_entries, max_rows;
    int64_t *kv_indptr, *q_indptr, *free_end;
    int32_t* kv_indices;
    int64_t* slot_map;
    int32_t *positions, *row_req, *n_held_new, *status;
};

struct Need {
    int32_t entries, rows, take, ctx, held;
    bool ok;
};
__device__ __forceinline__ Need need_of(const TablesArgs& a, int r) {
    const int64_t c = a.ctx_len[r], n = a.new_len[r], h = a.n_held[r];
    const int64_t need = (c + n + kBsT - 1) / kBsT;
    const bool ok = c >= 0 && n >= 0 && c + n <= 0x7fffffffll - kBsT && need <= a.held_stride && h >= (c + kBsT - 1) / kBsT && h <= a.held_stride;
    return ok ? Need{(int32_t)need, (int32_t)n, (int32_t)(need > h ? need - h : 0), (int32_t)c, (int32_t)h, true} : Need{0, 0, 0, 0, 0, false};
}
__device__ __forceinline__ void report(int32_t* status, int32_t bit, int r) {
    atomicOr(status, bit);
    atomicCAS(status + 1, 0, r + 1);
}
// The request that owns flat position x: the last r with p[r] <= x (requests without positions are skipped).
__device__ __forceinline__ int owner_of(const int32_t* p, int batch, int32_t x) {
    int lo = 0, hi = batch;                        // p[lo] <= x < p[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kTablesThreads)
block_tables_kernel(const TablesArgs a) {
    // per request: prefix sums of table entries, rows and blocks taken (one more each), committed tokens, blocks held
    extern __shared__ int32_t pre[];
    __shared__ int64_t warp_sum[3][kTablesThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int32_t *const kvp = pre, *const qp = pre + a.batch + 1, *const tp = qp + a.batch + 1, *const ctx = tp + a.batch + 1, *const held_n = ctx + a.batch;
    const int per = (a.batch + kTablesThreads - 1) / kTablesThreads;
    const int r0 = min(tid * per, a.batch), r1 = min(r0 + per, a.batch);
    int64_t fb = a.free_begin ? *a.free_begin : 0;
    int64_t mine[3] = {0, 0, 0};
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
        const Need d = need_of(a, r);
        kvp[r] = d.entries, qp[r] = d.rows, tp[r] = d.take;            // for the moment the request's own
        ctx[r] = d.ctx, held_n[r] = d.held;
        mine[0] += d.entries, mine[1] += d.rows, mine[2] += d.take;
        if (!d.ok && blockIdx.x == 0) report(a.status, STATUS_BAD_TOKEN, r);
    }
    int64_t inc[3] = {mine[0], mine[1], mine[2]};
#pragma unroll
    for (int s = 1; s < 32; s <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int64_t v = __shfl_up_sync(0xffffffffu, inc[k], s);
            if (lane >= s) inc[k] += v;
        }
    if (lane == 31)
        for (int k = 0; k < 3; ++k) warp_sum[k][warp] = inc[k];
    __syncthreads();
    int64_t at[3], total[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        int64_t before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kTablesThreads / 32; ++w) {
            if (w < warp) before += warp_sum[k][w];
            all += warp_sum[k][w];
        }
        at[k] = before + inc[k] - mine[k];
        total[k] = all;
    }
    // positions past 2^31 are past every buffer: the sums may saturate there
    auto sat = [](int64_t v) { return (int32_t)(v > 0x7fffffffll ? 0x7fffffffll : v); };
    for (int r = r0; r < r1; ++r) {
        const int32_t e = kvp[r], n = qp[r], t = tp[r];
        kvp[r] = sat(at[0]), qp[r] = sat(at[1]), tp[r] = sat(at[2]);
        at[0] += e, at[1] += n, at[2] += t;
    }
    if (tid == 0) kvp[a.batch] = sat(total[0]), qp[a.batch] = sat(total[1]), tp[a.batch] = sat(total[2]);
    __syncthreads();

    if (fb < 0 || fb > a.n_free) {
        if (blockIdx.x == 0 && tid == 0) report(a.status, STATUS_BAD_BLOCK, -1);
        fb = a.n_free;
    }
    // What a request takes has to be in its table and in held, or the step would store to blocks that it does not read and the
    // next one would trust entries that nobody wrote: from the table entry max_entries on nothing is taken.  Takes are in
    // the order of the entries, so what is left out is the end of the takes, as it is where the free list runs out.
    auto taken = [&](int r) -> int32_t {
        const int64_t take = tp[r + 1] - tp[r], left = a.n_free - fb - tp[r], fit = a.max_entries - kvp[r] - held_n[r];
        return (int32_t)max((int64_t)0, min(take, min(left, fit)));
    };
    // block k of request r's table: its own or one from the free list, -1 where none is taken
    auto block_of = [&](int r, int k) -> int32_t {
        const int held = held_n[r];
        if (k < held) return a.held[(int64_t)r * a.held_stride + k];
        return k - held < taken(r) ? a.free_blocks[fb + tp[r] + (k - held)] : -1;
    };
    // flat position x is both a table entry and a row: the searches and loads of a thread's positions run side by side
    constexpr int kEach = kTablesPerCta / kTablesThreads;
    const int64_t x0 = (int64_t)blockIdx.x * kTablesPerCta + tid;
    int er[kEach], rr[kEach], pos[kEach];
    int32_t eid[kEach], rid[kEach];
    const int64_t n_entries = min((int64_t)kvp[a.batch], a.max_entries), n_rows = min((int64_t)qp[a.batch], a.max_rows);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int64_t x = x0 + u * kTablesThreads;
        er[u] = rr[u] = eid[u] = rid[u] = -1, pos[u] = 0;
        if (x < n_entries) {
            er[u] = owner_of(kvp, a.batch, (int32_t)x);
            eid[u] = block_of(er[u], (int)x - kvp[er[u]]);
        }
        if (x < n_rows) {
            rr[u] = owner_of(qp, a.batch, (int32_t)x);
            pos[u] = ctx[rr[u]] + (int32_t)x - qp[rr[u]];
            rid[u] = block_of(rr[u], pos[u] / kBsT);
        }
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int64_t x = x0 + u * kTablesThreads;
        if (er[u] >= 0) {
            const int r = er[u], k = (int)x - kvp[r];
            a.kv_indices[x] = eid[u];
            if ((uint32_t)eid[u] >= (uint32_t)a.num_blocks) report(a.status, STATUS_BAD_BLOCK, r);
            // a bad id of the free list counts as taken, so it is recorded too: the next step reports it again
            if (k >= held_n[r] && k - held_n[r] < taken(r)) a.held[(int64_t)r * a.held_stride + k] = eid[u];
        }
        if (x < a.max_rows) {
            if (a.slot_map) a.slot_map[x] = (uint32_t)rid[u] < (uint32_t)a.num_blocks ? (int64_t)rid[u] * kBsT + pos[u] % kBsT : -1;
            if (a.positions) a.positions[x] = pos[u];
            if (a.row_req) a.row_req[x] = rr[u];
        }
    }
    // the per-request outputs, shared out over the CTAs
    for (int r = blockIdx.x * kTablesThreads + tid; r <= a.batch; r += gridDim.x * kTablesThreads) {
        a.kv_indptr[r] = min((int64_t)kvp[r], a.max_entries);           // a reader of the tables stays inside them
        a.q_indptr[r] = qp[r];
        if (r == a.batch) {
            // the request with the first entry that does not fit is the last to take anything
            const int last = r > 0 ? (kvp[r] > a.max_entries ? owner_of(kvp, r, (int32_t)a.max_entries) : r - 1) : 0;
            *a.free_end = fb + (r > 0 ? min((int64_t)tp[last] + taken(last), max(a.n_free - fb, (int64_t)0)) : 0);
            if (kvp[r] > a.max_entries || (qp[r] > a.max_rows && (a.slot_map || a.positions || a.row_req))) report(a.status, STATUS_BAD_TOKEN, -1);
        } else {
            a.n_held_new[r] = a.n_held[r] + taken(r);
        }
    }
}

// ---- rotary positions + append ----------------------------------------------------------------
// (a, b) -> (a cos - b sin, b cos + a sin) for the pairs of every q and k head of a row, q to its
// buffer, k and v to the pool: each value is read once and written once, so the bound is HBM.
// The angle is position * frequency with a position up to millions and a result needed modulo
// 2 pi: it is formed in turns and reduced in 64 bits, then sincospi in 32.
// A warp owns a row (or a share of its heads, when there are few rows: the sines are then formed
// again, which costs less than idle SMs).  A lane keeps 16 dims of a head -- two 16-byte pieces,
// both members of eight pairs -- and meets the same eight pairs in every head it visits, so
// sines and cosines stay in registers: they are formed once per row, two pairs per lane, and
// handed round by shuffles.  Four heads per lane (two in fp32) are loaded ahead, the first of them
// while the sines are formed: 8192 rows of 32 + 8 + 8 heads of 128 in bf16 take 36.5 us, 5.5 TB/s
// (57 us one head at a time); 320 rows 4.4 us, of which most is the launch and one trip to HBM.  Pair by pair
// (below) nothing is loaded ahead and accesses are of two bytes: 8192 rows with 29 pairs 81 us, unaligned ones 103.
struct RopeArgs {
    int64_t n_rows;
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride, qo_stride;
    uint16_t* q_out;
    uint16_t* slab;
    const int32_t* positions;
    const float* inv_freq;
    const int64_t* slot_map;
    int32_t* status;
    int32_t Hq, Hkv, num_blocks, pairs, adjacent;
    int32_t log2_parts;                            // warps per row
    int32_t hq0;                                   // first head of the walk: 0, or Hq when there is no q
    int32_t heads;                                 // one past its last: Hq + 2 Hkv, or Hq without k and v
    uint8_t axis[64];
};

// 16 dims of a head as they lie in memory: eight at d0, eight at d1.
template <typename T> struct Dims;
template <> struct Dims<float> {
    float4 v[4];
    __device__ __forceinline__ void load(const float* p, int d0, int d1) {
        v[0] = __ldcs(reinterpret_cast<const float4*>(p + d0)), v[1] = __ldcs(reinterpret_cast<const float4*>(p + d0) + 1);
        v[2] = __ldcs(reinterpret_cast<const float4*>(p + d1)), v[3] = __ldcs(reinterpret_cast<const float4*>(p + d1) + 1);
    }
    __device__ __forceinline__ void get(float* x) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * i] = v[i].x, x[4 * i + 1] = v[i].y, x[4 * i + 2] = v[i].z, x[4 * i + 3] = v[i].w;
    }
};
template <> struct Dims<__nv_bfloat16> {
    uint4 v[2];
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int d0, int d1) {
        v[0] = __ldcs(reinterpret_cast<const uint4*>(p + d0)), v[1] = __ldcs(reinterpret_cast<const uint4*>(p + d1));
    }
    __device__ __forceinline__ void get(float* x) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) x[8 * i + 2 * j] = __uint_as_float(w[j] << 16), x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
};
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void store8(uint16_t* p, const float* x) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}

// VEC: every row of q, k, v and q_out starts on 16 bytes and the members of a pair sit at the same place of two pieces
// (adjacent pairs, or pairs a multiple of eight apart): 16-byte loads and stores.  Otherwise pair by pair.
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(256)
rope_append_kernel(const __grid_constant__ RopeArgs a) {
    constexpr int kUnits = D / 16;                 // a head in units of two 16-byte pieces
    constexpr int kHeads = 32 / kUnits;            // heads a warp has under way
    const int lane = threadIdx.x & 31;
    const int64_t w = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    const int64_t row = w >> a.log2_parts;
    const int part = (int)(w & ((1 << a.log2_parts) - 1));
    if (row >= a.n_rows) return;
    const int64_t slot = a.slot_map ? a.slot_map[row] : 0;
    if (slot < 0) return;                          // a padding row
    const bool stored = slot < (int64_t)a.num_blocks * kBsT;
    if (!stored && lane == 0 && part == 0) report(a.status, STATUS_BAD_BLOCK, (int)row);
    const int Hk0 = a.Hq, Hv0 = a.Hq + a.Hkv;
    const int per = (a.heads - a.hq0 + (1 << a.log2_parts) - 1) >> a.log2_parts;
    const int h_begin = a.hq0 + part * per, h_end = min(h_begin + per, a.heads);
    auto source = [&](int h) -> const T* {
        if (h < Hk0) return static_cast<const T*>(a.q) + row * a.q_stride + h * D;
        if (h < Hv0) return static_cast<const T*>(a.k) + row * a.k_stride + (h - Hk0) * D;
        return static_cast<const T*>(a.v) + row * a.v_stride + (h - Hv0) * D;
    };
    // tile of (block, K|V, kv head): block * 2 Hkv + K|V * Hkv + head = block * 2 Hkv + (h - Hq)
    uint16_t* const kv_at = a.slab + (((slot / kBsT) * 2 * a.Hkv - Hk0) * kBsT + slot % kBsT) * D;
    auto target = [&](int h) -> uint16_t* {
        if (h < Hk0) return a.q_out + row * a.qo_stride + h * D;
        return stored ? kv_at + (int64_t)h * (kBsT * D) : nullptr;
    };
    // adjacent: a unit's 16 dims are its eight pairs.  Apart: dims p and p + pairs for the units that turn, and the dims
    // from 2 pairs on, 16 at a time, for the rest.
    const int u = lane % kUnits;
    const int d0 = a.adjacent ? u * 16 : (u * 8 < a.pairs ? u * 8 : 2 * a.pairs + (u - a.pairs / 8) * 16);
    const int d1 = a.adjacent || u * 8 >= a.pairs ? d0 + 8 : d0 + a.pairs;
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2; // heads per lane whose loads are in flight together
    Dims<T> now[kAhead];
    int h0 = h_begin + lane / kUnits;
    auto fetch = [&](Dims<T>* to, int h) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (h + j * kHeads < h_end) to[j].load(source(h + j * kHeads), d0, d1);
    };
    if constexpr (VEC) fetch(now, h0);             // under way while the sines are formed
    // two pairs per lane (one where a head has 32): 2 lane, 2 lane + 1
    constexpr int kMine = D / 64;
    float cs[kMine], sn[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int p = lane * kMine + i;
        cs[i] = 1.f, sn[i] = 0.f;
        if (p < a.pairs) {
            const double turns = (double)a.positions[(int64_t)a.axis[p] * a.n_rows + row] * ((double)a.inv_freq[p] * 0.15915494309189533577);
            sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
        }
    }
    if constexpr (VEC) {
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = u * 8 + i;               // sits with lane p / kMine
            c[i] = __shfl_sync(0xffffffffu, cs[i % kMine], p / kMine);
            s[i] = __shfl_sync(0xffffffffu, sn[i % kMine], p / kMine);
        }
        for (; h0 < h_end; h0 += kHeads * kAhead) {
            Dims<T> next[kAhead];
            fetch(next, h0 + kHeads * kAhead);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int h = h0 + j * kHeads;
                if (h >= h_end) break;
                uint16_t* dst = target(h);
                if (!dst) continue;
                float x[16];
                now[j].get(x);
                if (h < Hv0) {
                    if (a.adjacent) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            if (u * 8 + i >= a.pairs) continue;            // dims that do not turn stay bit for bit
                            const float p = x[2 * i], q = x[2 * i + 1];
                            x[2 * i] = p * c[i] - q * s[i];
                            x[2 * i + 1] = q * c[i] + p * s[i];
                        }
                    } else if (u * 8 < a.pairs) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float p = x[i], q = x[8 + i];
                            x[i] = p * c[i] - q * s[i];
                            x[8 + i] = q * c[i] + p * s[i];
                        }
                    }
                }
                store8(dst + d0, x);
                store8(dst + d1, x + 8);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) now[j] = next[j];
        }
    } else {
        // a lane keeps its own pairs and walks the heads; dims that do not turn are copied two by two
        for (int h = h_begin; h < h_end; ++h) {
            const T* src = source(h);
            uint16_t* dst = target(h);
            if (!dst) continue;
            const bool turns = h < Hv0;
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int p = lane * kMine + i;
                const bool mine = p < a.pairs;
                const int e0 = mine && !a.adjacent ? p : 2 * p, e1 = mine && !a.adjacent ? p + a.pairs : 2 * p + 1;
                const float x = to_float(src[e0]), y = to_float(src[e1]);
                const uint32_t out = mine && turns ? pack2(x * cs[i] - y * sn[i], y * cs[i] + x * sn[i]) : pack2(x, y);
                dst[e0] = (uint16_t)out, dst[e1] = (uint16_t)(out >> 16);
            }
        }
    }
}

}  // namespace

cudaError_t launch_block_tables(int32_t batch, int32_t num_blocks, const int32_t* ctx_len, const int32_t* new_len, int32_t* held,
                                int64_t held_stride, const int32_t* n_held, const int32_t* free_blocks, int64_t n_free,
                                const int64_t* free_begin, int64_t max_entries, int64_t max_rows, int64_t* kv_indptr,
                                int32_t* kv_indices, int64_t* q_indptr, int64_t* slot_map, int32_t* positions, int32_t* row_req,
                                int32_t* n_held_new, int64_t* free_end, int32_t* status, cudaStream_t stream) {
    const TablesArgs a{batch, num_blocks, ctx_len, new_len, n_held, free_blocks, held, held_stride, n_free, free_begin, max_entries,
                       max_rows, kv_indptr, q_indptr, free_end, kv_indices, slot_map, positions, row_req, n_held_new, status};
    const int64_t most = max_entries > max_rows ? max_entries : max_rows;
    const int64_t grid = most > 0 ? (most + kTablesPerCta - 1) / kTablesPerCta : 1;
    block_tables_kernel<<<(unsigned)grid, kTablesThreads, (5 * (size_t)batch + 3) * sizeof(int32_t), stream>>>(a);
    return cudaGetLastError();
}

cudaError_t tables_init() {
    return cudaFuncSetAttribute(block_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (5 * kMaxTableBatch + 3) * (int)sizeof(int32_t));
}

cudaError_t launch_rope_append(const RopeLaunch& l, cudaStream_t stream) {
    RopeArgs a{};
    a.n_rows = l.n_rows;
    a.q = l.q, a.k = l.k, a.v = l.v;
    a.q_stride = l.q_stride, a.k_stride = l.k_stride, a.v_stride = l.v_stride, a.qo_stride = l.q_out_stride;
    a.q_out = l.q_out;
    a.slab = l.slab;
    a.positions = l.positions;
    a.inv_freq = l.inv_freq;
    a.slot_map = l.slot_map;
    a.status = l.status;
    a.Hq = l.shape.Hq, a.Hkv = l.shape.Hkv, a.num_blocks = l.shape.num_blocks;
    a.pairs = l.pairs, a.adjacent = l.adjacent;
    a.hq0 = l.q ? 0 : a.Hq;
    a.heads = l.k ? a.Hq + 2 * a.Hkv : a.Hq;
    for (int p = 0; p < l.pairs; ++p) a.axis[p] = l.axis[p];
    const int elem = l.in_bf16 ? 2 : 4;
    auto aligned = [](const void* p, int64_t stride_bytes) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride_bytes % 16 == 0; };
    const bool vec = (l.adjacent || l.pairs % 8 == 0) && (!l.q || (aligned(l.q, l.q_stride * elem) && aligned(l.q_out, l.q_out_stride * 2))) &&
                     (!l.k || (aligned(l.k, l.k_stride * elem) && aligned(l.v, l.v_stride * elem)));
    // Few rows: a row's heads go to several warps, until the machine has some eight warps per SM (320 rows: 4.3 us with four
    // warps a row, 6.2 with one or eight).
    while (a.log2_parts < 3 && (l.n_rows << a.log2_parts) < 8LL * l.n_sms && ((a.heads - a.hq0) >> (a.log2_parts + 1)) >= 4) ++a.log2_parts;
    const int64_t warps = l.n_rows << a.log2_parts;
    const unsigned grid = (unsigned)((warps * 32 + 255) / 256);
#define NSD_ROPE(T, D, V) rope_append_kernel<T, D, V><<<grid, 256, 0, stream>>>(a)
    if (l.in_bf16) {
        if (l.shape.D == 128) vec ? NSD_ROPE(__nv_bfloat16, 128, true) : NSD_ROPE(__nv_bfloat16, 128, false);
        else vec ? NSD_ROPE(__nv_bfloat16, 64, true) : NSD_ROPE(__nv_bfloat16, 64, false);
    } else {
        if (l.shape.D == 128) vec ? NSD_ROPE(float, 128, true) : NSD_ROPE(float, 128, false);
        else vec ? NSD_ROPE(float, 64, true) : NSD_ROPE(float, 64, false);
    }
#undef NSD_ROPE
    return cudaGetLastError();
}

}  // namespace nsd
