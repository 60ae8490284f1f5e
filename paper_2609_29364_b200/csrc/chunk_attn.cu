// Attention of a chunk of new tokens over the paged pool: any number of rows per request, from a
// single token to a whole prompt (Section 3, block maps; Appendix G.2, the target's forward pass).
#include <cuda_bf16.h>

#include "nsd_internal.h"
#include "tcgen05_ops.h"

namespace nsd {
namespace {

constexpr int kTileKeys = 128;
constexpr int kRows = 128;                             // stacked rows of a tile
constexpr uint32_t kMagic = 0x4e534443u;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// What work costs, for the split over the CTAs: a key tile 1 in a unit of one row tile and 2 in a unit of two, and a unit what
// two of its tiles do (loading Q, filling the pipeline, writing O).  Measured with 122 single tokens over 4600 keys beside
// 2500 tokens of prompts (D = 128, four q heads per kv head, no masks): 578 us; 749 with all tiles alike, 623 with 1.5, 607
// with 2.5.  Other shapes, masks and caps share the rule unmeasured; the split stays exact, only its balance depends on it.
constexpr int kUnitTiles = 2;

__device__ __forceinline__ void report(int32_t* status, int32_t bit, int r) {
    atomicOr(status, bit);
    atomicCAS(status + 1, 0, r + 1);
}

__device__ __forceinline__ int tile_cost(const ChunkUnit& u, int T) { return u.ntok > T ? 2 : 1; }
__device__ __forceinline__ int64_t unit_cost(const ChunkUnit& u, int T) { return ((int64_t)u.n_tiles + kUnitTiles) * tile_cost(u, T); }

// A buffer that nsd_chunk_plan has filled for these rows, this shape and this layout (max_units follows from max_batch, and
// with max_rows and n_ctas places every part up to the partial results).
__device__ __forceinline__ bool is_plan(const ChunkPlan& p, int T, int Hkv) {
    const ChunkHeader h = *p.header;
    return h.magic == kMagic && h.max_rows == p.max_rows && h.max_units == p.max_units && h.n_ctas == p.n_ctas && h.T == T && h.Hkv == Hkv;
}

// ---- plan -------------------------------------------------------------------------------------
// Two kernels.  The first works on every request's units side by side: the visible keys of each
// row and their hull over the unit.  Unit j of request r sits at r + floor(q_indptr[r] / TU) + j,
// an index that needs no prefix sum and leaves at most one gap per request.  The second, one CTA,
// closes the gaps, sums the costs and cuts the whole work -- units x kv heads x key tiles in one
// line -- into n_ctas equal pieces.  Two launches and two chains of dependent loads bound it: 7 to
// 9 us for a prompt of 8192, for 64 single tokens and for 128 mixed requests alike, once per step.
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
            int lo = 0x7fffffff, hi = 0, reach = 0;    // reach: the largest stop so far
            bool gaps = false;
            for (int b = i0; b < i0 + u.ntok; b += 32) {
                const int i = b + lane, pos = ctx + i;
                const int stop = max(pos + 1, prefix);
                int first = a.masks.window > 0 ? max(pos + 1 - a.masks.window, 0) : 0;
                bool any = false;
                if (i < i0 + u.ntok) {
                    if (a.masks.row_first) first = max(first, a.masks.row_first[s + i]);
                    any = first < stop;
                    a.p.row_lo[s + i] = any ? first : 0;
                    a.p.row_hi[s + i] = any ? stop : 0;
                    if (any) lo = min(lo, first), hi = max(hi, stop);
                }
                // Stops grow from row to row, so the keys of rows that follow one another without an empty one between leave no
                // gap, and the first row behind a gap begins above every stop before it.
                if (a.masks.row_first) {
                    int upto = any ? stop : 0;
#pragma unroll
                    for (int d = 1; d < 32; d <<= 1) upto = max(upto, __shfl_up_sync(0xffffffffu, upto, d));
                    const int left = __shfl_up_sync(0xffffffffu, upto, 1), before = max(reach, lane > 0 ? left : 0);
                    gaps |= any && before > 0 && first > before;
                    reach = max(reach, __shfl_sync(0xffffffffu, upto, 31));
                }
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            u.gaps = __any_sync(0xffffffffu, gaps);
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
        if (a.p.raw[i].ntok > 0) ++n_mine, c_mine += unit_cost(a.p.raw[i], a.T);
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
        c_at += unit_cost(u, a.T);
    }
    if (tid == 0) {
        cost[n_units] = c_all;
        *a.p.header = ChunkHeader{kMagic, n_units, a.p.max_rows, a.p.max_units, a.p.n_ctas, a.masks.window == 0 && !a.masks.prefix_len && !a.masks.row_first, a.T, a.Hkv};
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
            st.tile = (int)max((int64_t)0, (rem - cost[lo]) / tile_cost(a.p.units[lo], a.T) - kUnitTiles);
        }
        a.p.starts[c] = st;
    }
}

// ---- attention ----------------------------------------------------------------------------------
// A unit is up to 2 T tokens of one request (T = 128 / G) times the G q heads of a kv head: the
// stacked rows of a token sit side by side, T tokens fill a tile of 128 rows, two tiles make a
// unit.  Per key tile of 128 keys and row tile, on the tensor cores:
//     S[128 x 128]  = Q K^T          Q and K in shared memory (K-major, 128-byte swizzle)
//     O[128 x D]   += P V            P in tensor memory over S's own columns, V in shared memory
// The two row tiles are two streams that share every K and V tile and run half a step apart: while
// one stream's softmax works, the tensor cores work for the other.  A unit of one row tile (single
// tokens, the end of a chunk) gives the streams alternate key tiles instead, each with its own O
// and statistics, joined at the end through tensor memory; so short rows keep the same two tiles
// in flight and stay bound by HBM.
//
// One persistent CTA per SM, twelve warps:
//   0-3 / 4-7  softmax of stream 0 / 1: a thread owns a row (its TMEM lane).  Scores to the log2
//              domain with the scale folded in, maximum (refreshed, and O rescaled, only when a
//              score outgrows it by 2^8), P = 2^(s - m) to bf16 in two halves so that P V can start on
//              the first, sums in 32 bits over the unrounded weights.  They also write the rows out.
//   8 / 9      issue the MMAs of stream 0 / 1.  One thread issues S of a tile, then P V of it, so the
//              commit of S also tells that the stream's earlier P V are complete: O may be rescaled.
//   10         Q and K producer; 11: V producer.  A pool block (16 keys) of a head is one 5-D box
//              whose layout in shared memory -- [8-key group][64-dim half][8 keys][64 dims] -- puts
//              the 8-key groups of all eight blocks at one pitch (K's descriptor wants that) and a
//              block's groups and halves at fixed pitches (V's): one copy per block serves both.
// Keys are walked from the last tile to the first: the diagonal, with its masks, comes first, and
// with a bias on distance the largest scores do, so the maximum hardly moves.
//
// Work is cut into equal shares of the line (request, kv head, unit, key tile), one per CTA,
// whatever the lengths: a CTA may begin and end inside a unit.  Such a piece leaves its O
// (unnormalised) and statistics in the plan, and a small kernel behind this one joins them in order.
//
// Every wait is bounded.  When one runs out, the CTA raises its abort flag; once all warps have left
// their loops, each issuer waits for its MMAs in flight and each producer for its copies (bounded
// again), and the call ends with STATUS_TIMEOUT.
//
// Measured (32 q heads, 8 kv heads of 128): a prompt of 8192 tokens 480 us = 1146 TFLOP/s -- the
// exponentials (16 per SM and cycle) and the tensor cores are each busy 57 % of it, the rest is the
// chain S -> maximum -> exponentials -> P V within a step of two streams; 2047 tokens over 62 221
// keys 2150-2240 us = 950-990 TFLOP/s at the board's power limit (1420 MHz; 1890 us = 1122 on a cool
// board); 64 single tokens over 512 to 2048 keys 66 us = 5.4 TB/s, 5 over 30 000 to 120 000
// 218 us = 6.7 TB/s: HBM; one token over 16 keys 8.9 us: launches and one pass through the pipeline.
// D = 64 halves the products but shortens the chain little: a prompt of 4096 121 us against 153 (the
// exponentials would take 59), 64 single tokens over 4096 keys 108 us = 5.0 TB/s against 170 = 6.3.
constexpr int kBsA = 16;
constexpr int kBlocks = kTileKeys / kBsA;
constexpr int kThreadsA = 384;
constexpr int kWarpIssue = 8, kWarpK = 10, kWarpV = 11;
constexpr float kMaxSlack = 8.0f;                      // the running maximum may lag the true one by this much (log2 units)
constexpr uint32_t kPollLimit = 1u << 30;              // polls of one wait, if nsd_config.wait_budget does not say
enum : int { MODE_CAP = 1, MODE_BIAS = 2 };

struct AttnArgs {
    CUtensorMap kv_map, q_map;
    ChunkPlan p;
    uint16_t* o;
    float* lse;
    const int32_t* kv_indices;
    const float* slopes;
    float sc;                                          // scale, in the log2 domain; with a cap: scale / cap
    float cap;                                         // cap in the log2 domain
    int32_t *status, Hq, Hkv, G, T, num_blocks;
    uint32_t wait_budget;
};

template <int D>
struct Smem {
    static constexpr int kHalves = D / 64;
    static constexpr int kBlockBytes = kBsA * D * 2;
    static constexpr int kTile = kTileKeys * D * 2;    // a K or V tile
    static constexpr int kQ = kRows * D * 2;
    static constexpr int kGroupPitch = kHalves * 1024; // between 8-key groups
    static constexpr int kKStages = D == 128 ? 3 : 5, kVStages = D == 128 ? 2 : 5;
    static constexpr int kOffK = 2 * kQ, kOffV = kOffK + kKStages * kTile;
    static constexpr int kOffMl = kOffV + kVStages * kTile;              // [2] statistics for a join, by the stream that joins
    static constexpr int kOffBars = kOffMl + 2 * kRows * 8;
    static constexpr int kNumBars = 3 * kKStages + 3 * kVStages + 2 + 4 + 2 + 4 + 2 + 4 + 2 + 2;
    static constexpr int kOffMisc = kOffBars + kNumBars * 8;
    static constexpr int kBytes = kOffMisc + 16;
    static_assert(kBytes <= 227 * 1024, "shared memory budget");
};
constexpr int kTmemColsA = 512, kTmemOBase = 256;      // S0, S1, O0, O1: 128 columns each

// A CTA's walk over its share of the line.
struct Walk {
    const ChunkUnit* units;
    ChunkStart at, end;
    int Hkv;
    // the piece under way
    ChunkUnit u;
    int head, k0, k1, slot;                            // key tiles [k0, k1) in walking order; partial slot or -1
    __device__ __forceinline__ Walk(const ChunkPlan& p, int Hkv_, bool planned) : units(p.units), at{}, end{}, Hkv(Hkv_) {
        if (planned) at = p.starts[blockIdx.x], end = p.starts[blockIdx.x + 1];
    }
    __device__ __forceinline__ bool next() {
        if (at.unit == end.unit && at.head == end.head && at.tile == end.tile) return false;
        u = units[at.unit];
        head = at.head;
        k0 = at.tile;
        const bool cut = at.unit == end.unit && at.head == end.head;
        k1 = cut ? end.tile : u.n_tiles;
        slot = k0 > 0 ? 2 * (int)blockIdx.x : (cut ? 2 * (int)blockIdx.x + 1 : -1);
        if (cut) {
            at = end;
        } else {
            at.tile = 0;
            if (at.unit < u.last) ++at.unit;
            else if (at.head + 1 < Hkv) ++at.head, at.unit = u.first;
            else at.head = 0, at.unit = u.last + 1;
        }
        return true;
    }
};

// A bounded wait of a whole warp.  Unlike mbar_wait it gives the hardware no time slice: a barrier that is ready then costs
// 78 cycles instead of 113, and a signal from one warp to another as much instead of 112.  The bound is a number of polls
// (limit) and, since a poll may sleep, a time: about four seconds of SM clocks.
constexpr long long kWaitCycles = 1ll << 33;
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
    const long long t0 = clock64();
    for (uint32_t i = 0; i < limit; ++i) {
        if (bar_try(bar, parity)) return true;
        if (*abort_flag) return false;
        if (clock64() - t0 > kWaitCycles) break;
    }
    *abort_flag = 1;
    return false;
}
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p)::"memory");
    return p;
}
// Waits for this thread's tensor-memory loads; the registers of one of them are operands, so that no use of them can be moved
// in front of the wait.
__device__ __forceinline__ void tmem_wait_ld32(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                   "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                   "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]),
                   "+r"(r[31])::"memory");
}
// Two floats in one 64-bit register pair: the packed FMA, add and multiply of sm_100 do both in one issue slot.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpair(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// x becomes cap * tanh(x * sc) for 32 scores of a row.  Where every score of the warp's 32 rows allows, tanh(t) is t times a
// polynomial in t^2 fitted to least relative error: degree 4 up to 3/4 (6e-7), degree 7 up to 3/2 (7e-7) -- no MUFU
// instruction, of which 1 - 2 / (1 + e^2t), for the rest, takes two.  (tanh.approx is one, but off by 2^-11: times a cap of 30
// to 50, one weight in fifty.)  That difference is off by 2^-21 of the cap, however small the score: with caps up to kCapExp
// less than a quarter of what the weights' rounding costs, above them the small scores of a mixed lot take the polynomial one by one.
constexpr float kCapExp = 2048.f;                      // in the log2 domain
template <int N>
__device__ __forceinline__ void cap32_poly(uint32_t* x, uint64_t sc2, uint64_t cap2, const float (&k)[N]) {
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        const uint64_t t = mul2(pair(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), sc2), y = mul2(t, t);
        uint64_t p = pair(k[N - 1], k[N - 1]);
#pragma unroll
        for (int i = N - 2; i >= 0; --i) p = fma2(p, y, pair(k[i], k[i]));
        const float2 r = unpair(mul2(mul2(t, cap2), p));
        x[j] = __float_as_uint(r.x), x[j + 1] = __float_as_uint(r.y);
    }
}
__device__ __forceinline__ void cap32(uint32_t* x, float sc, float cap) {
    float big = 0.f, big1 = 0.f;
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        big = fmaxf(fmaxf(big, fabsf(__uint_as_float(x[j]))), fabsf(__uint_as_float(x[j + 1])));
        big1 = fmaxf(fmaxf(big1, fabsf(__uint_as_float(x[j + 2]))), fabsf(__uint_as_float(x[j + 3])));
    }
    big = fmaxf(big, big1) * sc;
    const uint64_t sc2 = pair(sc, sc), cap2 = pair(cap, cap);
    const float small[5] = {0.999999463558197f, -0.3332825303077698f, 0.13259011507034302f, -0.050057198852300644f, 0.01293052639812231f};
    if (!__any_sync(0xffffffffu, big > 0.75f)) {
        cap32_poly(x, sc2, cap2, small);
    } else if (!__any_sync(0xffffffffu, big > 1.5f)) {
        const float k[8] = {0.9999993443489075f, -0.33329400420188904f, 0.13294775784015656f, -0.0524834468960762f,
                            0.018927596509456635f, -0.005435946863144636f, 0.001021950040012598f, -8.943479042500257e-05f};
        cap32_poly(x, sc2, cap2, k);
    } else if (cap > kCapExp) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float t = __uint_as_float(x[j]) * sc, y = t * t;
            float r, p = small[4];
#pragma unroll
            for (int i = 3; i >= 0; --i) p = fmaf(p, y, small[i]);
            const float e = ex2_approx(t * (2.f * kLog2e)) + 1.f;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e));
            x[j] = __float_as_uint(fabsf(t) <= 0.75f ? t * cap * p : fmaf(-2.f * cap, r, cap));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            float r;
            const float e = ex2_approx(__uint_as_float(x[j]) * (2.f * kLog2e * sc)) + 1.f;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e));
            x[j] = __float_as_uint(fmaf(-2.f * cap, r, cap));
        }
    }
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int32_t tile, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(tile), "r"(bar)
                 : "memory");
}

template <int D, int MODE>
__global__ void __launch_bounds__(kThreadsA, 1)
chunk_attn_kernel(const __grid_constant__ AttnArgs a) {
    using L = Smem<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    pdl_release_dependents();
    const uint32_t smem0 = smem_u32(smem);
    if ((smem0 & 1023u) != 0) {
        pdl_wait();
        if (threadIdx.x == 0) atomicOr(a.status, STATUS_LAYOUT);
        return;
    }
    const uint32_t bar0 = smem0 + L::kOffBars;
    const uint32_t k_full = bar0, k_empty = k_full + 16 * L::kKStages, v_full = k_empty + 8 * L::kKStages, v_empty = v_full + 16 * L::kVStages;
    const uint32_t v_land = v_empty + 8 * L::kVStages; // [2] a V tile whose hidden rows have to be cleared lands here first
    const uint32_t q_full = v_land + 16, q_empty = q_full + 16;                          // [2] per Q buffer
    const uint32_t s_full = q_empty + 16, p_full = s_full + 16, o_full = p_full + 32;   // [2], [2][2 halves], [2] per stream
    const uint32_t x_ready = o_full + 16, x_done = x_ready + 16;                        // [2] the join of a one-tile unit's streams
    const uint32_t begun = x_done + 16;                                                 // [2] a stream has taken a tile's scores out
    const uint32_t flushed = begun + 16;                                                // [2] an issuer that gives up has no MMA in flight
    uint32_t& tmem_base_s = *reinterpret_cast<uint32_t*>(smem + L::kOffMisc);
    volatile int& abort_s = *reinterpret_cast<volatile int*>(smem + L::kOffMisc + 4);
    float2* const ml_s = reinterpret_cast<float2*>(smem + L::kOffMl);
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);                             // the compiler then knows it is the warp's
    const uint32_t limit = a.wait_budget ? a.wait_budget : kPollLimit;

    if (tid == 0) {
        for (int s = 0; s < L::kKStages; ++s) mbar_init(k_full + 16 * s, 1), mbar_init(k_full + 16 * s + 8, 1), mbar_init(k_empty + 8 * s, 2);
        for (int s = 0; s < L::kVStages; ++s) mbar_init(v_full + 16 * s, 1), mbar_init(v_full + 16 * s + 8, 1), mbar_init(v_empty + 8 * s, 2);
        mbar_init(v_land, 1), mbar_init(v_land + 8, 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(q_full + 8 * s, 1), mbar_init(q_empty + 8 * s, 2);
            mbar_init(s_full + 8 * s, 1), mbar_init(o_full + 8 * s, 1);
            mbar_init(x_ready + 8 * s, 4), mbar_init(x_done + 8 * s, 4), mbar_init(begun + 8 * s, 4), mbar_init(flushed + 8 * s, 1);
            mbar_init(p_full + 16 * s, 4), mbar_init(p_full + 16 * s + 8, 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        abort_s = 0;
    }
    if (warp == kWarpIssue) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "n"(kTmemColsA) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
    // Everything so far ran beside the end of the kernel before this one; what it writes (the plan, q, the pool) is read, and what
    // it reads is written, from here on.
    pdl_wait();
    const bool planned = is_plan(a.p, a.T, a.Hkv);
    if (!planned && blockIdx.x == 0 && tid == 0) report(a.status, STATUS_BAD_TOKEN, -1);
    Walk w(a.p, a.Hkv, planned);
    // the count-th completion; the same answer in every lane
    auto poll = [&](uint32_t bar, uint32_t count) { return (bool)__all_sync(0xffffffffu, bar_try(bar, count & 1)); };
    auto wait = [&](uint32_t bar, uint32_t count) {
        bool ok = bar_try(bar, count & 1);
        if (__all_sync(0xffffffffu, ok)) return true;
        ok = bar_wait_slow(bar, count & 1, &abort_s, limit);
        return (bool)__all_sync(0xffffffffu, ok);
    };

    // A ring's stage has two "full" barriers, for its even and its odd uses.  A wait by parity takes a phase that has not begun
    // for the one two before it; with alternate tiles an issuer does not watch every use of a stage, and one that runs ahead of
    // the other could so take a tile that is still in flight for landed.  The use two before lies an even number of tiles back:
    // it was the same stream's, or part of a unit of two row tiles, and has been watched.
    auto full_bar = [](uint32_t full, uint32_t tile, uint32_t stages) { return full + 16 * (tile % stages) + 8 * ((tile / stages) & 1); };
    auto full_phase = [](uint32_t tile, uint32_t stages) { return tile / stages / 2; };

    // Behind this barrier every warp has left its loop and the abort flag is final: one that looked at it earlier could leave
    // copies or MMAs in flight behind when another warp gives up later.
    auto all_done = [] {
        __syncwarp();
        asm volatile("barrier.cta.sync 1, %0;" ::"n"(kThreadsA) : "memory");
    };

    if (warp < kWarpIssue) {
        // ================================ softmax and output ================================
        // A row's 128 scores stay in registers.  The block was launched with 384 x 168 registers; the warpgroup of issuers
        // and producers gives up 104 of each thread's, the two softmax warpgroups take 48: 128 x 64 + 256 x 216 <= 384 x 168.
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int s = warp >> 2, q = warp & 3;
        const uint32_t lanes = (uint32_t)(q * 32) << 16;
        const uint32_t tmem_s = tmem + s * 128 + lanes, tmem_o = tmem + kTmemOBase + s * 128 + lanes;
        const int m = q * 32 + lane, tok = m / a.G, g = m - tok * a.G;
        // One register of parities: phases of S, of O of this stream and of the other, of joins by this stream and by the other,
        // key tiles so far; and whether the other stream is still reading this one's O.
        enum : uint32_t { PH_S = 1, PH_O = 2, PH_O_OTHER = 4, PH_X = 8, PH_X_OTHER = 16, PH_TILE = 32, LENT = 64, CAUSAL = 128 };
        uint32_t ph = planned && a.p.header->causal ? CAUSAL : 0;    // CAUSAL: a row's keys follow from its position
        bool fail = false;
        auto wait_all = [&](uint32_t bar, uint32_t phase) {
            fail = !wait(bar, (ph & phase) ? 1 : 0);
            return !fail;
        };
        auto give_back = [&] {                         // waits until the other stream has read this one's O
            if (wait_all(x_done + 8 * (s ^ 1), PH_X_OTHER)) ph ^= PH_X_OTHER | LENT;
        };
        while (!fail && w.next()) {
            const int n = w.k1 - w.k0;
            const bool dual = w.u.ntok > a.T;
            // Alternate tiles: tile c of the CTA's walk belongs to stream c & 1, and the stream of a piece's first tile writes its
            // rows out.  So a piece of a single tile leaves the other stream free for the next.
            const bool leads = dual || ((ph & PH_TILE) ? 1 : 0) == s, join = !dual && n > 1;
            const int i0 = leads ? 0 : 1;
            if (n & 1) ph ^= PH_TILE;
            if (!leads && !join) {
                if (n > 0) ph ^= PH_O_OTHER;
                continue;
            }
            const int t_row = (dual ? s * a.T : 0) + tok;                               // token of the unit
            const bool live = tok < a.T && t_row < w.u.ntok;
            const bool warp_live = __any_sync(0xffffffffu, live);
            const int64_t row = w.u.row0 + t_row;
            const int h = w.head * a.G + g;
            int lo = 0, hi = 0x7fffffff;                                                // lanes without a row never mask
            float slope = 0.f;
            if constexpr (MODE & MODE_BIAS) slope = live ? a.slopes[h] * kLog2e : 0.f;
            const int pos = w.u.pos0 + t_row;
            if (live) {
                if (ph & CAUSAL) hi = pos + 1;
                else lo = a.p.row_lo[row], hi = a.p.row_hi[row];
            }
            float m_run = -INFINITY, l_run = 0.f;
            bool huge = false;                                                          // a row of the warp has had a maximum beyond 2^24
            const int t_hi = (w.u.key_hi + kTileKeys - 1) / kTileKeys;
            int mine = 0;                                                               // tiles of this stream
            if (n > 0 && (ph & LENT)) give_back();                                      // P V overwrites O
            if (fail) break;
            for (int i = i0; i < n; i += dual ? 1 : 2, ++mine) {
                if (!wait_all(s_full + 8 * s, PH_S)) break;
                ph ^= PH_S;
                tc_fence_after();
                if (warp_live) {
                    const int key0 = (t_hi - 1 - (w.k0 + i)) * kTileKeys;
                    const int v0 = lo - key0, v1 = hi - key0;                           // visible: v0 <= j < v1
                    constexpr bool kRaw = MODE == 0;                                    // x is q . k: the scale is part of the exponent's FFMA
                    float f = kRaw ? a.sc : 1.f;
                    uint32_t x[4][32];                                                  // scores, then pairs of weights
                    uint64_t l2[2] = {0, 0};                                            // the tile's sums
                    auto scores = [&](int c) {                                          // to what the softmax is of
                        if constexpr (MODE & MODE_BIAS) {
                            const float b = slope * (float)(key0 - pos + c * 32), sc = MODE & MODE_CAP ? 1.f : a.sc;
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[c][j] = __float_as_uint(fmaf(__uint_as_float(x[c][j]), sc, fmaf(slope, (float)j, b)));
                        }
                    };
                    auto largest = [&] {
                        float m0[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int j = 0; j < 32; j += 2)
#pragma unroll
                            for (int c = 0; c < 4; ++c) m0[c] = fmaxf(fmaxf(m0[c], __uint_as_float(x[c][j])), __uint_as_float(x[c][j + 1]));
                        return fmaxf(fmaxf(m0[0], m0[1]), fmaxf(m0[2], m0[3])) * f;
                    };
                    auto weights = [&](int c) {                                         // 32 scores become 16 words of P
                        const float nm = m_run == -INFINITY ? 0.f : -m_run;
                        const uint64_t f2 = pair(f, f), nm2 = pair(nm, nm);
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float2 p = unpair(fma2(pair(__uint_as_float(x[c][2 * j]), __uint_as_float(x[c][2 * j + 1])), f2, nm2));
                            p.x = ex2_approx(p.x), p.y = ex2_approx(p.y);
                            l2[j & 1] = add2(l2[j & 1], pair(p.x, p.y));
                            x[c][j] = pack_bf16(p.x, p.y);
                        }
                    };
                    auto store = [&](int half) {
                        tmem_st16(tmem_s + half * 32, x[2 * half]);
                        tmem_st16(tmem_s + half * 32 + 16, x[2 * half + 1]);
                    };
                    auto hand_over = [&](int half) {                                    // the half's P is in tensor memory
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(p_full + 16 * s + 8 * half);
                    };
                    // Scores are capped and hidden where they lie, 32 at a time, in a loop of its own: one copy of that code, and
                    // none of it in the way of a tile that needs neither.
                    const bool masked = __any_sync(0xffffffffu, v0 > 0 || v1 < kTileKeys);
                    if ((MODE & MODE_CAP) || masked) {
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            tmem_ld32(tmem_s + c * 32, x[0]);
                            tmem_wait_ld32(x[0]);
                            if constexpr (MODE & MODE_CAP) cap32(x[0], a.sc, a.cap);
                            if (masked) {
                                const int first = v0 - c * 32, stop = v1 - c * 32;
#pragma unroll
                                for (int j = 0; j < 32; ++j) x[0][j] = j >= first && j < stop ? x[0][j] : 0xff800000u;
                            }
                            tmem_st32(tmem_s + c * 32, x[0]);
                        }
                        tmem_wait_st();
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(tmem_s + c * 32, x[c]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        tmem_wait_ld32(x[c]);
                        scores(c);
                    }
                    if (dual && lane == 0) mbar_arrive(begun + 8 * s);
                    const float m_tile = largest();
                    const bool outgrown = mine == 0 || m_tile > m_run + kMaxSlack;  // the piece's first tile sets the maximum
                    if (__any_sync(0xffffffffu, outgrown)) {
                        const float m_new = outgrown ? m_tile : m_run;
                        // O holds this piece's earlier tiles, complete since S of this one is
                        if (mine > 0) {
                            const float r = outgrown ? (m_run == -INFINITY ? 0.f : ex2_approx(m_run - m_new)) : 1.f;
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t y[16];
                                tmem_ld16(tmem_o + c, y);
                                tmem_wait_ld();
#pragma unroll
                                for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * r);
                                tmem_st16(tmem_o + c, y);
                            }
                            tmem_wait_st();
                            l_run *= r;
                        }
                        m_run = m_new;
                        if (kRaw) huge = huge || __any_sync(0xffffffffu, live && fabsf(m_run) > 0x1p24f && m_run != -INFINITY);
                    }
                    // The FFMA does not round x f, but the maximum is rounded, and what it loses beyond 2^24 can put all of a row's
                    // weights out of range.  Such a row's products are rounded too: the largest weight is then 1.
                    if (kRaw && huge) {
                        const bool big = fabsf(m_run) > 0x1p24f;
                        const float g = big ? a.sc : 1.f;
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int j = 0; j < 32; ++j) x[c][j] = __float_as_uint(__uint_as_float(x[c][j]) * g);
                        if (big) f = 1.f;
                    }
                    weights(0);
                    weights(1);
                    store(0);
                    weights(2);
                    hand_over(0);
                    weights(3);
                    store(1);
                    hand_over(1);
                    const float2 l = unpair(add2(l2[0], l2[1]));
                    l_run += l.x + l.y;
                } else {
                    if (dual && lane == 0) mbar_arrive(begun + 8 * s);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + 16 * s), mbar_arrive(p_full + 16 * s + 8);
                }
            }
            if (fail) break;
            // A score that is no number makes the row's sum one, though not its maximum, which passes it over.  Such a row joins
            // with a maximum of infinity: every factor of a join is then 0 or not a number, and its output too.
            if (l_run != l_run) m_run = INFINITY;
            // ---- the piece's rows
            if (!leads) {
                ml_s[(s ^ 1) * kRows + m] = make_float2(m_run, l_run);
                __syncwarp();
                if (lane == 0) mbar_arrive(x_ready + 8 * (s ^ 1));
                ph = (ph | LENT) ^ (PH_O | PH_O_OTHER);
                continue;
            }
            if (n > 0) {
                if (!wait_all(o_full + 8 * s, PH_O)) break;
                ph ^= PH_O;
            }
            float r0 = 1.f, r1 = 0.f;                                                   // weights of the two streams' O
            if (join) {
                if (!wait_all(x_ready + 8 * s, PH_X) || !wait_all(o_full + 8 * (s ^ 1), PH_O_OTHER)) break;
                ph ^= PH_X;
                const float2 ml = ml_s[s * kRows + m];
                const float top = fmaxf(m_run, ml.x);
                r0 = m_run == -INFINITY ? 0.f : ex2_approx(m_run - top);
                r1 = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
                l_run = l_run * r0 + ml.y * r1;
                m_run = top;
            }
            if (join || (dual && n > 0)) ph ^= PH_O_OTHER;
            const uint32_t tmem_other = tmem + kTmemOBase + (s ^ 1) * 128 + lanes;
            tc_fence_after();
            if (warp_live) {
                const int64_t orow = row * a.Hq + h;
                const bool part = w.slot >= 0;
                const int64_t prow = (int64_t)w.slot * 2 * kRows + (dual ? s * kRows : 0) + m;
                const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
                if (!part) r0 *= inv, r1 *= inv;
#pragma unroll 1
                for (int c = 0; c < D; c += 16) {
                    uint32_t y[16], z[16];
                    if (n > 0) {
                        tmem_ld16(tmem_o + c, y);
                        if (join) tmem_ld16(tmem_other + c, z);
                        tmem_wait_ld();
                    }
                    if (live) {
                        // a weight of zero means that the stream saw nothing: its O may be anything
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float v = r0 != 0.f && n > 0 ? __uint_as_float(y[j]) * r0 : 0.f;
                            if (join && r1 != 0.f) v = fmaf(__uint_as_float(z[j]), r1, v);
                            y[j] = __float_as_uint(v);
                        }
                        if (part) {
                            float4* pa = reinterpret_cast<float4*>(a.p.part_acc + prow * D + c);
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                pa[j] = make_float4(__uint_as_float(y[4 * j]), __uint_as_float(y[4 * j + 1]), __uint_as_float(y[4 * j + 2]), __uint_as_float(y[4 * j + 3]));
                        } else {
                            uint4* po = reinterpret_cast<uint4*>(a.o + orow * D + c);
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                uint32_t k[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) k[i] = pack_bf16(__uint_as_float(y[8 * j + 2 * i]), __uint_as_float(y[8 * j + 2 * i + 1]));
                                po[j] = make_uint4(k[0], k[1], k[2], k[3]);
                            }
                        }
                    }
                    __syncwarp();
                }
                if (live && part) *reinterpret_cast<float2*>(a.p.part_ml + prow * 2) = make_float2(m_run, l_run);
                if (live && !part && a.lse) a.lse[orow] = m_run == -INFINITY ? -INFINITY : (m_run + log2f(l_run)) * kLn2;
            }
            tc_fence_before();
            __syncwarp();
            if (join && lane == 0) mbar_arrive(x_done + 8 * s);
        }
        all_done();
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp < kWarpK) {
        // ================================ MMA issuers ================================
        const int s = warp - kWarpIssue;
        auto wait_full = [&](uint32_t full, uint32_t tile, uint32_t stages) { return wait(full_bar(full, tile, stages), full_phase(tile, stages)); };
        const uint32_t idesc_s = instr_desc(kRows, kTileKeys, 0, 0), idesc_o = instr_desc(kRows, D, 0, 1);
        const uint32_t tmem_s = tmem + s * 128, tmem_o = tmem + kTmemOBase + s * 128;
        uint32_t n_k = 0, n_p = 0, q_slot = 0, n_begun = 0;
        bool ok = true;
        // The whole warp waits, one elected thread issues: a branch of one lane around the waits costs hundreds of cycles.
        while (ok && w.next()) {
            const int n = __shfl_sync(0xffffffffu, w.k1 - w.k0, 0);
            if (n == 0) continue;
            const bool dual = __shfl_sync(0xffffffffu, (int)(w.u.ntok > a.T), 0) != 0;
            // both issuers watch every Q slot, so that none takes a slot in flight for the one two before it
            const uint32_t slot = q_slot + (dual ? s : 0), qb = slot & 1;
            ok = wait(q_full + 8 * (q_slot & 1), q_slot >> 1) && (!dual || wait(q_full + 8 * ((q_slot + 1) & 1), (q_slot + 1) >> 1));
            if (!ok) break;
            q_slot += dual ? 2 : 1;
            // and a slot of a pair is filled anew only when this issuer, whose it is not, has watched it too: it could else be
            // full twice between two looks, which a wait by parity takes for not full yet
            if (dual && lane == 0) mbar_arrive(q_empty + 8 * (qb ^ 1));
            const int step = dual ? 1 : 2, i0 = dual ? 0 : (int)((n_k ^ s) & 1);
            if (i0 >= n && lane == 0) mbar_arrive(q_empty + 8 * qb);                    // a single key tile, the other stream's
            const uint64_t dq = smem_desc(smem0 + qb * L::kQ, 16, 1024, 2);
            for (int i = i0; i < n; i += step, ++n_p) {
                const uint32_t c = n_k + i, ks = c % L::kKStages, vs = c % L::kVStages;
                const bool last = i + step >= n;
                if (!(ok = wait_full(k_full, c, L::kKStages))) break;
                if (dual) {
                    // The streams keep half a step apart: S of a tile goes once the other stream has taken the scores of the tile
                    // before out (in step both would wait for S and then both for the MUFU unit: a prompt of 8192 tokens 565 us
                    // instead of 525).
                    ok = s == 1 ? wait(begun, n_begun) : (n_begun == 0 || wait(begun + 8, n_begun - 1));
                    if (!ok) break;
                    ++n_begun;
                }
                tc_fence_after();
                const uint64_t dk = smem_desc(smem0 + L::kOffK + ks * L::kTile, 16, L::kGroupPitch, 2);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k)                                    // 16 dims each, 64 per swizzled half
                        umma_ss(tmem_s, dq + (((k >> 2) * (kRows * 128) + (k & 3) * 32) >> 4), dk + (((k >> 2) * 1024 + (k & 3) * 32) >> 4), idesc_s, k > 0);
                    umma_commit(s_full + 8 * s);
                    umma_commit(k_empty + 8 * ks);
                    if (!dual) mbar_arrive(k_empty + 8 * ks);                           // the other stream has no use for this tile
                    if (last) umma_commit(q_empty + 8 * qb);
                }
                if (!(ok = wait_full(v_full, c, L::kVStages))) break;
                const uint64_t dv = smem_desc(smem0 + L::kOffV + vs * L::kTile, 1024, L::kGroupPitch, 2);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (!(ok = wait(p_full + 16 * s + 8 * half, n_p))) break;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int k = half * 4; k < half * 4 + 4; ++k)                   // 16 keys each: a block of V, 8 columns of P
                            umma_ts(tmem_o, tmem_s + k * 8, dv + ((k * L::kBlockBytes) >> 4), idesc_o, (i > i0 || k > 0) ? 1u : 0u);
                        if (half == 1) {
                            umma_commit(v_empty + 8 * vs);
                            if (!dual) mbar_arrive(v_empty + 8 * vs);
                            if (last) umma_commit(o_full + 8 * s);
                        }
                    }
                }
                if (!ok) break;
            }
            n_k += n;
        }
        all_done();
        if (abort_s) {
            // the CTA is giving up: what is still in flight reads shared memory and writes tensor memory
            if (elect_one()) umma_commit(flushed + 8 * s);
            const long long t0 = clock64();
            while (!bar_try(flushed + 8 * s, 0) && clock64() - t0 < kWaitCycles) {}
        }
    } else {
        // ================================ producers ================================
        const bool is_v = warp == kWarpV;
        const int stages = is_v ? L::kVStages : L::kKStages;
        const uint32_t full = is_v ? v_full : k_full, empty = is_v ? v_empty : k_empty;
        const uint32_t ring = smem0 + (is_v ? L::kOffV : L::kOffK);
        const int32_t oob = a.num_blocks * 2 * a.Hkv;                                   // past the slab: zero fill
        uint32_t n_t = 0, q_slot = 0, n_land = 0;      // copies sent out: tiles, Q buffers, tiles by way of a landing barrier
        uint32_t landing = 0;                          // of the latest tiles, the newest in bit 0: by way of a landing barrier
        bool ok = true;
        // Hidden rows of V have to be finite, since 0 x NaN is NaN: those of a block that also holds visible keys are cleared once
        // the tile has landed (blocks outside the unit's hull are zero fill).  The next tile's copies go out first.
        struct Due {
            uint32_t at, full, land;                   // the tile, its full barrier, which landing
            int first, last, head, rows;               // rows [first, first + head) and [last, last + rows - head); rows = 0: nothing due
        } due{};
        auto clear = [&] {
            if (!wait(v_land + 8 * (due.land & 1), due.land >> 1)) {
                ok = false;
                due.rows = 0;
                return;
            }
            for (int c = lane; c < due.rows * (D / 8); c += 32) {
                const int k = c / (D / 8), ch = c % (D / 8), r = k < due.head ? due.first + k : due.last + k - due.head;
                *reinterpret_cast<int4*>(smem + due.at + (r >> 4) * L::kBlockBytes + ((r >> 3) & 1) * L::kGroupPitch + (ch >> 3) * 1024 + (r & 7) * 128 + (ch & 7) * 16) = make_int4(0, 0, 0, 0);
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(due.full);
            due.rows = 0;
        };
        // Keys inside the hull that no row sees, in a unit with gaps: the lanes take four keys each and look at every row.  Rare
        // enough to be done at once, with the warp waiting for the tile: 10 000 tokens in documents of 300 to 900 take 122 us
        // without gaps and 155 with a padding row behind each document.
        auto clear_gaps = [&](int key0) {
            if (!wait(v_land + 8 * (due.land & 1), due.land >> 1)) {
                ok = false;
                due.rows = 0;
                return;
            }
            const int k0 = key0 + lane * 4;
            uint32_t seen = 0;
#pragma unroll 1
            for (int i = 0; i < w.u.ntok; ++i) {
                const int lo = a.p.row_lo[w.u.row0 + i] - k0, hi = a.p.row_hi[w.u.row0 + i] - k0;
#pragma unroll
                for (int j = 0; j < 4; ++j) seen |= (uint32_t)(j >= lo && j < hi) << j;
            }
#pragma unroll 1
            for (int j = 0; j < 4; ++j) {
                const int r = lane * 4 + j;
                if (seen >> j & 1) continue;
#pragma unroll 1
                for (int ch = 0; ch < D / 8; ++ch)
                    *reinterpret_cast<int4*>(smem + due.at + (r >> 4) * L::kBlockBytes + ((r >> 3) & 1) * L::kGroupPitch + (ch >> 3) * 1024 + (r & 7) * 128 + (ch & 7) * 16) = make_int4(0, 0, 0, 0);
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(due.full);
            due.rows = 0;
        };
        while (ok && w.next()) {
            const int n = w.k1 - w.k0;
            if (n == 0) continue;
            const bool dual = w.u.ntok > a.T;
            const int32_t* table = a.kv_indices + w.u.tbl;
            const int b_lo = w.u.key_lo / kBsA, b_hi = (w.u.key_hi + kBsA - 1) / kBsA;  // blocks that hold a visible key
            const int t0 = (w.u.key_hi + kTileKeys - 1) / kTileKeys - 1 - w.k0;         // first key tile
            // a lane's block of the next tile: its id is read one tile ahead
            auto block_id = [&](int t) -> int32_t {
                const int b = t * kBlocks + lane;
                if (lane >= kBlocks || b < b_lo || b >= b_hi) return -2;                // not needed
                return b < w.u.nblk ? __ldg(table + b) : -1;
            };
            int32_t id_next = block_id(t0);
            // Q, one buffer for each row tile, the two buffers in turn: a piece of one row tile finds the other one free.  It goes
            // first if its buffers are free, else behind the first K tiles, which need not wait for the last S of the piece
            // before.
            bool q_sent = is_v;
            auto send_q = [&](bool must) {
                const uint32_t last = q_slot + (dual ? 1 : 0);
                for (uint32_t k = q_slot; k <= last; ++k)
                    if (k >= 2 && !(must ? wait(q_empty + 8 * (k & 1), (k >> 1) - 1) : poll(q_empty + 8 * (k & 1), (k >> 1) - 1))) {
                        if (must) ok = false;
                        return;
                    }
                const uint32_t k = q_slot + lane, bar = q_full + 8 * (k & 1);
                if (k <= last) {
                    mbar_expect_tx(bar, a.T * a.G * D * 2);
#pragma unroll
                    for (int hh = 0; hh < L::kHalves; ++hh)
                        tma_load_3d(smem0 + (k & 1) * L::kQ + hh * (kRows * 128), &a.q_map, hh * 64, w.head * a.G, w.u.row0 + lane * a.T, bar);
                }
                __syncwarp();
                q_slot = last + 1;
                q_sent = true;
            };
            if (!is_v) send_q(false);
            for (int i = 0; i < n; ++i) {
                const uint32_t st = n_t % stages, use = n_t / stages;
                const int t = t0 - i;
                const int32_t id = id_next;
                if (i + 1 < n) id_next = block_id(t - 1);
                int32_t tile = oob;
                if (id != -2) {
                    if ((uint32_t)id < (uint32_t)a.num_blocks) tile = (id * 2 + (is_v ? 1 : 0)) * a.Hkv + w.head;
                    else report(a.status, STATUS_BAD_BLOCK, w.u.req);
                }
                if (use > 0) {
                    if (due.rows && !poll(empty + 8 * st, use - 1)) clear();
                    if (ok && !wait(empty + 8 * st, use - 1)) ok = false;
                }
                if (!ok) break;
                const int z0 = w.u.key_lo - t * kTileKeys, z1 = w.u.key_hi - t * kTileKeys;             // visible keys of the tile: [z0, z1)
                const int head_rows = z0 > 0 ? z0 & 15 : 0, tail_rows = z1 < kTileKeys ? -z1 & 15 : 0;
                const bool ragged = is_v && (head_rows | tail_rows | (int)w.u.gaps);
                const uint32_t full_now = full_bar(full, n_t, stages), bar = ragged ? v_land + 8 * (n_land & 1) : full_now;
                if (lane == 0) mbar_expect_tx(bar, L::kTile);
                __syncwarp();
                if (lane < kBlocks) tma_load_5d(ring + st * L::kTile + lane * L::kBlockBytes, &a.kv_map, tile, bar);
                ++n_t;                                                                  // from here on the tile is in flight, whatever gives up next
                landing = landing << 1 | (uint32_t)ragged;
                if (due.rows) clear();                                                  // the tile before, now that this one is under way
                if (ragged) due = Due{ring + st * L::kTile - smem0, full_now, n_land++, z0 - head_rows, z1, head_rows, head_rows + tail_rows};
                if (!ok) break;
                if (is_v && w.u.gaps) clear_gaps(t * kTileKeys);
                if (!q_sent && i == min(1, n - 1)) send_q(true);
                if (!ok) break;
            }
        }
        if (ok && due.rows) clear();
        all_done();
        if (abort_s && lane == 0) {
            // the CTA is giving up: copies that nobody waited for may still be landing; each barrier's latest phase gets a
            // bounded wait of its own before the shared memory goes back to the SM
            auto drain = [&](uint32_t bar, uint32_t count) {
                const long long t0 = clock64();
                while (!bar_try(bar, count & 1) && clock64() - t0 < kWaitCycles) {}
            };
            for (uint32_t back = 0; back < (uint32_t)stages && back < n_t; ++back)
                if (!(landing >> back & 1)) drain(full_bar(full, n_t - 1 - back, stages), full_phase(n_t - 1 - back, stages));
            for (uint32_t back = 1; back <= 2 && back <= n_land; ++back) drain(v_land + 8 * ((n_land - back) & 1), (n_land - back) >> 1);
            for (uint32_t back = 1; back <= 2 && back <= q_slot; ++back) drain(q_full + 8 * ((q_slot - back) & 1), (q_slot - back) >> 1);
        }
    }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kWarpIssue) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemColsA) : "memory");
    if (tid == 0 && abort_s) atomicOr(a.status, STATUS_TIMEOUT);
}

// Joins the pieces of the units that CTA boundaries cut: boundary c cuts unit (unit, head) when CTA c starts inside it, and
// the first such boundary of a unit does the work for all of them.  Pieces are read in walking order, so the result does not
// depend on timing.  A thread = four dims of one row at a time, four pieces' loads under way together: the chain of loads
// bounds it (one request of 8000 tokens, cut into 64 pieces, with one after another 27 us for both kernels, so 18).
constexpr int kJoinThreads = 256, kJoinSlices = 4, kMaxCtas = 511;
template <int D>
__global__ void __launch_bounds__(kJoinThreads)
chunk_join_kernel(const __grid_constant__ ChunkPlan p, uint16_t* __restrict__ o, float* __restrict__ lse, int32_t Hq, int32_t Hkv, int32_t G, int32_t T) {
    __shared__ ChunkStart starts[kMaxCtas + 1];
    const int c = blockIdx.x + 1;
    pdl_wait();
    if (!is_plan(p, T, Hkv)) return;
    const ChunkStart cut = p.starts[c], before = p.starts[c - 1];
    auto same = [&](const ChunkStart& x) { return x.unit == cut.unit && x.head == cut.head && x.tile > 0; };
    if (cut.tile == 0 || same(before)) return;
    const ChunkUnit u = p.units[cut.unit];
    const int elements = u.ntok * G * (D / 4);
    if ((int)blockIdx.y * kJoinThreads >= elements) return;
    for (int k = c + threadIdx.x; k <= p.n_ctas; k += kJoinThreads) starts[k] = p.starts[k];
    __syncthreads();
    int end = c;                                       // CTAs c .. end - 1 start inside the unit
    while (end < p.n_ctas && same(starts[end])) ++end;
    // a CTA without work left nothing
    auto left = [&](int k) {
        if (k < c) return true;
        const ChunkStart x = starts[k], y = starts[k + 1];
        return x.unit != y.unit || x.head != y.head || x.tile != y.tile;
    };
    for (int e = blockIdx.y * kJoinThreads + threadIdx.x; e < elements; e += kJoinSlices * kJoinThreads) {
        const int r = e / (D / 4), d4 = e % (D / 4), t = r / G, g = r - t * G;
        const int64_t in = (int64_t)(t / T) * kRows + (t % T) * G + g;                  // row of a partial slot
        float m = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kAhead = 4;                      // pieces whose loads are under way together
        for (int k0 = c - 1; k0 < end; k0 += kAhead) {
            float2 ml[kAhead];
            float4 v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int k = k0 + i;
                ml[i] = make_float2(-INFINITY, 0.f);
                v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < end && left(k)) {
                    const int64_t at = (int64_t)(k < c ? 2 * k + 1 : 2 * k) * 2 * kRows + in;
                    ml[i] = *reinterpret_cast<const float2*>(p.part_ml + at * 2);
                    v[i] = *reinterpret_cast<const float4*>(p.part_acc + at * D + d4 * 4);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (ml[i].x == -INFINITY) continue;    // this piece holds no key the row sees
                const float top = fmaxf(m, ml[i].x), f = m == -INFINITY ? 0.f : exp2f(m - top), x = exp2f(ml[i].x - top);
                acc.x = acc.x * f + v[i].x * x, acc.y = acc.y * f + v[i].y * x, acc.z = acc.z * f + v[i].z * x, acc.w = acc.w * f + v[i].w * x;
                l = l * f + ml[i].y * x;
                m = top;
            }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t orow = (int64_t)(u.row0 + t) * Hq + cut.head * G + g;
        *reinterpret_cast<uint2*>(o + orow * D + d4 * 4) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
        if (lse && d4 == 0) lse[orow] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * kLn2;
    }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn tensor_map_encoder() {
    static const EncodeFn f = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) fn = nullptr;
        return reinterpret_cast<EncodeFn>(fn);
    }();
    return f;
}
bool encode(CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    const EncodeFn f = tensor_map_encoder();
    return f && f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// A slab as [tile = (block, K|V, kv head)][8-key group][64-dim half][key][dim]; the box is one tile.
bool kv_map5(CUtensorMap* map, const void* slab, const Shape& s) {
    const cuuint64_t D = s.D;
    const cuuint64_t dims[5] = {64, 8, D / 64, 2, (cuuint64_t)s.num_blocks * 2 * s.Hkv};
    const cuuint64_t strides[4] = {D * 2, 128, 8 * D * 2, 16 * D * 2};
    const cuuint32_t box[5] = {64, 8, (cuuint32_t)(D / 64), 2, 1};
    return encode(map, slab, 5, dims, strides, box);
}
// The queries as [row][head][dim]; the box is T tokens of a kv head's G heads, 64 dims.
bool q_map3(CUtensorMap* map, const void* q, const Shape& s, int64_t rows, int64_t stride, int G, int T) {
    const cuuint64_t dims[3] = {(cuuint64_t)s.D, (cuuint64_t)s.Hq, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)s.D * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)T};
    return encode(map, q, 3, dims, strides, box);
}

template <int D, int MODE>
cudaError_t allow_smem() {
    return cudaFuncSetAttribute(chunk_attn_kernel<D, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<D>::kBytes);
}
template <int D>
cudaError_t allow_smem_all() {
    cudaError_t e = allow_smem<D, 0>();
    if (e == cudaSuccess) e = allow_smem<D, MODE_CAP>();
    if (e == cudaSuccess) e = allow_smem<D, MODE_BIAS>();
    if (e == cudaSuccess) e = allow_smem<D, MODE_CAP | MODE_BIAS>();
    return e;
}
template <int D>
cudaError_t launch_attn_d(const AttnArgs& a, int mode, int n_ctas, cudaStream_t st) {
    const dim3 grid(n_ctas), block(kThreadsA);
    const size_t smem = Smem<D>::kBytes;
    // a programmatic dependent of whatever precedes it: the kernel waits before it touches anything but its own shared memory
    switch (mode) {
        case 0: return launch_kernel(chunk_attn_kernel<D, 0>, grid, block, smem, st, true, a);
        case MODE_CAP: return launch_kernel(chunk_attn_kernel<D, MODE_CAP>, grid, block, smem, st, true, a);
        case MODE_BIAS: return launch_kernel(chunk_attn_kernel<D, MODE_BIAS>, grid, block, smem, st, true, a);
        default: return launch_kernel(chunk_attn_kernel<D, MODE_CAP | MODE_BIAS>, grid, block, smem, st, true, a);
    }
}

}  // namespace

size_t chunk_plan_layout(ChunkPlan* p, void* base, const Shape& s, int32_t max_batch, int64_t max_rows, int32_t n_sms) {
    n_sms = n_sms < kMaxCtas ? n_sms : kMaxCtas;
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
    cudaError_t e = cudaFuncSetAttribute(chunk_split_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kCostSmem * (int)sizeof(int64_t));
    if (e == cudaSuccess) e = allow_smem_all<128>();
    if (e == cudaSuccess) e = allow_smem_all<64>();
    return e;
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
    AttnArgs a{};
    a.G = l.shape.Hq / l.shape.Hkv;
    a.T = kRows / a.G;
    if (!kv_map5(&a.kv_map, l.slab, l.shape) || !q_map3(&a.q_map, l.q, l.shape, p.max_rows, l.q_stride, a.G, a.T)) return cudaErrorNotSupported;
    a.p = p;
    a.o = l.o, a.lse = l.lse, a.kv_indices = l.kv_indices, a.slopes = l.slopes;
    a.sc = l.softcap > 0.f ? l.scale / l.softcap : l.scale * kLog2e;
    a.cap = l.softcap * kLog2e;
    a.status = l.status;
    a.Hq = l.shape.Hq, a.Hkv = l.shape.Hkv, a.num_blocks = l.shape.num_blocks;
    a.wait_budget = l.wait_budget;
    const int mode = (l.softcap > 0.f ? MODE_CAP : 0) | (l.slopes ? MODE_BIAS : 0);
    cudaError_t e = l.shape.D == 128 ? launch_attn_d<128>(a, mode, p.n_ctas, stream) : launch_attn_d<64>(a, mode, p.n_ctas, stream);
    if (e != cudaSuccess) return e;
    *launched = 1;
    if (p.n_ctas < 2) return e;
    const dim3 grid(p.n_ctas - 1, kJoinSlices);
    e = l.shape.D == 128 ? launch_kernel(chunk_join_kernel<128>, grid, dim3(kJoinThreads), 0, stream, true, p, l.o, l.lse, a.Hq, a.Hkv, a.G, a.T)
                         : launch_kernel(chunk_join_kernel<64>, grid, dim3(kJoinThreads), 0, stream, true, p, l.o, l.lse, a.Hq, a.Hkv, a.G, a.T);
    if (e == cudaSuccess) *launched = 2;
    return e;
}

}  // namespace nsd
