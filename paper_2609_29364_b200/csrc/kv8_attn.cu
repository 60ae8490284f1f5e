// Attention over the 8-bit cache: the rows of a verification round, single tokens, short chunks, under a plan of its own kind
// (Section 3, block maps; Appendix G.2, the target's forward pass).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "chunk_walk.h"
#include "kv8_codec.h"
#include "nsd_internal.h"
#include "tcgen05_ops.h"

namespace nsd {
namespace {

// A unit is up to 40 stacked rows (tokens of one request times the G q heads of a kv head).  The keys sit on the tensor-memory
// lanes, the rows on the columns; per tile of 128 keys
//     S[128 keys x R]  = K Q^T       A = K's codes (e4m3, K-major), B = Q as three e5m2 terms
//     O[D x 3 R]      += V^T P^T     A = V's codes (MN-major), B = the weights as three e5m2 terms side by side
// so that the cache's bytes go from TMA to the tensor cores as they are.  No product is rounded: a bf16 query has eight
// significant bits and a 16-bit weight eleven, the three terms hold nine and eleven, and the accumulators are 32 bits.  The
// keys' powers of two are one number per lane: K's multiplies the scores, V's the weights before they are split.  The third
// term of a weight keeps its bits down to 2^-24 because the terms have columns of O of their own and may each have a scale.
// Rows on the lanes, as in the 16-bit kernels, would leave 100 of 128 lanes idle at the sizes this is for, and put the
// exponentials of 4 to 40 rows on one or two warps.
//
// The weights are 2^(s - m).  What has to stay within 16 bits is a weight times its key's power of two, so the reference m of
// a row is set by that product: in a piece's first tile so that the largest is 2^3, and moved only when one would pass 2^15.875
// (61440 is where an e5m2 term would round to infinity; all softmax warps vote in every tile).  A row thus keeps the keys that make up
// its output, whatever the V of keys that it gives no weight or does not see.  From 2^4 references would move twice as often (512
// requests of 3 to 5 rows over 128 to 4096 keys: 416 us instead of 404).  Sums of the weights are 32-bit and of the unrounded ones, a
// thread's own until the end of the piece.
// One reference for both serves while V's powers of two lie in 2^-60 to 2^40 (kLow, kHigh): a weight is then at most 2^76, and the
// sums of pieces can be joined in 32 bits.  A piece that meets another power where it sees to its references, or a score beyond 2^12
// (one rounding with a reference and one without would then differ by more than a weight's), goes on in wide form
// (wide_tile): the row's sum has a reference of its own (off), the products another (sh), both brought up to date in every tile, in
// a function apart from the others.  It takes two to three times as long (512 requests over 2048 keys: 1 row 793 us, 5 rows 1403).
//
// Two CTAs per SM, each a pipeline of its own with an equal share of the line (request, kv head, unit, key tile), twelve warps:
//   0-7   softmax: warp w has the keys of lane quarter w % 4 and one half of the rows; they also write the rows out
//   8     issues the MMAs: S of a tile ahead of P V of the one before it
//   9, 10 K (with the scales of K and V) and V, one TMA box per pool block, two stages each (four at D = 64)
//   11    Q of the next piece, and what the other warps have to know of it
// Pieces that a CTA boundary cuts leave their O and statistics in the plan, and chunk_join_kernel joins them in order.
//
// What bounds it: single tokens HBM (512 over 2048 keys each, 32 q heads and 8 kv heads of 128: 343 us = 6.3 TB/s, 0.98 of
// the copy rate; the 16-bit kernel reads twice the bytes); five rows per request the chain of a tile's softmax (412 us = 5.3
// TB/s; 3 to 5 rows over 128 to 4096 keys 413); ten rows (40 stacked) 124 us for 4 x 60 000 keys = 4.0 TB/s; 64 single tokens
// over 512 to 2048 keys 41 us, of which some 15 are the start, the last pieces and the join; 512 x 256 keys 102 us, with five rows
// 150: a piece of two or three tiles costs as much again in its beginning and end (its queries, the first references, rows out).
// D = 64 halves the bytes but not the softmax: 512 over 2048 keys 266 us, with five rows 373.  With up to four stacked rows (a token of
// four heads) half of the softmax warps have rows of padding only, which go through every step.  The instructions of a tile matter
// more than their number of cycles alone: with a longer loop (waits with time limits, eight rows of Q at a time, a fourth term) the
// SM's instruction cache no longer held it and times rose by a fifth.
//
// Tried: one CTA per SM with two streams over alternate tiles (1126 us; 668 with two CTAs); four warps for Q (516 instead of
// 499); S of a tile after P V of the one before (513 instead of 449); the wide form between the other tiles' instructions (357 and 439
// us for 1 and 5 rows over 2048 keys instead of 343 and 413); the look at the references as a function too (353 and 418).
//
// Every wait is bounded.  When one runs out, the CTA raises its abort flag; once all warps have left their loops, the issuer
// waits for its MMAs in flight and each producer for its copies (bounded again), and the call ends with STATUS_TIMEOUT.
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTileKeys = 128, kBs = 16, kBlocks = kTileKeys / kBs;
constexpr int kMaxRows = kKv8Kind.rows;
constexpr int kThreads = 384, kSoftThreads = 256;
constexpr int kWarpIssue = 8, kWarpV = 10, kWarpQ = 11;   // 9: the producer of K
constexpr uint32_t kPollLimit = 1u << 21;              // polls of one wait, if nsd_config.wait_budget does not say: one that finds nothing takes 1.4 us, so three seconds
constexpr float kTop = 3.f, kMost = 15.875f;           // log2 of a row's largest product when its reference is set, and at most
constexpr int kLow = -60, kHigh = 40;                  // exponents of V that one reference serves
constexpr float kFar = 4096.f;                         // scores that one reference serves: those beyond are rounded to more than 2^-12
constexpr float kMid = 8.f, kFine = 16.f;              // a weight's second term is held times kMid, its third times both
constexpr int kNoScale = -1000;                        // exponent of a V that no row sees, or that makes its rows NaN

__device__ __forceinline__ void report(int32_t* status, int32_t bit, int r) {
    atomicOr(status, bit);
    atomicCAS(status + 1, 0, r + 1);
}

struct Attn8Args {
    CUtensorMap kv_map;
    ChunkPlan p;
    const uint8_t* scales;
    const uint16_t* q;
    int64_t q_stride;
    uint16_t* o;
    float* lse;
    const int32_t* kv_indices;
    float sc;                                          // scale, in the log2 domain
    int32_t *status, Hq, Hkv, G, T, num_blocks;
    uint32_t wait_budget;
};

struct __align__(16) Meta {                            // a piece, beside its Q buffer
    int lo[kMaxRows], hi[kMaxRows];                    // visible keys
    int lo_max, hi_min;                                // keys [lo_max, hi_min) are visible to every row
    int n, rows;                                       // key tiles, -1 behind the last piece; stacked rows
    int row0, head, slot;                              // first token's row; kv head; partial slot or -1
    int key_first;                                     // of the first tile
    int key_lo, key_hi, gaps;                          // keys that some row sees: [key_lo, key_hi), unless there are gaps
    float c;                                           // sc 2^-k 2^-key_up, where the rows were multiplied by 2^k
    int key_up;                                        // what is added to a key's exponent instead: 7, less where c would leave the normal numbers
};
struct __align__(16) State {
    float neg[kMaxRows];                               // minus the reference of each row's weights
    float off[kMaxRows];                               // the row's sum is of weights 2^-off: 0, but in wide form; -inf: no key seen yet
    float sh[kMaxRows];                                // and its products of those times 2^sh: 0, but in wide form
    float sum[kMaxRows];                               // in wide form the row's sum so far
    float step[kMaxRows];                              // what the reference moves by
    float fac[kMaxRows];
    float top[4][kMaxRows];                            // a quarter's largest products or weights; at the end its sums
    volatile int odd, far, wide;                       // the piece has to go on in wide form, by a power of V or by a score; does so
    volatile int fail[2];                              // a warp has given up, by barriers in turn
};

template <int D>
struct Smem8 {
    static constexpr int kTile = kTileKeys * D;        // a K or V tile
    static constexpr int kBlock = kBs * D;
    static constexpr int kStages = D == 128 ? 2 : 4;   // of K, and of V
    static constexpr int kP = kTileKeys * 128;         // up to 128 columns, 16 at a time
    static constexpr int kQ = 3 * kMaxRows * D;
    static constexpr int kOffQ = kP;
    static constexpr int kOffK = (kOffQ + 2 * kQ + 1023) / 1024 * 1024, kOffV = kOffK + kStages * kTile;
    static constexpr int kOffScales = kOffV + kStages * kTile;          // [stage][block][K|V][16]
    static constexpr int kOffMeta = kOffScales + kStages * kBlocks * 32;
    static constexpr int kOffState = kOffMeta + 2 * (int)sizeof(Meta);
    static constexpr int kOffBars = kOffState + (int)sizeof(State);
    static constexpr int kNumBars = 4 * kStages + 2 * 3 + 3;
    static constexpr int kOffMisc = kOffBars + kNumBars * 8;
    static constexpr int kBytes = kOffMisc + 16;
    static constexpr int kSwizzle = D == 128 ? 2 : 4;  // rows of 128 or 64 bytes, swizzled over as much
    static_assert(2 * (kBytes + 1024) <= 228 * 1024, "two CTAs per SM");
};
constexpr int kTmemCols = 256, kTmemO = 128;           // two buffers of S, 64 columns apart, and O
// With up to 16 rows the three terms of S have columns of their own (four rows and three terms after another, as in P and O) and
// one pass over K serves them all: 512 single tokens over 2048 keys 341 us instead of 347, 64 over 512 to 2048 40 instead of 42.
// With more rows the sums of the terms cost the softmax warps more than two passes cost the tensor cores (5 rows 430 instead of
// 426): then they are summed where they lie.
constexpr int kApart = 16;

__device__ __forceinline__ float max_over_lanes(float v) {               // of those that are numbers
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// Four rows' values over the lanes of a warp: row j on lanes 8 j .. 8 j + 7.
template <typename Op>
__device__ __forceinline__ float over_lanes(float (&v)[4], int lane, Op op) {
#pragma unroll
    for (int k = 2; k > 0; k >>= 1) {
        const bool up = lane & (k * 8);
#pragma unroll
        for (int j = 0; j < k; ++j) {
            const float send = up ? v[j] : v[j + k], keep = up ? v[j + k] : v[j];
            v[j] = op(keep, __shfl_xor_sync(0xffffffffu, send, k * 8));
        }
    }
#pragma unroll
    for (int k = 4; k > 0; k >>= 1) v[0] = op(v[0], __shfl_xor_sync(0xffffffffu, v[0], k));
    return v[0];
}

// Pairs of 16-bit floats to the nearest ones of two mantissa bits (their upper bytes are then e5m2), and what is left, exactly.
__device__ __forceinline__ uint32_t upper(uint32_t h) { return (h + 0x00800080u) & 0xff00ff00u; }
__device__ __forceinline__ uint32_t minus(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t times(uint32_t a, float by) {
    const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), __float2half2_rn(by));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Four 16-bit floats in two words as three e5m2 terms each, four bytes per term: they sum to the value, exactly down to 2^-16,
// the format's least step.  FINE: the second term is held times 8 and the third times 128 (what is left is that much smaller),
// so that a value keeps its bits down to 2^-24, where 16-bit floats end.
template <bool FINE>
__device__ __forceinline__ void split4(uint32_t a, uint32_t b, uint32_t* terms) {
    const uint32_t a0 = upper(a), b0 = upper(b);
    uint32_t ra = minus(a, a0), rb = minus(b, b0);
    if constexpr (FINE) ra = times(ra, kMid), rb = times(rb, kMid);
    const uint32_t a1 = upper(ra), b1 = upper(rb);
    uint32_t a2 = minus(ra, a1), b2 = minus(rb, b1);
    if constexpr (FINE) a2 = times(a2, kFine), b2 = times(b2, kFine);
    a2 += 0x00800080u, b2 += 0x00800080u;
    terms[0] = __byte_perm(a0, b0, 0x7531);
    terms[1] = __byte_perm(a1, b1, 0x7531);
    terms[2] = __byte_perm(a2, b2, 0x7531);
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// 12 or 24 columns
__device__ __forceinline__ void tmem_ld_terms(uint32_t at, uint32_t (&r)[12]) { tmem_ld8(at, r), tmem_ld4(at + 8, r + 8); }
__device__ __forceinline__ void tmem_ld_terms(uint32_t at, uint32_t (&r)[24]) { tmem_ld16(at, r), tmem_ld8(at + 16, r + 16); }
// Waits for this thread's tensor-memory loads; their registers are operands, so that no use moves in front of the wait.
template <int N>
__device__ __forceinline__ void tmem_wait(uint32_t* r) {
    static_assert(N % 4 == 0, "four registers at a time");
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < N; i += 4) asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3])::"memory");
}
__device__ __forceinline__ bool any_of_softmax(bool p) {                 // over the softmax threads
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 2, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)p), "n"(kSoftThreads) : "memory");
    return r != 0;
}
__device__ __forceinline__ void softmax_sync() { asm volatile("barrier.cta.sync 2, %0;" ::"n"(kSoftThreads) : "memory"); }
__device__ __forceinline__ uint64_t bits2(uint32_t lo, uint32_t hi) { return pair(__uint_as_float(lo), __uint_as_float(hi)); }

__device__ __forceinline__ float best_of(const State& st, int r) { return fmaxf(fmaxf(st.top[0][r], st.top[1][r]), fmaxf(st.top[2][r], st.top[3][r])); }
__device__ __forceinline__ float sum_of(const State& st, int r) { return (st.top[0][r] + st.top[1][r]) + (st.top[2][r] + st.top[3][r]); }
// O, which holds a piece's earlier tiles: the rows of this thread's chunks times fac.
__device__ __forceinline__ void scale_rows(const State& st, uint32_t tmem_o, int r0, int chunks) {
#pragma unroll 1
    for (int ch = 0; ch < chunks; ++ch) {
        uint32_t o[12];
#pragma unroll
        for (int t = 0; t < 3; ++t) tmem_ld4(tmem_o + ch * 12 + t * 4, o + 4 * t);
        const float4 f = *reinterpret_cast<const float4*>(st.fac + r0 + ch * 4);
        const float by[4] = {f.x, f.y, f.z, f.w};
        tmem_wait<12>(o);
#pragma unroll
        for (int j = 0; j < 12; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * by[j & 3]);
#pragma unroll
        for (int t = 0; t < 3; ++t) tmem_st4(tmem_o + ch * 12 + t * 4, o + 4 * t);
    }
    tmem_wait_st();
}
// A tile in wide form, by all softmax threads: scores from S (in three terms, or summed), both references brought up to date, the
// tile's weights added to the rows' sums, and the products' exponents left where S was.  A function of its own, since the tiles of
// other pieces slow down by up to a tenth with this between them.  form: chunks of a thread; 8: the first such tile of a piece, the sums
// so far in top; 16: O holds earlier tiles.
__device__ __noinline__ void wide_tile(State& st, int form, uint32_t tmem_s, uint32_t tmem_o, float kk, float ev) {
    const int tid = threadIdx.x, lane = tid & 31, q = tid >> 5 & 3, chunks = form & 7, rows = chunks * 8, r0 = tid >> 7 ? rows / 2 : 0;
    const bool terms = rows <= kApart, enter = form & 8, later = form & 16;
    const int apart = terms ? 12 : 4;
    if (enter) {                                       // from here on neg is 0 and off all of the reference: scores are rounded alike in every tile
        softmax_sync();
        if (tid < rows) {
            st.sum[tid] = sum_of(st, tid);
            if (st.off[tid] != -INFINITY) st.off[tid] = -st.neg[tid];
            st.neg[tid] = 0.f;
        }
        softmax_sync();
    }
    bool first = false, still = false;                 // the row sees its first key; has seen none
    float by = 0.f;
    // Largest scores, which become the weights' references; sums of weights; largest products, against the row's so far, which are
    // smaller by as much as that reference has grown; and the products' exponents.
#pragma unroll 1
    for (int pass = 0; pass < 4; ++pass) {
#pragma unroll 1
        for (int ch = 0; ch < chunks; ++ch) {
            uint32_t y[4];
            float v[4];
            if (terms && pass == 0) {
                uint32_t t[12];
                tmem_ld_terms(tmem_s + ch * 12, t);
                tmem_wait<12>(t);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = __float_as_uint((__uint_as_float(t[j]) + __uint_as_float(t[4 + j])) + __uint_as_float(t[8 + j]));
            } else {
                tmem_ld4(tmem_s + ch * apart, y);
                tmem_wait<4>(y);
            }
            if (pass == 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * kk);
                tmem_st4(tmem_s + ch * apart, y);
                tmem_wait_st();
            }
            const float4 off = *reinterpret_cast<const float4*>(st.off + r0 + ch * 4), sh = *reinterpret_cast<const float4*>(st.sh + r0 + ch * 4);
            const float less[4] = {off.x, off.y, off.z, off.w}, more[4] = {sh.x, sh.y, sh.z, sh.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = __uint_as_float(y[j]) - (pass == 0 || less[j] == -INFINITY ? 0.f : less[j]);
                if (pass == 1) v[j] = ex2_approx(v[j]);
                if (pass >= 2) v[j] += ev + more[j];
                y[j] = __float_as_uint(v[j]);
            }
            if (pass == 3) {
                tmem_st4(tmem_s + ch * apart, y);
                continue;
            }
            const float all = over_lanes(v, lane, [&](float a, float b) { return pass == 1 ? a + b : fmaxf(a, b); });
            if ((lane & 7) == 0) st.top[q][r0 + ch * 4 + (lane >> 3)] = all;
        }
        if (pass == 3) break;
        softmax_sync();
        if (tid < rows) {
            if (pass == 0) {
                const float best = best_of(st, tid), was = st.off[tid];
                still = was == -INFINITY && best == -INFINITY, first = was == -INFINITY && !still;
                const float to = first ? best : fmaxf(was, best);
                by = first || still ? 0.f : to - was;
                st.off[tid] = to;
            } else if (pass == 1) {
                st.sum[tid] = (first ? 0.f : st.sum[tid] * ex2_approx(-by)) + sum_of(st, tid);
            } else {
                const float best = best_of(st, tid), up = still ? 0.f : (first ? best : fmaxf(best, kTop - by)) - kTop;
                st.sh[tid] -= up;
                st.fac[tid] = first ? 0.f : ex2_approx(-by - up);
            }
        }
        softmax_sync();
    }
    tmem_wait_st();
    if (later) scale_rows(st, tmem_o, r0, chunks);
}

// A CTA's walk over its share of the line, the next unit read ahead.
struct Walk8 {
    Walk w;
    ChunkUnit ahead;
    bool more;
    __device__ __forceinline__ Walk8(const ChunkPlan& p, int T, int Hkv) : w(p, T, Hkv), ahead{} { look(); }
    __device__ __forceinline__ void look() {
        more = !(w.at.unit == w.end.unit && w.at.head == w.end.head && w.at.tile == w.end.tile);
        if (more) ahead = w.units[w.at.unit];
    }
    __device__ __forceinline__ bool next() {
        if (!more) return false;
        w.step(ahead);
        look();
        return true;
    }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
kv8_attn_kernel(const __grid_constant__ Attn8Args a) {
    using L = Smem8<D>;
    constexpr int kStages = L::kStages;
    extern __shared__ __align__(1024) unsigned char smem[];
    pdl_release_dependents();
    const uint32_t smem0 = smem_u32(smem);
    if ((smem0 & 1023u) != 0) {
        pdl_wait();
        if (threadIdx.x == 0) atomicOr(a.status, STATUS_LAYOUT);
        return;
    }
    const uint32_t bar0 = smem0 + L::kOffBars;
    const uint32_t k_full = bar0, k_empty = k_full + 8 * kStages, v_full = k_empty + 8 * kStages, v_empty = v_full + 8 * kStages;
    const uint32_t q_full = v_empty + 8 * kStages, q_empty = q_full + 16, s_full = q_empty + 16;    // [2] per Q buffer, [2] per buffer of S
    const uint32_t p_full = s_full + 16, o_done = p_full + 8, flushed = o_done + 8;                 // an issuer's MMAs when it gives up
    Meta* const meta = reinterpret_cast<Meta*>(smem + L::kOffMeta);
    State& st = *reinterpret_cast<State*>(smem + L::kOffState);
    uint32_t& tmem_base_s = *reinterpret_cast<uint32_t*>(smem + L::kOffMisc);
    volatile int& abort_s = *reinterpret_cast<volatile int*>(smem + L::kOffMisc + 4);
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t limit = a.wait_budget ? a.wait_budget : kPollLimit;

    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(k_full + 8 * i, 1 + 16), mbar_init(k_empty + 8 * i, 8);
            mbar_init(v_full + 8 * i, 1), mbar_init(v_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) mbar_init(q_full + 8 * i, 1), mbar_init(q_empty + 8 * i, 1 + 8), mbar_init(s_full + 8 * i, 1);
        mbar_init(p_full, 8), mbar_init(o_done, 1), mbar_init(flushed, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        abort_s = 0;
        st.fail[0] = st.fail[1] = 0;
    }
    if (warp == kWarpIssue) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "n"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_s, 0);
    pdl_wait();                                        // from here on: what the kernel before writes
    // Waits for the count-th completion, bounded by a number of polls; the same answer in every lane.  Short, since it stands in
    // many places: what the warps of an SM execute has to stay near the size of its instruction cache.
    auto wait = [&](uint32_t bar, uint32_t count) {
        for (uint32_t i = 0; i < limit; ++i) {
            if (__all_sync(0xffffffffu, bar_try(bar, count & 1))) return true;
            if (__any_sync(0xffffffffu, abort_s)) return false;
        }
        abort_s = 1;
        return false;
    };
    auto ready = [&](uint32_t bar, uint32_t count) { return (bool)__all_sync(0xffffffffu, bar_try(bar, count & 1)); };
    // Behind this barrier every warp has left its loop and the abort flag is final.
    auto all_done = [] {
        __syncwarp();
        asm volatile("barrier.cta.sync 1, %0;" ::"n"(kThreads) : "memory");
    };
    auto columns = [](int rows) { return (rows + 7) & ~7; };                            // of one term
    // P and O: a warp's half of the rows, four rows and three terms after another, filled up to 16 columns
    auto half_columns = [](int rows) { return (3 * rows + 15) & ~15; };

    if (warp < kWarpIssue) {
        // ================================ softmax and output ================================
        // Launched with 384 x 80 registers: 256 x 88 + 128 x 64 of them.
        asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
        const int q = warp & 3, half = warp >> 2, key = q * 32 + lane;
        const uint32_t lanes = (uint32_t)(q * 32) << 16;
        // The warps meet at barriers that have no bound, so they have to leave together: one whose wait has run out goes on to
        // the next barrier, without waiting any more, and tells the others there.  A flag for every other barrier, since a
        // warp may be one ahead.
        bool fail = false;
        uint32_t turn = 0;
        auto hold = [&](uint32_t bar, uint32_t count) {
            if (!fail) fail = !wait(bar, count);
        };
        auto agreed = [&](bool p, bool& any) {         // whether all go on; any: p of any thread
            if (fail) st.fail[turn] = 1;
            any = any_of_softmax(p);
            fail = st.fail[turn] != 0;
            turn ^= 1;
            return !fail;
        };
        uint32_t n_t = 0;                              // tiles so far
        bool any, out = false;
        // A piece begins behind the barrier that ends the one before: its Q has been waited for there, and the references are anew.
        auto anew = [&](uint32_t n_q) {
            if (tid < kMaxRows) st.neg[tid] = st.sh[tid] = 0.f, st.off[tid] = -INFINITY;
            if (tid == 0) st.odd = st.far = st.wide = 0;
            hold(q_full + 8 * (n_q & 1), n_q >> 1);
            return agreed(false, any);
        };
        if (!anew(0)) out = true;
        for (uint32_t n_q = 0; !out; ++n_q) {
            const Meta& mt = meta[n_q & 1];
            const int n = mt.n, R = mt.rows, RP = columns(R), HP = RP / 2, r0 = half * HP;
            if (n < 0) break;
            const int G = a.G, part = mt.slot;
            if (n == 0) {                              // rows that see nothing; a piece of such a unit is the whole of it
                if (part < 0)
                    for (int r = warp; r < R; r += 8) {
                        const int64_t orow = (int64_t)(mt.row0 + r / G) * a.Hq + mt.head * G + r % G;
                        for (int d = lane; d < D; d += 32) a.o[orow * D + d] = 0;
                        if (a.lse && lane == 0) a.lse[orow] = -INFINITY;
                    }
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty + 8 * (n_q & 1));
                if (!anew(n_q + 1)) break;
                continue;
            }
            const int NH = half_columns(HP);
            const uint32_t tmem_o = tmem + kTmemO + lanes + half * NH;
            const uint32_t p_at = smem0 + half * (NH / 16) * (kTileKeys * 16) + key * 16;
            const int lo_max = mt.lo_max, hi_min = mt.hi_min;
            int key0 = mt.key_first;
            bool pending = true;                       // every tile sees to the references: some row has none yet, or the form is wide
            // A piece of NC chunks of four rows per thread, without a branch between them.
            auto tiles = [&](auto chunks) {
                constexpr int NC = decltype(chunks)::value;
                uint64_t l2[2 * NC];
#pragma unroll
                for (int i = 0; i < 2 * NC; ++i) l2[i] = 0;
                auto sum_rows = [&] {                  // over the lanes (a chunk's four rows end up on lanes 0, 8, 16, 24)
#pragma unroll
                    for (int ch = 0; ch < NC; ++ch) {
                        const float2 f0 = unpair(l2[ch * 2]), f1 = unpair(l2[ch * 2 + 1]);
                        float v[4] = {f0.x, f0.y, f1.x, f1.y};
                        const float sum = over_lanes(v, lane, [](float a, float b) { return a + b; });
                        if ((lane & 7) == 0) st.top[q][r0 + ch * 4 + (lane >> 3)] = sum;
                    }
                };
                for (int i = 0; i < n; ++i, ++n_t, key0 += kTileKeys) {
                    const uint32_t stage = n_t % kStages, use = n_t / kStages;
                    const int at = key0 + key;
                    const bool masked = key0 < lo_max || key0 + kTileKeys > hi_min;
                    bool seen = true;                  // by some row
                    if (masked) {
                        seen = at >= mt.key_lo && at < mt.key_hi;
                        if (mt.gaps) {
                            seen = false;
#pragma unroll 1
                            for (int r = 0; r < R; r += G) seen = seen || (at >= mt.lo[r] && at < mt.hi[r]);
                        }
                    }
                    hold(s_full + 8 * (n_t & 1), n_t >> 1);
                    tc_fence_after();
                    // The scales landed with K, before the issuer could send the product that s_full stands for.  (A look at k_full beside
                    // it costs 5 to 10 %.)
                    const unsigned char* const sb = smem + L::kOffScales + stage * (kBlocks * 32) + (key >> 4) * 32 + (key & 15);
                    const uint32_t kb = sb[0], vb = sb[16];
                    // The key's power of two, times 2^key_up against the rows' 2^-key_up, and theirs: not 0, so that a hidden score stays -inf,
                    // and finite, so that a score of 0 stays that.
                    const bool none = kb > 247 || vb > 247;
                    const float kk = none ? (masked ? 1.f : __uint_as_float(0x7fc00000u)) : fminf(fmaxf(__uint_as_float((uint32_t)max((int)kb + mt.key_up, 0) << 23) * mt.c, 1.17549435e-38f), 3.4e38f);
                    const uint64_t kk2 = pair(kk, kk);
                    int ev = seen && !none ? (int)vb - 127 : kNoScale;  // of a key that makes its rows NaN: nothing, for the other rows
                    const float look_at = ev < kHigh ? (float)max(ev, kLow) : 1000.f;   // beyond kMost with the largest weight: see to the references
                    constexpr bool kTerms = 8 * NC <= kApart;
                    const uint32_t tmem_s = tmem + (n_t & 1) * 64 + lanes + (kTerms ? 3 * r0 : r0);
                    // Scores are hidden where they lie, in a loop of its own: rare, and out of the way of the others.
                    if (masked) {
#pragma unroll 1
                        for (int k = 0; k < (kTerms ? 3 : 1) * NC; ++k) {
                            const int ch = kTerms ? k / 3 : k;
                            uint32_t y[4];
                            tmem_ld4(tmem_s + k * 4, y);
                            const int4 lo4 = *reinterpret_cast<const int4*>(mt.lo + r0 + ch * 4), hi4 = *reinterpret_cast<const int4*>(mt.hi + r0 + ch * 4);
                            const int lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, hi[4] = {hi4.x, hi4.y, hi4.z, hi4.w};
                            tmem_wait<4>(y);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                if (none) y[j] = 0x7fc00000u;
                                if (at < lo[j] || at >= hi[j]) y[j] = 0xff800000u;
                            }
                            tmem_st4(tmem_s + k * 4, y);
                        }
                        tmem_wait_st();
                    }
                    // The scores of this thread's key and rows less the rows' references, -inf where a row does not see the key.  (Product and
                    // difference become one instruction with one rounding.)
                    uint32_t x[4 * NC];
                    uint64_t sum[2 * NC];
                    if constexpr (kTerms) {
                        uint32_t y[12 * NC];
                        tmem_ld_terms(tmem_s, y);
                        tmem_wait<12 * NC>(y);
#pragma unroll
                        for (int k = 0; k < 2 * NC; ++k) {
                            const uint32_t* const v = y + (k >> 1) * 12 + (k & 1) * 2;
                            sum[k] = add2(add2(bits2(v[0], v[1]), bits2(v[4], v[5])), bits2(v[8], v[9]));
                        }
                    } else {
#pragma unroll
                        for (int ch = 0; ch < NC; ++ch) tmem_ld4(tmem_s + ch * 4, x + ch * 4);
                        tmem_wait<4 * NC>(x);
#pragma unroll
                        for (int k = 0; k < 2 * NC; ++k) sum[k] = bits2(x[2 * k], x[2 * k + 1]);
                    }
                    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int ch = 0; ch < NC; ++ch) {
                        const float4 m = *reinterpret_cast<const float4*>(st.neg + r0 + ch * 4);
                        const float2 f0 = unpair(add2(mul2(sum[2 * ch], kk2), pair(m.x, m.y))), f1 = unpair(add2(mul2(sum[2 * ch + 1], kk2), pair(m.z, m.w)));
                        x[ch * 4] = __float_as_uint(f0.x), x[ch * 4 + 1] = __float_as_uint(f0.y);
                        x[ch * 4 + 2] = __float_as_uint(f1.x), x[ch * 4 + 3] = __float_as_uint(f1.y);
                        top[0] = fmaxf(fmaxf(top[0], f0.x), f0.y), top[1] = fmaxf(fmaxf(top[1], f1.x), f1.y);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(k_empty + 8 * stage);                    // S is complete and the scales are read
                    if (fail) st.fail[turn] = 1;
                    any = any_of_softmax(fail || pending || fmaxf(top[0], top[1]) + look_at > kMost);
                    turn ^= 1;
                    // The references: in a piece's first tile, and in the rare ones where a product would leave the range of 16 bits, a
                    // weight or a power of two that of one reference, or some row has seen nothing yet.
                    if (any) {
                        if (st.fail[turn ^ 1]) {
                            fail = out = true;
                            break;
                        }
                        const bool enter = !st.wide;   // written behind a barrier that follows this
                        bool wide = !enter;
                        if (enter) {
                            if (ev > kNoScale && (ev < kLow || ev >= kHigh)) st.odd = 1;
#pragma unroll
                            for (int ch = 0; ch < NC; ++ch) {
                                float v[4];
#pragma unroll
                                for (int j = 0; j < 4; ++j) v[j] = max_over_lanes(__uint_as_float(x[ch * 4 + j]) + (float)ev);
                                if (lane == 0) *reinterpret_cast<float4*>(&st.top[q][r0 + ch * 4]) = make_float4(v[0], v[1], v[2], v[3]);
                            }
                            softmax_sync();
                            wide = st.odd;
                            if (!wide) {
                                bool still = false;
                                float neg = 0.f, off = 0.f;
                                if (tid < RP) {
                                    const float best = best_of(st, tid);
                                    neg = st.neg[tid], off = st.off[tid];
                                    const bool first = off == -INFINITY && best != -INFINITY;
                                    const float up = first || best > kTop ? best - kTop : 0.f;
                                    if (fabsf(neg - up) > kFar) st.far = 1;
                                    st.neg[tid] = neg - up;
                                    st.step[tid] = up;
                                    st.fac[tid] = first ? 0.f : ex2_approx(-up);
                                    if (first) st.off[tid] = 0.f;
                                    still = off == -INFINITY && !first;
                                }
                                pending = any_of_softmax(still);
                                wide = st.far;
                                if (wide && tid < RP) st.neg[tid] = neg, st.off[tid] = off;              // as they were
                            }
                        }
                        if (!wide) {
                            if (i > 0) {
#pragma unroll
                                for (int j = 0; j < 2 * NC; ++j) {
                                    const float2 f = *reinterpret_cast<const float2*>(st.fac + r0 + 2 * j);
                                    l2[j] = mul2(l2[j], pair(f.x, f.y));
                                }
                                hold(o_done, n_t - 1);
                                tc_fence_after();
                                scale_rows(st, tmem_o, r0, NC);
                            }
#pragma unroll
                            for (int ch = 0; ch < NC; ++ch) {
                                const float4 up = *reinterpret_cast<const float4*>(st.step + r0 + ch * 4);
                                x[ch * 4] = __float_as_uint(__uint_as_float(x[ch * 4]) - up.x), x[ch * 4 + 1] = __float_as_uint(__uint_as_float(x[ch * 4 + 1]) - up.y);
                                x[ch * 4 + 2] = __float_as_uint(__uint_as_float(x[ch * 4 + 2]) - up.z), x[ch * 4 + 3] = __float_as_uint(__uint_as_float(x[ch * 4 + 3]) - up.w);
                            }
                        } else {
                            // In place of S, which the issuer leaves alone until the weights are there.
                            if (enter) sum_rows();
                            if (i > 0) hold(o_done, n_t - 1);
                            tc_fence_after();
                            wide_tile(st, NC | (enter ? 8 : 0) | (i > 0 ? 16 : 0), tmem_s, tmem_o, kk, (float)ev);
#pragma unroll
                            for (int ch = 0; ch < NC; ++ch) tmem_ld4(tmem_s + ch * (kTerms ? 12 : 4), x + ch * 4);
                            tmem_wait<4 * NC>(x);
                            if (tid == 0) st.wide = 1;
                            pending = true;
                            ev = 0;                    // of a product only 2^x is left
#pragma unroll
                            for (int j = 0; j < 2 * NC; ++j) l2[j] = 0;                 // no longer counts
                        }
                    }
                    const bool p_free = i == 0 || bar_try(o_done, (n_t - 1) & 1);       // looked at here, needed below
                    // weights: their sums in 32 bits; times V's power of two, and split, for the product
                    constexpr int kUnits = (3 * NC + 3) / 4;
                    uint32_t word[4 * kUnits] = {};
                    const float vs = __uint_as_float((uint32_t)(min(max(ev, -126), 127) + 127) << 23);
                    const uint64_t vs2 = pair(vs, vs);
#pragma unroll
                    for (int ch = 0; ch < NC; ++ch) {
                        uint32_t h[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint64_t p = pair(ex2_approx(__uint_as_float(x[ch * 4 + 2 * j])), ex2_approx(__uint_as_float(x[ch * 4 + 2 * j + 1])));
                            l2[ch * 2 + j] = add2(l2[ch * 2 + j], p);
                            const float2 wv = unpair(mul2(p, vs2));
                            h[j] = pack_half(wv.x, wv.y);
                        }
                        split4<true>(h[0], h[1], word + 3 * ch);
                    }
                    if (!__all_sync(0xffffffffu, p_free)) hold(o_done, n_t - 1);        // P V of the tile before has read P
#pragma unroll
                    for (int k = 0; k < kUnits; ++k)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(p_at + k * (kTileKeys * 16)), "r"(word[4 * k]), "r"(word[4 * k + 1]), "r"(word[4 * k + 2]), "r"(word[4 * k + 3]) : "memory");
                    // Hidden rows of V have to be finite, since 0 x NaN is NaN.
                    if (masked) {
                        hold(v_full + 8 * stage, use);
                        if (!seen && half == 0) {
                            const uint32_t row = smem0 + L::kOffV + stage * L::kTile + key * D;
#pragma unroll 1
                            for (int ch = 0; ch < D / 16; ++ch)
                                asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(row + ((ch + lane) % (D / 16)) * 16), "r"(0) : "memory");
                        }
                    }
                    fence_async_smem();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full);
                }
                sum_rows();
            };
            const int n_ch = HP / 4;
            // A round's units alternate between neighbouring sizes, and an SM's instruction cache holds two of these loops or not by where
            // they lie: neighbours stand apart (512 requests of 3 to 5 rows over 128 to 4096 keys 426 us, 459 in order of size; of 2 to 6
            // over 2048 keys 480 and 499).
            if (n_ch == 2) tiles(std::integral_constant<int, 2>());
            else if (n_ch == 5) tiles(std::integral_constant<int, 5>());
            else if (n_ch == 3) tiles(std::integral_constant<int, 3>());
            else if (n_ch == 1) tiles(std::integral_constant<int, 1>());
            else tiles(std::integral_constant<int, 4>());
            if (out) break;
            // ---- the piece's rows; what needs no product, while the last one is under way
            softmax_sync();
            const int64_t part0 = (int64_t)part * kMaxRows, orow0 = (int64_t)mt.row0 * a.Hq + mt.head * G;
            if (tid < R) {
                const float m_run = st.off[tid] - st.neg[tid], l = st.wide ? st.sum[tid] : sum_of(st, tid), a_o = -st.sh[tid];
                float f = 0.f, more = 1.f;             // a sum of zero: nothing was seen, O may be anything
                // What the products' reference differs by is shared out, half each: between a piece's sum and its products (f), so that both
                // stay in range wherever V lies, or between the two factors of a row.  A row whose sum is no number joins with a reference
                // of infinity: all factors are then 0 or not a number.
                if (part >= 0) {
                    const float m = m_run + 0.5f * a_o, by = m - m_run;                 // by: what it has moved by after its rounding
                    if (l != 0.f) f = l == l ? ex2_approx(a_o - by) : l;
                    *reinterpret_cast<float2*>(a.p.part_ml + (part0 + tid) * 2) = make_float2(l != l ? INFINITY : (l == 0.f ? -INFINITY : m), l != 0.f ? l * ex2_approx(-by) : 0.f);
                } else {
                    if (l != 0.f) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(f) : "f"(l));
                    more = ex2_approx(0.5f * a_o);
                    f *= more;
                    if (a.lse) a.lse[orow0 + (tid / G) * a.Hq + tid % G] = l == 0.f ? -INFINITY : (m_run + log2f(l)) * kLn2;
                }
                st.fac[tid] = f;
                st.step[tid] = more;
            }
            hold(o_done, n_t - 1);
            if (!anew(n_q + 1)) break;
            tc_fence_after();
            // O is [dim][half, chunk, term, row]: a thread has one dim (64 dims sit on 16 lanes of each quarter) and its half of the rows
            const bool live = D == 128 || lane < 16, whole = part < 0;
            int g = r0 % G;
            const int size = whole ? 2 : 4, jump = whole ? (a.Hq - G) * D * 2 : 0;      // bytes of a value; from a token's last row of the head to the next one's first
            char* to = whole ? reinterpret_cast<char*>(a.o + (orow0 + (int64_t)(r0 / G) * a.Hq + g) * D) : reinterpret_cast<char*>(a.p.part_acc + (part0 + r0) * D);
            to += (D == 128 ? key : q * 16 + lane) * size;
#pragma unroll 1
            for (int ch = 0; ch < n_ch; ++ch) {
                if (r0 + ch * 4 >= R) break;
                uint32_t y[12];
#pragma unroll
                for (int t = 0; t < 3; ++t) tmem_ld4(tmem_o + ch * 12 + t * 4, y + 4 * t);
                const float4 f4 = *reinterpret_cast<const float4*>(st.fac + r0 + ch * 4), g4 = *reinterpret_cast<const float4*>(st.step + r0 + ch * 4);
                const float f[4] = {f4.x, f4.y, f4.z, f4.w}, more[4] = {g4.x, g4.y, g4.z, g4.w};
                tmem_wait<12>(y);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float sum = fmaf(fmaf(__uint_as_float(y[8 + j]), 1.f / kFine, __uint_as_float(y[4 + j])), 1.f / kMid, __uint_as_float(y[j]));
                    const float v = f[j] != 0.f ? sum * f[j] * more[j] : 0.f;
                    if (live && r0 + ch * 4 + j < R) {
                        if (whole) {
                            const __nv_bfloat16 b = __float2bfloat16_rn(v);
                            *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(&b);
                        } else {
                            *reinterpret_cast<float*>(to) = v;
                        }
                    }
                    to += D * size;
                    if (++g == G) g = 0, to += jump;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_empty + 8 * (n_q & 1));
        }
        all_done();
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == kWarpIssue) {
        // ================================ MMA issuer ================================
        // S of a tile goes before P V of the tile before it, also from one piece to the next, so that it is there when the
        // softmax warps come to it.
        const uint64_t dp = smem_desc(smem0, 128, kTileKeys * 16, 0);
        uint32_t n_s = 0, n_p = 0, n_q = 0;            // tiles whose S has gone, whose P V has gone; pieces begun
        int i = 0, n = 0, RP = 0;                      // next tile of the piece whose S is under way
        bool ok = true, end = false;
        auto begin = [&] {                             // the next piece with tiles
            for (;;) {
                if (!(ok = wait(q_full + 8 * (n_q & 1), n_q >> 1))) return;
                const Meta& mt = meta[n_q & 1];
                n = __shfl_sync(0xffffffffu, mt.n, 0), RP = __shfl_sync(0xffffffffu, columns(mt.rows), 0);
                ++n_q;
                i = 0;
                if (n < 0) end = true;
                if (n != 0) return;
                if (lane == 0) mbar_arrive(q_empty + 8 * ((n_q - 1) & 1));
            }
        };
        auto issue_s = [&] {
            const uint32_t stage = n_s % kStages, slot = (n_q - 1) & 1;
            if (!(ok = wait(k_full + 8 * stage, n_s / kStages))) return;
            tc_fence_after();
            const bool apart = RP <= kApart;
            const uint32_t idesc = instr_desc_f8(kTileKeys, ((apart ? 3 * RP : RP) + 15) & ~15, 0, 0);
            const uint64_t dk = smem_desc(smem0 + L::kOffK + stage * L::kTile, 16, 8 * D, L::kSwizzle);
            const uint64_t dq = smem_desc(smem0 + L::kOffQ + slot * L::kQ, 16, 8 * D, L::kSwizzle);
            if (elect_one()) {
#pragma unroll 1
                for (int t = 0; t < (apart ? 1 : 3); ++t)
#pragma unroll
                    for (int k = 0; k < D / 32; ++k)                                    // 32 dims each
                        umma_ss_f8(tmem + (n_s & 1) * 64, dk + 2 * k, dq + ((t * RP * D) >> 4) + 2 * k, idesc, t > 0 || k > 0);
                umma_commit(s_full + 8 * (n_s & 1));
                if (i + 1 == n) umma_commit(q_empty + 8 * slot);
            }
            ++n_s, ++i;
        };
        begin();
        if (ok && !end) issue_s();
        bool fresh = true;                             // the next P V is the first of its piece
        int rp = RP;                                   // of the piece whose P V is next
        while (ok && n_p < n_s) {
            const bool last = i == n;                  // the tile whose P V is next is the last of its piece
            // S of the next tile first, if K is there: P V does not wait for it
            bool gone = last;
            if (!last && ready(k_full + 8 * (n_s % kStages), n_s / kStages)) {
                issue_s();
                gone = true;
            }
            const uint32_t stage = n_p % kStages;
            if (!(ok = wait(v_full + 8 * stage, n_p / kStages)) || !(ok = wait(p_full, n_p))) break;
            tc_fence_after();
            const uint32_t idesc = instr_desc_f8(D, 2 * half_columns(rp / 2), 1, 1);
            const uint64_t dv = smem_desc(smem0 + L::kOffV + stage * L::kTile, 16, 8 * D, L::kSwizzle);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < kTileKeys / 32; ++k)                                // 32 keys each
                    umma_ss_f8(tmem + kTmemO, dv + ((k * 32 * D) >> 4), dp + ((k * 32 * 16) >> 4), idesc, (!fresh || k > 0) ? 1u : 0u);
                umma_commit(v_empty + 8 * stage);
                umma_commit(o_done);
            }
            ++n_p;
            fresh = false;
            if (!gone) {
                issue_s();
            } else if (last && !end) {
                begin();
                if (!ok || end) break;
                issue_s();
                fresh = true, rp = RP;
            }
        }
        all_done();
        if (abort_s) {
            // the CTA is giving up: what is still in flight reads shared memory and writes tensor memory
            if (elect_one()) umma_commit(flushed);
            const long long t0 = clock64();
            while (!bar_try(flushed, 0) && clock64() - t0 < kWaitCycles) {}
        }
    } else if (warp < kWarpQ) {
        // ================================ K and V producers ================================
        const bool is_v = warp == kWarpV;
        const uint32_t full = is_v ? v_full : k_full, empty = is_v ? v_empty : k_empty;
        const uint32_t ring = smem0 + (is_v ? L::kOffV : L::kOffK);
        const int32_t oob = a.num_blocks * 2 * a.Hkv;                                   // past the slab: zero fill
        uint32_t n_t = 0;
        bool ok = true;
        Walk8 walk(a.p, a.T, a.Hkv);
        const Walk& w = walk.w;
        while (ok && walk.next()) {
            const int n = w.k1 - w.k0;
            if (n == 0) continue;
            const int32_t* table = a.kv_indices + w.u.tbl;
            const int b_lo = w.u.key_lo / kBs, b_hi = (w.u.key_hi + kBs - 1) / kBs;     // blocks that hold a visible key
            const int t0 = w.u.key_lo / kTileKeys + w.k0;                               // first key tile
            // the block of a tile whose copy this lane sends: its id is read one tile ahead
            auto block_id = [&](int t) -> int32_t {
                const int b = t * kBlocks + lane;
                if (lane >= kBlocks || b < b_lo || b >= b_hi) return -2;                // not needed
                return b < w.u.nblk ? __ldg(table + b) : -1;
            };
            int32_t id_next = block_id(t0);
            for (int i = 0; i < n; ++i) {
                const uint32_t stage = n_t % kStages, use = n_t / kStages;
                const int32_t id = id_next;
                if (i + 1 < n) id_next = block_id(t0 + i + 1);
                const bool good = (uint32_t)id < (uint32_t)a.num_blocks;
                if (!good && id != -2) report(a.status, STATUS_BAD_BLOCK, w.u.req);
                if (use > 0 && !(ok = wait(empty + 8 * stage, use - 1))) break;
                const uint32_t bar = full + 8 * stage;
                if (lane == 0) mbar_expect_tx(bar, L::kTile);
                __syncwarp();
                if (lane < kBlocks) tma_load_3d(ring + stage * L::kTile + lane * L::kBlock, &a.kv_map, 0, 0, good ? (id * 2 + (is_v ? 1 : 0)) * a.Hkv + w.head : oob, bar);
                if (!is_v) {
                    // the scales of K and V: two pieces of 16 bytes per block, zeros for a block that is not read
                    const int32_t sid = __shfl_sync(0xffffffffu, good ? id : -1, lane >> 1);
                    if (lane < 2 * kBlocks) {
                        const uint8_t* const src = a.scales + (sid < 0 ? 0 : (((int64_t)sid * a.Hkv + w.head) * 2 + (lane & 1)) * kBs);
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem0 + L::kOffScales + stage * (kBlocks * 32) + lane * 16), "l"(src), "r"(sid < 0 ? 0 : 16) : "memory");
                        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
                    }
                }
                ++n_t;                                                                  // from here on the tile is in flight, whatever gives up next
            }
        }
        all_done();
        if (abort_s && lane == 0) {
            // the CTA is giving up: copies that nobody waited for may still be landing
            for (uint32_t back = 1; back <= (uint32_t)kStages && back <= n_t; ++back) {
                const uint32_t c = n_t - back;
                const long long t0 = clock64();
                while (!bar_try(full + 8 * (c % kStages), (c / kStages) & 1) && clock64() - t0 < kWaitCycles) {}
            }
        }
    } else {
        // ================================ Q and the pieces ================================
        // The rows times the power of two that brings their largest element to [2^14, 2^15), split into three e5m2 terms: rows
        // of the product's second operand, in the order of S's columns.  bf16 has eight significant bits, the terms nine: nothing
        // is lost but what lies below 2^-16 then.
        constexpr int kLanes = D / 8, kStep = 32 / kLanes;                              // lanes of a row, eight elements each; rows at a time
        const int sub = lane / kLanes, d = lane % kLanes;
        const uint32_t inv_G = (65536 + a.G - 1) / a.G;                                 // r / G for the few rows there are
        const int64_t gap = a.q_stride - a.G * D;                                       // from a token's last row of the head to the next one's first
        uint32_t n_q = 0;
        bool ok = true;
        Walk8 walk(a.p, a.T, a.Hkv);
        const Walk& w = walk.w;
        const bool causal = w.planned && a.p.header->causal;
        if (!w.planned && blockIdx.x == 0 && lane == 0) report(a.status, STATUS_BAD_TOKEN, -1);
        for (;;) {
            const bool piece = walk.next();
            // The next piece's rows towards the L2: this warp takes 2 to 7 us for a piece, most of it waiting for them (512 requests of
            // 5 rows over 128 keys 113 us instead of 130).
            if (walk.more && lane < walk.ahead.ntok)
                asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(a.q + (walk.ahead.row0 + lane) * a.q_stride + w.at.head * a.G * D), "r"(a.G * D * 2) : "memory");
            const int slot = n_q & 1, R = piece ? w.u.ntok * a.G : 0, RP = columns(R);
            const uint32_t qb = smem0 + L::kOffQ + slot * L::kQ;
            Meta& mt = meta[slot];
            const uint16_t* const q0 = a.q + (int64_t)w.u.row0 * a.q_stride + w.head * a.G * D + d * 8;
            auto read = [&](int r) {
                if (r >= R) return make_uint4(0, 0, 0, 0);
                return __ldg(reinterpret_cast<const uint4*>(q0 + r * D + ((r * inv_G) >> 16) * gap));
            };
            const bool tiles = piece && w.k1 > w.k0;
            uint32_t big = 0;                          // magnitude bits of the largest element
            uint4 ahead[2] = {};
            if (tiles) {                               // while the buffer is not free yet
#pragma unroll 1
                for (int first = 0; first < R; first += 4 * kStep) {
                    uint4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = read(first + i * kStep + sub);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        big = __vmaxu2(big, __vmaxu2(__vmaxu2(v[i].x & 0x7fff7fffu, v[i].y & 0x7fff7fffu), __vmaxu2(v[i].z & 0x7fff7fffu, v[i].w & 0x7fff7fffu)));
                }
                big = __reduce_max_sync(0xffffffffu, max(big & 0xffffu, big >> 16));
                ahead[0] = read(sub), ahead[1] = read(sub + kStep);
            }
            const bool odd = big >= 0x7f80u;           // some value is no number: the largest of the others
            if (odd) {
                big = 0;
#pragma unroll 1
                for (int first = 0; first < R; first += kStep) {
                    const uint4 v = read(first + sub);
                    const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t m = word[j >> 1] >> (16 * (j & 1)) & 0x7fffu;
                        big = max(big, m < 0x7f80u ? m : 0u);
                    }
                }
                big = __reduce_max_sync(0xffffffffu, big);
            }
            const int k = min(141 - max((int)(big >> 7), 1), 127);
            const float f = __uint_as_float((uint32_t)(k + 127) << 23);
            if (n_q >= 2 && !(ok = wait(q_empty + 8 * slot, (n_q >> 1) - 1))) break;
            if (tiles) {
                // A row's 16-byte pieces are exchanged by its number (the swizzle), of which a term changes one bit at most.
                const bool apart = RP <= kApart;
                const uint32_t term = (apart ? 4 : RP) * D, flip = apart ? D / 2 : 0;
                auto place = [&](int r) {
                    const int row = apart ? 3 * (r & ~3) + (r & 3) : r;
                    return qb + row * D + (((d >> 1) ^ (D == 128 ? row & 7 : row >> 1 & 3)) << 4) + (d & 1) * 8;
                };
#pragma unroll 1
                for (int first = 0; first < RP; first += 2 * kStep) {                   // two rows per lane: one hides the other's latency
                    const uint4 now[2] = {ahead[0], ahead[1]};
#pragma unroll
                    for (int i = 0; i < 2; ++i) ahead[i] = read(first + (2 + i) * kStep + sub);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t word[4] = {now[i].x, now[i].y, now[i].z, now[i].w};
                        uint32_t h[4], t0[3], t1[3];
#pragma unroll
                        for (int j = 0; j < 4; ++j) h[j] = pack_half(__uint_as_float(word[j] << 16) * f, __uint_as_float(word[j] & 0xffff0000u) * f);
                        split4<false>(h[0], h[1], t0);
                        split4<false>(h[2], h[3], t1);
                        const uint32_t to = place(first + i * kStep + sub);
#pragma unroll
                        for (int t = 0; t < 3; ++t)
                            asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"((t == 1 ? to ^ flip : to) + t * term), "r"(t0[t]), "r"(t1[t]) : "memory");
                    }
                }
                if (odd) {                             // a row with such a value is none: not a number in all its elements
#pragma unroll 1
                    for (int first = 0; first < R; first += kStep) {
                        const uint4 v = read(first + sub);
                        const uint32_t word[4] = {v.x, v.y, v.z, v.w};
                        bool none = false;
#pragma unroll
                        for (int j = 0; j < 4; ++j) none = none || (word[j] & 0x7fffu) >= 0x7f80u || (word[j] >> 16 & 0x7fffu) >= 0x7f80u;
                        if (__ballot_sync(0xffffffffu, none) >> (sub * kLanes) & (uint32_t)((1ull << kLanes) - 1))
                            asm volatile("st.shared.v2.b32 [%0], {%1, %1};" ::"r"(place(first + sub)), "r"(0x7f7f7f7f) : "memory");
                    }
                }
                int lo_max = 0, hi_min = 0x7fffffff;
                for (int r = lane; r < RP; r += 32) {
                    int lo = 0, hi = 0x7fffffff;       // rows of padding never mask
                    if (r < R) {
                        const int t = (r * inv_G) >> 16;
                        if (causal) hi = w.u.pos0 + t + 1;
                        else lo = a.p.row_lo[w.u.row0 + t], hi = a.p.row_hi[w.u.row0 + t];
                    }
                    mt.lo[r] = lo, mt.hi[r] = hi;
                    lo_max = max(lo_max, lo), hi_min = min(hi_min, hi);
                }
                lo_max = __reduce_max_sync(0xffffffffu, lo_max), hi_min = __reduce_min_sync(0xffffffffu, hi_min);
                if (lane == 0) mt.lo_max = lo_max, mt.hi_min = hi_min;
            }
            if (lane == 0) {
                mt.n = piece ? w.k1 - w.k0 : -1, mt.rows = R;
                // Queries near the least numbers under a small scale: c keeps its bits, the keys' exponents take what it would fall below
                // the normal numbers by (keys so small that theirs then fall below add nothing to a score).
                const int least = (int)(__float_as_uint(a.sc) >> 23) - 127 - k - 7, under = max(-126 - least, 0);
                const int d0 = (under - k - 7) >> 1, d1 = under - k - 7 - d0;           // sc 2^(-k - 7 + under)
                mt.c = a.sc * __uint_as_float((uint32_t)(d0 + 127) << 23) * __uint_as_float((uint32_t)(d1 + 127) << 23);
                mt.key_up = 7 - under;
                if (piece) mt.row0 = w.u.row0, mt.head = w.head, mt.slot = w.slot, mt.key_first = (w.u.key_lo / kTileKeys + w.k0) * kTileKeys, mt.key_lo = w.u.key_lo, mt.key_hi = w.u.key_hi, mt.gaps = w.u.gaps;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full + 8 * slot);
            ++n_q;
            if (!piece) break;
        }
        all_done();
    }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kWarpIssue) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemCols) : "memory");
    if (tid == 0 && abort_s) atomicOr(a.status, STATUS_TIMEOUT);
}

// A slab as [tile = (block, K|V, kv head)][key][dim]; the box is one tile.
bool kv8_map(CUtensorMap* map, const void* slab, const Shape& s) {
    typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const EncodeFn encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) fn = nullptr;
        return reinterpret_cast<EncodeFn>(fn);
    }();
    const cuuint64_t D = s.D, dims[3] = {D, kBs, (cuuint64_t)s.num_blocks * 2 * s.Hkv}, strides[2] = {D, kBs * D};
    const cuuint32_t box[3] = {(cuuint32_t)D, kBs, 1}, ones[3] = {1, 1, 1};
    return encode && encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(slab), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t kv8_attn_init() {
    const cudaError_t e = cudaFuncSetAttribute(kv8_attn_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem8<128>::kBytes);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(kv8_attn_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem8<64>::kBytes);
}

cudaError_t launch_kv8_attn(const ChunkPlan& p, const Kv8AttnLaunch& l, cudaStream_t stream, int* launched) {
    Attn8Args a{};
    if (!kv8_map(&a.kv_map, l.codes, l.shape)) return cudaErrorNotSupported;
    a.p = p;
    a.scales = l.scales, a.q = l.q, a.q_stride = l.q_stride, a.o = l.o, a.lse = l.lse, a.kv_indices = l.kv_indices;
    a.sc = l.scale * kLog2e;
    a.status = l.status;
    a.Hq = l.shape.Hq, a.Hkv = l.shape.Hkv, a.G = a.Hq / a.Hkv, a.T = p.kind.tokens(a.G), a.num_blocks = l.shape.num_blocks;
    a.wait_budget = l.wait_budget;
    const dim3 grid(p.n_ctas), block(kThreads);
    cudaError_t e = l.shape.D == 128 ? launch_kernel(kv8_attn_kernel<128>, grid, block, Smem8<128>::kBytes, stream, true, a)
                                     : launch_kernel(kv8_attn_kernel<64>, grid, block, Smem8<64>::kBytes, stream, true, a);
    if (e != cudaSuccess) return e;
    *launched = 1;
    if (p.n_ctas < 2) return e;
    e = launch_chunk_join(p, l.shape, l.o, l.lse, stream);
    if (e == cudaSuccess) *launched = 2;
    return e;
}

}  // namespace nsd
