// Attention over the 8-bit cache: the rows of a verification round, single tokens, short chunks, under a plan of its own kind
// (Section 3, block maps; Appendix G.2, the target's forward pass).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "chunk_walk.h"
#include "kv8_codec.h"
#include "nsd_internal.h"
#include "tcgen05_ops.h"

namespace nsd {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTileKeys = 128, kBs = 16, kBlocks = kTileKeys / kBs;
constexpr int kMaxRows = kKv8Kind.rows, kChunks = kMaxRows / 8;
constexpr int kThreads = 512;
constexpr int kWarpIssue = 8, kWarpK = 10, kWarpV = 11, kWarpQ = 12;
constexpr uint32_t kPollLimit = 1u << 30;              // polls of one wait, if nsd_config.wait_budget does not say
constexpr float kTop = 10.f, kMost = 15.f;             // log2 of a row's largest weight when its reference is set, and at most
constexpr int kNoScale = -1000;                        // exponent of V's reference before any

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

struct Meta {                                          // what a piece's Q buffer comes with
    float c[kMaxRows];                                 // sc 2^-k 2^-7, where the row was multiplied by 2^k; NaN for a row with a value that is no number
    int lo[kMaxRows], hi[kMaxRows];                    // visible keys
    int lo_max, hi_min;                                // keys [lo_max, hi_min) are visible to every row
};
struct State {                                         // of the two softmax streams
    float neg[2][kMaxRows];                            // minus the reference of each row's weights
    float fac[2][kMaxRows];
    float top[2][4][kMaxRows];                         // a warp's largest scores; at the end its sums
    int exp_top[2][4];
    float2 ml[2][kMaxRows];                            // reference and sum, for the stream that joins
    int exp_ref[2];
    float2 join[2][kMaxRows];                          // factors of the two streams' O
    volatile int fail[2][2];                           // a warp of the stream has given up, by barriers in turn
};

template <int D>
struct Smem8 {
    static constexpr int kTile = kTileKeys * D;        // a K or V tile
    static constexpr int kBlock = kBs * D;
    static constexpr int kStages = D == 128 ? 4 : 8;   // of K, and of V; even: a stage always serves the same stream
    static constexpr int kP = kTileKeys * 128;         // up to 128 columns, 16 at a time
    static constexpr int kQ = 3 * kMaxRows * D;
    static constexpr int kOffQ = 2 * kP;
    static constexpr int kOffK = (kOffQ + 2 * kQ + 1023) / 1024 * 1024, kOffV = kOffK + kStages * kTile;
    static constexpr int kOffScales = kOffV + kStages * kTile;          // [stage][block][K|V][16]
    static constexpr int kOffMeta = kOffScales + kStages * kBlocks * 32;
    static constexpr int kOffState = kOffMeta + (2 * (int)sizeof(Meta) + 15) / 16 * 16;
    static constexpr int kOffBars = kOffState + ((int)sizeof(State) + 15) / 16 * 16;
    static constexpr int kNumBars = 4 * kStages + 2 * 2 + 2 * 6;
    static constexpr int kOffMisc = kOffBars + kNumBars * 8;
    static constexpr int kBytes = kOffMisc + 16;
    static constexpr int kSwizzle = D == 128 ? 2 : 4;  // rows of 128 or 64 bytes, swizzled over as much
    static_assert(kBytes <= 227 * 1024, "shared memory budget");
    static_assert(kOffMeta % 16 == 0 && sizeof(Meta) % 8 == 0, "rows are read four at a time");
};
constexpr int kTmemCols = 512, kTmemO = 256;           // S0, S1, O0, O1: 128 columns each

__device__ __forceinline__ int ordered(float x) {      // an integer that grows with x; NaN above everything
    const int b = __float_as_int(x);
    return x != x ? 0x7fffffff : b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b ^ ((b >> 31) & 0x7fffffff)); }

// Pairs of 16-bit floats to the nearest ones of two mantissa bits (their upper bytes are then e5m2), and what is left, exactly.
__device__ __forceinline__ uint32_t upper(uint32_t h) { return (h + 0x00800080u) & 0xff00ff00u; }
__device__ __forceinline__ uint32_t minus(uint32_t a, uint32_t b) {
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Four 16-bit floats in two words as three e5m2 terms each, four bytes per term: term by term they sum to the value, exactly
// down to 2^-16, the format's least step.
__device__ __forceinline__ void split4(uint32_t a, uint32_t b, uint32_t* terms) {
    const uint32_t a0 = upper(a), b0 = upper(b);
    const uint32_t ra = minus(a, a0), rb = minus(b, b0), a1 = upper(ra), b1 = upper(rb);
    const uint32_t a2 = minus(ra, a1) + 0x00800080u, b2 = minus(rb, b1) + 0x00800080u;
    terms[0] = __byte_perm(a0, b0, 0x7531);
    terms[1] = __byte_perm(a1, b1, 0x7531);
    terms[2] = __byte_perm(a2, b2, 0x7531);
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Waits for this thread's tensor-memory loads; their registers are operands, so that no use moves in front of the wait.
__device__ __forceinline__ void tmem_wait_ld24(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                   "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                   "+r"(r[21]), "+r"(r[22]), "+r"(r[23])::"memory");
}
__device__ __forceinline__ bool any_of_stream(int s, bool p) {           // over the 128 threads of a stream
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbarrier.cta.red.or.pred q, %1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(2 + s), "r"((uint32_t)p) : "memory");
    return r != 0;
}
__device__ __forceinline__ void stream_sync(int s) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(2 + s) : "memory"); }
__device__ __forceinline__ uint64_t bits2(uint32_t lo, uint32_t hi) { return pair(__uint_as_float(lo), __uint_as_float(hi)); }

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
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
    const uint32_t q_full = v_empty + 8 * kStages, q_empty = q_full + 16;               // [2] per Q buffer
    const uint32_t s_full = q_empty + 16, p_full = s_full + 16, o_full = p_full + 16;   // [2] per stream
    const uint32_t x_ready = o_full + 16, x_done = x_ready + 16, flushed = x_done + 16; // [2] the join of a piece's streams; an issuer's MMAs when it gives up
    Meta* const meta = reinterpret_cast<Meta*>(smem + L::kOffMeta);
    State& st = *reinterpret_cast<State*>(smem + L::kOffState);
    uint32_t& tmem_base_s = *reinterpret_cast<uint32_t*>(smem + L::kOffMisc);
    volatile int& abort_s = *reinterpret_cast<volatile int*>(smem + L::kOffMisc + 4);
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t limit = a.wait_budget ? a.wait_budget : kPollLimit;

    if (tid == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(k_full + 8 * i, 1 + 16), mbar_init(k_empty + 8 * i, 4);
            mbar_init(v_full + 8 * i, 1), mbar_init(v_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full + 8 * i, 4), mbar_init(q_empty + 8 * i, 2 + 8);
            mbar_init(s_full + 8 * i, 1), mbar_init(p_full + 8 * i, 4), mbar_init(o_full + 8 * i, 1);
            mbar_init(x_ready + 8 * i, 4), mbar_init(x_done + 8 * i, 4), mbar_init(flushed + 8 * i, 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        abort_s = 0;
        for (int i = 0; i < 4; ++i) st.fail[i >> 1][i & 1] = 0;
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
    const bool planned = is_plan(a.p, a.T, a.Hkv);
    if (!planned && blockIdx.x == 0 && tid == 0) report(a.status, STATUS_BAD_TOKEN, -1);
    Walk w(a.p, a.Hkv, planned);
    // the count-th completion; the same answer in every lane
    auto wait = [&](uint32_t bar, uint32_t count) {
        bool ok = bar_try(bar, count & 1);
        if (__all_sync(0xffffffffu, ok)) return true;
        ok = bar_wait_slow(bar, count & 1, &abort_s, limit);
        return (bool)__all_sync(0xffffffffu, ok);
    };
    // Behind this barrier every warp has left its loop and the abort flag is final.
    auto all_done = [] {
        __syncwarp();
        asm volatile("barrier.cta.sync 1, %0;" ::"n"(kThreads) : "memory");
    };
    auto columns = [](int rows) { return (rows + 7) & ~7; };                            // of one term

    if (warp < kWarpIssue) {
        // ================================ softmax and output ================================
        // Launched with 512 x 128 registers: 256 x 72 + 256 x 184 of them.
        asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
        const int s = warp >> 2, q = warp & 3, key = q * 32 + lane;
        const uint32_t lanes = (uint32_t)(q * 32) << 16;
        const uint32_t tmem_s = tmem + s * 128 + lanes, tmem_o = tmem + kTmemO + s * 128 + lanes;
        const uint32_t p_at = smem0 + s * L::kP + key * 16;
        float* const neg = st.neg[s];
        // parities: phases of S, of O of this stream and of the other, of joins by this stream and by the other, key tiles so
        // far; and whether the other stream is still reading this one's O
        enum : uint32_t { PH_S = 1, PH_O = 2, PH_O_OTHER = 4, PH_X = 8, PH_X_OTHER = 16, LENT = 32 };
        uint32_t ph = 0, n_t = 0, n_q = 0;
        // The four warps of a stream meet at barriers that have no bound, so they have to leave together: one whose wait has run
        // out goes on to the next barrier, without waiting any more, and tells the others there.  A flag for every other
        // barrier, since a warp may be one ahead.
        bool fail = false;
        uint32_t turn = 0;
        auto hold = [&](uint32_t bar, uint32_t count) {
            if (!fail) fail = !wait(bar, count);
        };
        auto hold_phase = [&](uint32_t bar, uint32_t phase) { hold(bar, (ph & phase) ? 1 : 0); };
        auto agreed = [&](bool p, bool& any) {         // whether all go on; any: p of any thread
            if (fail) st.fail[s][turn] = 1;
            any = any_of_stream(s, p);
            fail = st.fail[s][turn] != 0;
            turn ^= 1;
            return !fail;
        };
        bool any, out = false;
        while (w.next()) {
            const int n = w.k1 - w.k0, R = w.u.ntok * a.G;
            const bool leads = (int)(n_t & 1) == s, join = n > 1;
            if (n == 0) {                              // rows that see nothing; a piece of such a unit is the whole of it
                if (leads && w.slot < 0)
                    for (int r = q; r < R; r += 4) {
                        const int64_t orow = (int64_t)(w.u.row0 + r / a.G) * a.Hq + w.head * a.G + r % a.G;
                        for (int d = lane; d < D; d += 32) a.o[orow * D + d] = 0;
                        if (a.lse && lane == 0) a.lse[orow] = -INFINITY;
                    }
                continue;
            }
            const int slot = n_q & 1;
            hold(q_full + 8 * slot, n_q >> 1);
            ++n_q;
            const uint32_t c0 = n_t;
            n_t += n;
            if (!leads && !join) {
                ph ^= PH_O_OTHER;
                if (lane == 0) mbar_arrive(q_empty + 8 * slot);
                continue;
            }
            if (ph & LENT) {                           // P V overwrites O, and this stream's statistics are written anew
                hold_phase(x_done + 8 * (s ^ 1), PH_X_OTHER);
                ph ^= PH_X_OTHER | LENT;
            }
            const Meta& mt = meta[slot];
            const int RP = columns(R), n_ch = RP / 8;
            const int lo_max = mt.lo_max, hi_min = mt.hi_min;
            const int t_hi = (w.u.key_hi + kTileKeys - 1) / kTileKeys;
            uint64_t l2[kMaxRows / 2];
#pragma unroll
            for (int i = 0; i < kMaxRows / 2; ++i) l2[i] = 0;
            int ref_v = kNoScale;
            if (key < kMaxRows) neg[key] = INFINITY;   // no reference yet: a visible key's score is above every bound
            if (!agreed(false, any)) break;
            int mine = 0;
            for (int i = leads ? 0 : 1; i < n; i += 2, ++mine) {
                const uint32_t stage = (c0 + i) % kStages, use = (c0 + i) / kStages;
                hold(k_full + 8 * stage, use);         // the scales
                const unsigned char* const sb = smem + L::kOffScales + stage * (kBlocks * 32) + (key >> 4) * 32 + (key & 15);
                const uint32_t kb = sb[0], vb = sb[16];
                const int key0 = (t_hi - 1 - (w.k0 + i)) * kTileKeys, at = key0 + key;
                const bool masked = key0 < lo_max || key0 + kTileKeys > hi_min;
                bool seen = !masked;
                // the key's power of two, times 2^7 against the rows' 2^-7
                const float kk = __uint_as_float(kb > 247 || vb > 247 ? 0x7fc00000u : (kb + 7) << 23);
                const uint64_t kk2 = pair(kk, kk);
                hold_phase(s_full + 8 * s, PH_S);
                ph ^= PH_S;
                tc_fence_after();
                __syncwarp();
                if (lane == 0) mbar_arrive(k_empty + 8 * stage);                        // S is complete and the scales are read
                float x[kMaxRows];
                uint32_t y[2][24];
                auto load = [&](int ch) {
#pragma unroll
                    for (int t = 0; t < 3; ++t) tmem_ld8(tmem_s + t * RP + ch * 8, y[ch & 1] + 8 * t);
                };
                // scores of the eight rows of a chunk less `less`, -inf for a key that a row does not see
                auto scores = [&](int ch, const float* less) {
                    const uint32_t* const v = y[ch & 1];
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const int r = ch * 8 + j;
                        const uint64_t sum = add2(add2(bits2(v[j], v[j + 1]), bits2(v[8 + j], v[9 + j])), bits2(v[16 + j], v[17 + j]));
                        const float2 c = *reinterpret_cast<const float2*>(mt.c + r);
                        uint64_t z = mul2(mul2(sum, pair(c.x, c.y)), kk2);
                        if (less) {
                            const float2 m = *reinterpret_cast<const float2*>(less + r);
                            z = add2(z, pair(m.x, m.y));
                        }
                        const float2 f = unpair(z);
                        x[r] = f.x, x[r + 1] = f.y;
                    }
                    if (masked) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int r = ch * 8 + j;
                            const bool sees = at >= mt.lo[r] && at < mt.hi[r];
                            if (!sees) x[r] = -INFINITY;
                            seen = seen || (sees && r < R);
                        }
                    }
                };
                auto all_scores = [&](const float* less) {
                    load(0);
#pragma unroll
                    for (int ch = 0; ch < kChunks; ++ch) {
                        if (ch >= n_ch) break;
                        tmem_wait_ld24(y[ch & 1]);
                        if (ch + 1 < kChunks && ch + 1 < n_ch) load(ch + 1);
                        scores(ch, less);
                    }
                };
                all_scores(neg);
                float top = -INFINITY;
#pragma unroll
                for (int ch = 0; ch < kChunks; ++ch) {
                    if (ch >= n_ch) break;
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = fmaxf(top, x[ch * 8 + j]);
                }
                int ev = seen ? (int)vb - 127 : kNoScale;
                int dev = seen ? ev - ref_v : 0;
                if (!agreed(top + (float)max(dev, -40) > kMost, any)) {
                    out = true;
                    break;
                }
                // Rare but for a piece's first tile: a weight would leave the range of 16 bits, or a row sees its first key.
                if (any) {
                    all_scores(nullptr);
#pragma unroll
                    for (int ch = 0; ch < kChunks; ++ch) {
                        if (ch >= n_ch) break;
                        int best = 0;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int m = __reduce_max_sync(0xffffffffu, ordered(x[ch * 8 + j]));
                            if (lane == j) best = m;
                        }
                        if (lane < 8) st.top[s][q][ch * 8 + lane] = unordered(best);
                    }
                    const int e = __reduce_max_sync(0xffffffffu, ev);
                    if (lane == 0) st.exp_top[s][q] = e;
                    stream_sync(s);
                    if (key < RP) {
                        const float m = fmaxf(fmaxf(st.top[s][0][key], st.top[s][1][key]), fmaxf(st.top[s][2][key], st.top[s][3][key]));
                        const float old = -neg[key], now = fmaxf(old, m - kTop);
                        neg[key] = -now;
                        st.fac[s][key] = old == -INFINITY ? 0.f : ex2_approx(old - now);
                    }
                    const int ref = max(max(max(st.exp_top[s][0], st.exp_top[s][1]), max(st.exp_top[s][2], st.exp_top[s][3])), ref_v);
                    stream_sync(s);
                    const float shrink = ex2_approx((float)(ref_v - ref));
                    ref_v = ref;
                    dev = seen ? ev - ref_v : 0;
#pragma unroll
                    for (int ch = 0; ch < kChunks; ++ch) {
                        if (ch >= n_ch) break;
                        float f[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int r = ch * 8 + j;
                            f[j] = st.fac[s][r];
                            x[r] = x[r] == -INFINITY ? -INFINITY : x[r] + neg[r];
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) l2[ch * 4 + j] = mul2(l2[ch * 4 + j], pair(f[2 * j], f[2 * j + 1]));
                        if (mine > 0) {                // O holds this piece's earlier tiles, complete since S of this one is
#pragma unroll 1
                            for (int t = 0; t < 3; ++t) {
                                uint32_t o[8];
                                tmem_ld8(tmem_o + t * RP + ch * 8, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int j = 0; j < 8; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * (f[j] * shrink));
                                tmem_st8(tmem_o + t * RP + ch * 8, o);
                            }
                        }
                    }
                    tmem_wait_st();
                }
                // weights: their sums in 32 bits; times V's power of two, and split, for the product
                const float vs = __uint_as_float((uint32_t)(min(max(dev, -126), 127) + 127) << 23);
                const uint64_t vs2 = pair(vs, vs);
#pragma unroll
                for (int ch = 0; ch < kChunks; ++ch) {
                    if (ch >= n_ch) break;
                    uint32_t h[4], t0[3], t1[3];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint64_t p = pair(ex2_approx(x[ch * 8 + 2 * j]), ex2_approx(x[ch * 8 + 2 * j + 1]));
                        l2[ch * 4 + j] = add2(l2[ch * 4 + j], p);
                        const float2 wv = unpair(mul2(p, vs2));
                        h[j] = pack_half(wv.x, wv.y);
                    }
                    split4(h[0], h[1], t0);
                    split4(h[2], h[3], t1);
#pragma unroll
                    for (int t = 0; t < 3; ++t) {
                        const int col = t * RP + ch * 8;
                        asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(p_at + (col >> 4) * (kTileKeys * 16) + (col & 8)), "r"(t0[t]), "r"(t1[t]) : "memory");
                    }
                }
                // Hidden rows of V have to be finite, since 0 x NaN is NaN.
                if (masked) {
                    hold(v_full + 8 * stage, use);
                    if (!seen) {
                        const uint32_t row = smem0 + L::kOffV + stage * L::kTile + key * D;
#pragma unroll
                        for (int ch = 0; ch < D / 16; ++ch)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(row + ((ch + lane) % (D / 16)) * 16), "r"(0) : "memory");
                    }
                }
                fence_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * s);
            }
            if (out) break;
            // ---- the piece's rows: sums over the lanes (each chunk's eight rows end up on lanes 0, 4, .. 28), then over the warps
#pragma unroll
            for (int ch = 0; ch < kChunks; ++ch) {
                if (ch >= n_ch) break;
                float v[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 f = unpair(l2[ch * 4 + j]);
                    v[2 * j] = f.x, v[2 * j + 1] = f.y;
                }
#pragma unroll
                for (int half = 4; half > 0; half >>= 1) {
                    const int bit = half * 4;
                    const bool up = lane & bit;
#pragma unroll
                    for (int j = 0; j < half; ++j) {
                        const float send = up ? v[j] : v[j + half], keep = up ? v[j + half] : v[j];
                        v[j] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
                    }
                }
                v[0] += __shfl_xor_sync(0xffffffffu, v[0], 2);
                v[0] += __shfl_xor_sync(0xffffffffu, v[0], 1);
                if ((lane & 3) == 0) st.top[s][q][ch * 8 + (lane >> 2)] = v[0];
            }
            if (!agreed(false, any)) break;
            float m_run = 0.f, l_run = 0.f;
            if (key < RP) {
                m_run = -neg[key];
                l_run = (st.top[s][0][key] + st.top[s][1][key]) + (st.top[s][2][key] + st.top[s][3][key]);
            }
            if (!leads) {
                if (key < RP) st.ml[s][key] = make_float2(m_run, l_run);
                if (key == 0) st.exp_ref[s] = ref_v;
                __syncwarp();
                if (lane == 0) mbar_arrive(x_ready + 8 * (s ^ 1)), mbar_arrive(q_empty + 8 * slot);
                ph = (ph | LENT) ^ (PH_O | PH_O_OTHER);
                continue;
            }
            hold_phase(o_full + 8 * s, PH_O);
            ph ^= PH_O;
            int ref_other = kNoScale;
            if (join) {
                hold_phase(x_ready + 8 * s, PH_X);
                hold_phase(o_full + 8 * (s ^ 1), PH_O_OTHER);
                ph ^= PH_X | PH_O_OTHER;
                ref_other = st.exp_ref[s ^ 1];
            }
            const bool part = w.slot >= 0;
            const int64_t part0 = (int64_t)w.slot * kMaxRows;
            if (key < RP) {
                const float2 other = join ? st.ml[s ^ 1][key] : make_float2(0.f, 0.f);
                // a stream without a sum has seen nothing of the row: its reference may be anything
                const bool h0 = l_run != 0.f, h1 = other.y != 0.f;
                const float top = fmaxf(h0 ? m_run : -INFINITY, h1 ? other.x : -INFINITY);
                float f0 = h0 ? ex2_approx(m_run - top) : 0.f, f1 = h1 ? ex2_approx(other.x - top) : 0.f;
                const float l = l_run * f0 + other.y * f1;
                if (!part) {
                    const float inv = l == 0.f ? 0.f : 1.f / l;
                    f0 *= inv, f1 *= inv;
                }
                st.join[s][key] = make_float2(f0, f1);
                if (key < R) {
                    // A row whose sum is no number joins with a reference of infinity: all factors are then 0 or not a number.
                    if (part) *reinterpret_cast<float2*>(a.p.part_ml + (part0 + key) * 2) = make_float2(l != l ? INFINITY : top, l);
                    else if (a.lse) a.lse[(int64_t)(w.u.row0 + key / a.G) * a.Hq + w.head * a.G + key % a.G] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
                }
            }
            if (!agreed(false, any)) break;
            // O is [dim][term, row]: a thread has one dim (64 dims sit on 16 lanes of each quarter)
            const bool live = D == 128 || lane < 16;
            const int d = D == 128 ? key : q * 16 + lane;
            const uint32_t tmem_other = tmem + kTmemO + (s ^ 1) * 128 + lanes;
            const float v0 = ref_v == kNoScale ? 0.f : __uint_as_float((uint32_t)(ref_v + 127) << 23);
            const float v1 = ref_other == kNoScale ? 0.f : __uint_as_float((uint32_t)(ref_other + 127) << 23);
            tc_fence_after();
            int64_t orow = (int64_t)w.u.row0 * a.Hq + w.head * a.G;
            int g = 0;
#pragma unroll 1
            for (int ch = 0; ch < n_ch; ++ch) {
                uint32_t y[24], z[24];
#pragma unroll
                for (int t = 0; t < 3; ++t) tmem_ld8(tmem_o + t * RP + ch * 8, y + 8 * t);
                if (join) {
#pragma unroll
                    for (int t = 0; t < 3; ++t) tmem_ld8(tmem_other + t * RP + ch * 8, z + 8 * t);
                }
                tmem_wait_ld24(y);
                if (join) tmem_wait_ld24(z);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = ch * 8 + j;
                    if (r >= R) break;
                    const float2 f = st.join[s][r];
                    float v = f.x != 0.f ? ((__uint_as_float(y[j]) + __uint_as_float(y[8 + j])) + __uint_as_float(y[16 + j])) * f.x * v0 : 0.f;
                    if (join && f.y != 0.f) v += ((__uint_as_float(z[j]) + __uint_as_float(z[8 + j])) + __uint_as_float(z[16 + j])) * f.y * v1;
                    if (live) {
                        if (part) {
                            a.p.part_acc[(part0 + r) * D + d] = v;
                        } else {
                            const __nv_bfloat16 b = __float2bfloat16_rn(v);
                            a.o[(orow + g) * D + d] = *reinterpret_cast<const uint16_t*>(&b);
                        }
                    }
                    if (++g == a.G) g = 0, orow += a.Hq;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (join) mbar_arrive(x_done + 8 * s);
                mbar_arrive(q_empty + 8 * slot);
            }
        }
        all_done();
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp < kWarpK) {
        // ================================ MMA issuers ================================
        const int s = warp - kWarpIssue;
        const uint32_t tmem_s = tmem + s * 128, tmem_o = tmem + kTmemO + s * 128;
        const uint64_t dp = smem_desc(smem0 + s * L::kP, 128, kTileKeys * 16, 0);
        uint32_t n_t = 0, n_p = 0, n_q = 0;
        bool ok = true;
        while (ok && w.next()) {
            const int n = __shfl_sync(0xffffffffu, w.k1 - w.k0, 0);
            if (n == 0) continue;
            const int N = __shfl_sync(0xffffffffu, (3 * columns(w.u.ntok * a.G) + 15) & ~15, 0);
            const int slot = n_q & 1;
            if (!(ok = wait(q_full + 8 * slot, n_q >> 1))) break;
            ++n_q;
            const int i0 = (int)((n_t ^ s) & 1);
            if (i0 >= n && lane == 0) mbar_arrive(q_empty + 8 * slot);                  // a single key tile, the other stream's
            const uint32_t idesc_s = instr_desc_f8(kTileKeys, N, 0, 0), idesc_o = instr_desc_f8(D, N, 1, 1);
            const uint64_t dq = smem_desc(smem0 + L::kOffQ + slot * L::kQ, 16, 8 * D, L::kSwizzle);
            for (int i = i0; i < n; i += 2, ++n_p) {
                const uint32_t c = n_t + i, stage = c % kStages, use = c / kStages;
                const bool last = i + 2 >= n;
                if (!(ok = wait(k_full + 8 * stage, use))) break;
                tc_fence_after();
                const uint64_t dk = smem_desc(smem0 + L::kOffK + stage * L::kTile, 16, 8 * D, L::kSwizzle);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 32; ++k) umma_ss_f8(tmem_s, dk + 2 * k, dq + 2 * k, idesc_s, k > 0);     // 32 dims each
                    umma_commit(s_full + 8 * s);
                    if (last) umma_commit(q_empty + 8 * slot);
                }
                if (!(ok = wait(v_full + 8 * stage, use))) break;
                if (!(ok = wait(p_full + 8 * s, n_p))) break;
                tc_fence_after();
                const uint64_t dv = smem_desc(smem0 + L::kOffV + stage * L::kTile, 16, 8 * D, L::kSwizzle);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kTileKeys / 32; ++k)                            // 32 keys each
                        umma_ss_f8(tmem_o, dv + ((k * 32 * D) >> 4), dp + ((k * 32 * 16) >> 4), idesc_o, (i > i0 || k > 0) ? 1u : 0u);
                    umma_commit(v_empty + 8 * stage);
                    if (last) umma_commit(o_full + 8 * s);
                }
            }
            n_t += n;
        }
        all_done();
        if (abort_s) {
            // the CTA is giving up: what is still in flight reads shared memory and writes tensor memory
            if (elect_one()) umma_commit(flushed + 8 * s);
            const long long t0 = clock64();
            while (!bar_try(flushed + 8 * s, 0) && clock64() - t0 < kWaitCycles) {}
        }
    } else if (warp < kWarpQ) {
        // ================================ K and V producers ================================
        const bool is_v = warp == kWarpV;
        const uint32_t full = is_v ? v_full : k_full, empty = is_v ? v_empty : k_empty;
        const uint32_t ring = smem0 + (is_v ? L::kOffV : L::kOffK);
        const int32_t oob = a.num_blocks * 2 * a.Hkv;                                   // past the slab: zero fill
        uint32_t n_t = 0;
        bool ok = true;
        while (ok && w.next()) {
            const int n = w.k1 - w.k0;
            if (n == 0) continue;
            const int32_t* table = a.kv_indices + w.u.tbl;
            const int b_lo = w.u.key_lo / kBs, b_hi = (w.u.key_hi + kBs - 1) / kBs;     // blocks that hold a visible key
            const int t0 = (w.u.key_hi + kTileKeys - 1) / kTileKeys - 1 - w.k0;         // first key tile
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
                if (i + 1 < n) id_next = block_id(t0 - i - 1);
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
        // ================================ Q ================================
        // Every row times a power of two that brings its largest element to [2^14, 2^15), split into three e5m2 terms: rows
        // [term][row] of the product's second operand.  bf16 has eight significant bits, the terms nine: nothing is lost but
        // what lies below 2^-16 then.
        const int wq = warp - kWarpQ;
        constexpr int kPer = D / 32;                   // elements of a lane
        uint32_t n_q = 0;
        bool ok = true;
        while (ok && w.next()) {
            if (w.k1 == w.k0) continue;
            const int slot = n_q & 1, R = w.u.ntok * a.G, RP = columns(R);
            const uint32_t qb = smem0 + L::kOffQ + slot * L::kQ;
            Meta& mt = meta[slot];
            // a warp has rows wq, wq + 4, ..; the first half of them is read before the buffer is free
            constexpr int kRowsAhead = kMaxRows / 8;
            uint32_t v[kRowsAhead][kPer / 2];
            auto fetch = [&](int first) {
#pragma unroll
                for (int i = 0; i < kRowsAhead; ++i) {
                    const int r = first + 4 * i;
                    if (r < R) {
                        const uint16_t* const src = a.q + (int64_t)(w.u.row0 + r / a.G) * a.q_stride + (w.head * a.G + r % a.G) * D + lane * kPer;
                        if constexpr (D == 128) {
                            const uint2 z = __ldg(reinterpret_cast<const uint2*>(src));
                            v[i][0] = z.x, v[i][kPer / 2 - 1] = z.y;
                        } else {
                            v[i][0] = __ldg(reinterpret_cast<const uint32_t*>(src));
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < kPer / 2; ++j) v[i][j] = 0;
                    }
                }
            };
            auto put = [&](int first) {
#pragma unroll
                for (int i = 0; i < kRowsAhead; ++i) {
                    const int r = first + 4 * i;
                    if (r >= RP) break;
                    uint32_t big = 0;
#pragma unroll
                    for (int j = 0; j < kPer / 2; ++j) big = max(big, max(v[i][j] & 0x7fffu, (v[i][j] >> 16) & 0x7fffu));
                    big = __reduce_max_sync(0xffffffffu, big);
                    const int k = 141 - max((int)(big >> 7), 1);
                    const float f0 = __uint_as_float((uint32_t)((k >> 1) + 127) << 23), f1 = __uint_as_float((uint32_t)(k - (k >> 1) + 127) << 23);
                    uint32_t h[2], t[3];
#pragma unroll
                    for (int j = 0; j < kPer / 2; ++j)
                        h[j] = pack_half(__uint_as_float(v[i][j] << 16) * f0 * f1, __uint_as_float(v[i][j] & 0xffff0000u) * f0 * f1);
                    if constexpr (D == 64) h[1] = 0;
                    split4(h[0], h[1], t);
#pragma unroll
                    for (int j = 0; j < 3; ++j) {
                        const int row = j * RP + r;    // the swizzle exchanges 16-byte pieces by the row
                        if constexpr (D == 128)
                            asm volatile("st.shared.b32 [%0], %1;" ::"r"(qb + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4), "r"(t[j]) : "memory");
                        else
                            asm volatile("st.shared.b16 [%0], %1;" ::"r"(qb + row * 64 + (((lane >> 3) ^ ((row >> 1) & 3)) << 4) + (lane & 7) * 2), "h"((uint16_t)t[j]) : "memory");
                    }
                    if (lane == 0) mt.c[r] = r >= R ? 0.f : (big >= 0x7f80u ? __uint_as_float(0x7fc00000u) : ldexpf(a.sc, -k - 7));
                }
            };
            fetch(wq);
            if (n_q >= 2 && !(ok = wait(q_empty + 8 * slot, (n_q >> 1) - 1))) break;
            put(wq);
            if (wq + 4 * kRowsAhead < RP) {
                fetch(wq + 4 * kRowsAhead);
                put(wq + 4 * kRowsAhead);
            }
            if (wq == 0) {
                const bool causal = a.p.header->causal;
                int lo_max = 0, hi_min = 0x7fffffff;
                for (int r = lane; r < RP; r += 32) {
                    int lo = 0, hi = 0x7fffffff;       // rows of padding never mask
                    if (r < R) {
                        const int t = r / a.G;
                        if (causal) hi = w.u.pos0 + t + 1;
                        else lo = a.p.row_lo[w.u.row0 + t], hi = a.p.row_hi[w.u.row0 + t];
                    }
                    mt.lo[r] = lo, mt.hi[r] = hi;
                    lo_max = max(lo_max, lo), hi_min = min(hi_min, hi);
                }
                lo_max = __reduce_max_sync(0xffffffffu, lo_max), hi_min = __reduce_min_sync(0xffffffffu, hi_min);
                if (lane == 0) mt.lo_max = lo_max, mt.hi_min = hi_min;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full + 8 * slot);
            ++n_q;
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
