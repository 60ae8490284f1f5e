// Attention over the 8-bit cache.
#include "chunk_walk.h"
#include "kv8_codec.h"
#include "nsd_internal.h"

namespace nsd {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Attn8Args {
    ChunkPlan p;
    const uint8_t *codes, *scales;
    const uint16_t* q;
    int64_t q_stride;
    uint16_t* o;
    float* lse;
    const int32_t* kv_indices;
    float sc;                                          // scale, in the log2 domain
    int32_t *status, Hq, Hkv, G, T, num_blocks;
};

__device__ __forceinline__ void report(int32_t* status, int32_t bit, int r) {
    atomicOr(status, bit);
    atomicCAS(status + 1, 0, r + 1);
}

// A warp per (row, q head), one key after another: what the definition says, for every case.
template <int D>
__global__ void __launch_bounds__(256)
kv8_attn_plain_kernel(const __grid_constant__ Attn8Args a) {
    constexpr int kV = D / 32;
    if (!is_plan(a.p, a.T, a.Hkv)) {
        if (blockIdx.x == 0 && threadIdx.x == 0) report(a.status, STATUS_BAD_TOKEN, -1);
        return;
    }
    const int lane = threadIdx.x & 31;
    const ChunkHeader hd = *a.p.header;
    const int64_t per = a.T * (int64_t)a.Hq, all = hd.n_units * per;
    for (int64_t w = (blockIdx.x * 256ll + threadIdx.x) >> 5; w < all; w += gridDim.x * 8ll) {
        const ChunkUnit u = a.p.units[w / per];
        const int t = (int)(w % per) / a.Hq, h = (int)(w % per) % a.Hq, head = h / a.G;
        if (t >= u.ntok) continue;
        const int64_t row = u.row0 + t;
        const int lo = a.p.row_lo[row], hi = a.p.row_hi[row];
        float q[kV], o[kV] = {}, m = -INFINITY, l = 0.f;
        for (int i = 0; i < kV; ++i) q[i] = __uint_as_float((uint32_t)a.q[row * a.q_stride + h * D + lane * kV + i] << 16);
        for (int j = lo; j < hi; ++j) {
            const int b = j / 16;
            int32_t id = b < u.nblk ? a.kv_indices[u.tbl + b] : -1;
            const bool bad = (uint32_t)id >= (uint32_t)a.num_blocks;
            if (bad) {
                if (lane == 0) report(a.status, STATUS_BAD_BLOCK, u.req);
                id = 0;
            }
            const int64_t tile = (int64_t)id * 2 * a.Hkv + head, sc = (((int64_t)id * a.Hkv + head) * 2) * 16 + j % 16;
            const float ks = bad ? 0.f : kv8_scale(a.scales[sc]), vs = bad ? 0.f : kv8_scale(a.scales[sc + 16]);
            const uint8_t* k8 = a.codes + (tile * 16 + j % 16) * D + lane * kV;
            const uint8_t* v8 = k8 + (int64_t)a.Hkv * 16 * D;
            float s = 0.f, v[kV];
            for (int i = 0; i < kV; ++i) s += q[i] * (bad ? 0.f : kv8_values2(k8[i]).x), v[i] = bad ? 0.f : kv8_values2(v8[i]).x * vs;
            for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            s = vs != vs ? vs : s * ks * a.sc;
            const float top = fmaxf(m, s), f = m == -INFINITY ? 0.f : exp2f(m - top), e = s != s ? s : exp2f(s - top);
            for (int i = 0; i < kV; ++i) o[i] = o[i] * f + e * v[i];
            l = l * f + e;
            m = top;
        }
        const int64_t orow = row * a.Hq + h;
        for (int i = 0; i < kV; ++i) {
            const __nv_bfloat16 b = __float2bfloat16_rn(l == 0.f ? 0.f : o[i] / l);
            a.o[orow * D + lane * kV + i] = *reinterpret_cast<const uint16_t*>(&b);
        }
        if (a.lse && lane == 0) a.lse[orow] = l == 0.f ? -INFINITY : (l != l ? l : (m + log2f(l)) * kLn2);
    }
}

}  // namespace

cudaError_t kv8_attn_init() { return cudaSuccess; }

cudaError_t launch_kv8_attn(const ChunkPlan& p, const Kv8AttnLaunch& l, cudaStream_t stream, int* launched) {
    Attn8Args a{};
    a.p = p;
    a.codes = l.codes, a.scales = l.scales, a.q = l.q, a.q_stride = l.q_stride, a.o = l.o, a.lse = l.lse, a.kv_indices = l.kv_indices;
    a.sc = l.scale * kLog2e;
    a.status = l.status;
    a.Hq = l.shape.Hq, a.Hkv = l.shape.Hkv, a.G = a.Hq / a.Hkv, a.T = p.kind.tokens(a.G), a.num_blocks = l.shape.num_blocks;
    if (l.shape.D == 128) kv8_attn_plain_kernel<128><<<p.n_ctas * 8, 256, 0, stream>>>(a);
    else kv8_attn_plain_kernel<64><<<p.n_ctas * 8, 256, 0, stream>>>(a);
    *launched = 1;
    return cudaGetLastError();
}

}  // namespace nsd
