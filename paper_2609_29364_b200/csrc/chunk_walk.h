// What the attention kernels that work under a plan share: its check, a CTA's walk over its share of the work, and the
// bounded waits of a whole warp.  Included inside a .cu file; everything is a device function.
#pragma once
#include "nsd_internal.h"
#include "tcgen05_ops.h"

namespace nsd {

// A buffer that the plan call of this kind has filled for these rows, this shape and this layout (max_units follows from
// max_batch, and with max_rows and n_ctas places every part up to the partial results).
__device__ __forceinline__ bool is_plan(const ChunkPlan& p, int T, int Hkv) {
    const ChunkHeader h = *p.header;
    return h.magic == p.kind.magic && h.max_rows == p.max_rows && h.max_units == p.max_units && h.n_ctas == p.n_ctas && h.T == T && h.Hkv == Hkv;
}

// A CTA's walk over its share of the line.
struct Walk {
    const ChunkUnit* units;
    ChunkStart at, end;
    int Hkv;
    // the piece under way
    ChunkUnit u;
    int head, k0, k1, slot;                            // key tiles [k0, k1) in walking order; partial slot or -1
    bool planned;                                      // else there is no work
    // The share is read beside the header, not behind it: a trip to the L2 less before the first tile.
    __device__ __forceinline__ Walk(const ChunkPlan& p, int T, int Hkv_)
        : units(p.units), at(p.starts[blockIdx.x]), end(p.starts[blockIdx.x + 1]), Hkv(Hkv_), planned(is_plan(p, T, Hkv_)) {
        if (!planned) end = at;
    }
    __device__ __forceinline__ bool next() {
        if (at.unit == end.unit && at.head == end.head && at.tile == end.tile) return false;
        step(units[at.unit]);
        return true;
    }
    __device__ __forceinline__ void step(const ChunkUnit& here) {                       // here: unit at.unit
        u = here;
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
}  // namespace nsd
