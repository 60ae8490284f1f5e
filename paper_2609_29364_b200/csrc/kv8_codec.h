// The 8-bit form of a row of K or V (one token and kv head): e4m3 codes and one power of two 2^e, kept as the byte e + 127.
// Included inside a .cu file; everything is a device function.
//
// A power of two costs an e4m3 code nothing -- its relative error is 2^-4 wherever it lies among the normal numbers, 2^-6 to
// 448 -- and makes both directions exact but for the one rounding to e4m3: x 2^-e and code 2^e lose no bit, so that packing,
// unpacking and the products of the attention agree to the bit on what a cache holds.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace nsd {

__device__ __forceinline__ float kv8_magnitude(float x) {       // what counts towards a row's maximum: finite values
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.f;
}
// The least e >= -126 with top <= 448 2^e, plus 127.  448 = 1.75 2^8: adding 0x1fffff to the bits carries into the exponent
// exactly where the mantissa is above 1.75.
__device__ __forceinline__ uint32_t kv8_scale_byte(float top) {
    const uint32_t b = (__float_as_uint(top) + 0x1fffffu) >> 23;
    return b > 9 ? b - 8 : 1;
}
__device__ __forceinline__ float kv8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }   // 2^-e, byte in 1..247
// 2^e as the 8-bit exponent format has it: 0 is 2^-127, 255 not a number (neither is ever written here)
__device__ __forceinline__ float kv8_scale(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : (byte == 255 ? 0x7fc00000u : byte << 23));
}
// Two codes, round to nearest even; the lower byte is lo.  Infinities become the largest code: only for rows that have none.
__device__ __forceinline__ uint32_t kv8_codes2_finite(float lo, float hi, float inverse) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi * inverse), "f"(lo * inverse));
    return r;
}
// For any row: infinities become NaN.
__device__ __forceinline__ uint32_t kv8_codes2(float lo, float hi, float inverse) {
    return kv8_codes2_finite(fmaf(lo, 0.f, lo), fmaf(hi, 0.f, hi), inverse);
}
__device__ __forceinline__ float2 kv8_values2(uint32_t codes) {          // of the lower two bytes
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

}  // namespace nsd
