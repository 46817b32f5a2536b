// The 8-bit cache's number format.  A block is one page of one KV head, K and V apart; its rows are e4m3 values v that stand
// for v * 2^e, with one whole exponent e per block.  A power of two, so that
//   * a block whose exponent has to grow (a larger row is appended) is re-encoded by shifting: exact but for what drops below
//     e4m3's smallest step, where any scale would have put it too;
//   * the attention pass puts K's exponent into the fp32 scores, exactly, and turns V into fp16 without a rounding: e4m3's four
//     significant bits times 2^e, -24 <= e <= 7, is an fp16 number but for what lies below fp16's smallest step, 2^-24.
// e is the smallest exponent in [kExpMin, kExpMax] with (largest magnitude) <= 448 * 2^e; what exceeds 448 * 2^7 = 57344
// (fp16's own range ends at 65504) saturates there.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

#include "owl_common.cuh"

namespace owl {

constexpr int kExpMin = -24, kExpMax = 7;

// The exponent that a largest magnitude needs, given as the bits of a non-negative fp32 (infinity: the largest exponent).
// 448 = 1.75 * 2^8: adding 2^23 - 1.75's mantissa - 1 carries into the exponent exactly when the mantissa is above 1.75.
__host__ __device__ __forceinline__ int block_exponent(uint32_t magnitude_bits) {
    const int e = (int)((magnitude_bits + 0x1fffffu) >> 23) - 135;
    return e < kExpMin ? kExpMin : e > kExpMax ? kExpMax : e;
}
// An exponent as the cache holds it; one outside the format's range reads as the nearer end.
__device__ __forceinline__ int read_exponent(const int8_t* p) { return max(kExpMin, min(kExpMax, (int)*p)); }
__device__ __forceinline__ float exp2_int(int e) { return __int_as_float((e + 127) << 23); }      // -126 <= e <= 127

// Two fp32 to two e4m3 (x in the low byte), nearest even, saturating; a NaN stays one (0x7f).
__device__ __forceinline__ uint32_t pack_e4m3x2(float x, float y) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(y), "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
    return pack_e4m3x2(a, b) | pack_e4m3x2(c, d) << 16;
}
// Two e4m3 (the low 16 bits) to two fp16; exact.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t v) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)v));
    return r;
}
// Four e4m3 to four fp32; exact.
__device__ __forceinline__ float4 e4m3x4_to_f32(uint32_t v) {
    const uint32_t lo = e4m3x2_to_f16x2(v & 0xffffu), hi = e4m3x2_to_f16x2(v >> 16);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    return make_float4(a.x, a.y, b.x, b.y);
}
// Four e4m3 times a power of two, as e4m3.
__device__ __forceinline__ uint32_t rescale_e4m3x4(uint32_t v, float factor) {
    const float4 x = e4m3x4_to_f32(v);
    return pack_e4m3x4(x.x * factor, x.y * factor, x.z * factor, x.w * factor);
}

}  // namespace owl
