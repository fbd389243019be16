// The e4m3 key / value cache: layout, scales, conversions.
//
//   cache  [n_blocks, Hkv, bt, d] bytes   codes; a block holds bt consecutive tokens of one sequence
//   scale  [n_blocks, Hkv] fp32           value = code * scale, one scale per block and head
//
// The library only writes scales that are powers of two, 2^e with e >= -64.  A code then converts to
// another scale without a second rounding as long as it stays a normal e4m3 number, so a block whose
// scale has to grow when a larger token joins it does not wear down the tokens that were there before.
#pragma once

#include <cuda_fp8.h>
#include "bs_common.cuh"

namespace bs {

// Smallest block scale 2^-64.  The attention puts the scale of V into the exponent of a probability, where fp32 has room for
// 2^96 between the scales of a sequence beside 2^30 between its probabilities: with this floor up to 2^32.
constexpr int kCacheMinExp = -64;

// The smallest power of two s >= 2^-64 with amax / s <= 448 (amax finite, >= 0).
__device__ __forceinline__ float pow2_scale(float amax) {
    const uint32_t u = __float_as_uint(amax);
    // amax = 1.f x 2^k, 448 = 1.75 x 2^8: the exponent is k - 8, one more if the significand is above 1.75
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < kCacheMinExp ? kCacheMinExp : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Two floats to two e4m3 codes (round to nearest even, too large to +-448, NaN to NaN); `lo` in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    return e4m3x2(a, b) | (e4m3x2(c, d) << 16);
}
// Two codes (low 16 bits) to two halves: exact.
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t v) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)v));
    return r;
}
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t v) {
    const uint32_t h = e4m3x2_to_half2(v);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// Four codes brought to another scale: code * f, rounded once.
__device__ __forceinline__ uint32_t rescale_codes(uint32_t v, float f) {
    const float2 a = e4m3x2_to_float2(v & 0xffffu), b = e4m3x2_to_float2(v >> 16);
    return e4m3x4(a.x * f, a.y * f, b.x * f, b.y * f);
}

inline bool cache_geometry_ok(int Hkv, int d, int n_blocks, int bt) {
    return Hkv >= 1 && n_blocks >= 1 && (d == 64 || d == 128) && (bt == 16 || bt == 32 || bt == 64 || bt == 128) &&
           (long long)n_blocks * bt <= 0x7fffffffLL && (long long)n_blocks * Hkv <= 0x7fffffffLL;
}

}  // namespace bs
