// Codes of a K/V cache in 8 bits: e4m3 (1 sign, 4 exponent, 3 fraction bits; largest value 448; no infinities, one NaN per sign).
#pragma once
#include <cuda_fp16.h>
#include <stdint.h>

namespace mtv {

// Two values to codes, round to nearest even; beyond the largest code (infinities too) the largest code; NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// Every code is a number of fp16.  Codes in the lower or upper half of a word.
__device__ __forceinline__ uint32_t f16x2_lo(uint32_t codes) {
    uint32_t r;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, l;\n}" : "=r"(r) : "r"(codes));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_hi(uint32_t codes) {
    uint32_t r;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.rn.f16x2.e4m3x2 %0, h;\n}" : "=r"(r) : "r"(codes));
    return r;
}
// A pair of fp32 values as fp16, round to nearest even.
__device__ __forceinline__ uint32_t pack2_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// The top bit of every byte of the result: the code there is NaN.
__device__ __forceinline__ uint32_t nan_codes(uint32_t codes) { return ((codes & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// Codes that are NaN become 0.
__device__ __forceinline__ uint32_t without_nans(uint32_t codes) { return codes & ~((nan_codes(codes) >> 7) * 0xffu); }
__device__ __forceinline__ float2 f16x2_values(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

}  // namespace mtv
