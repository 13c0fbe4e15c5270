// Rows in 8 bits: e4m3 numbers (four exponent bits, three of the fraction, no infinities) and one power of two a row.
//
//   2^e: the smallest, e from kLeastExp to kMostExp, with max |x| <= 448 * 2^e over the row's finite features
//   code = x / 2^e to nearest even, at most 448; NaN where x is not finite          x' = code * 2^e
//
// A power of two costs a floating format no precision, and its products are exact: what a code stands for is a bf16 and an fp32 number
// as it is (codes have 4 bits, their smallest step is 2^-9, so kLeastExp keeps every value a normal number and kMostExp a finite one).
// The scale byte is e + 127, the exponent of the fp32 number 2^e.
#pragma once

#include "attend_dev.h"

namespace mukv {

constexpr int kLeastExp = -117, kMostExp = 119;
constexpr float kMostCode = 448.f; // 1.75 * 2^8

__device__ __forceinline__ int scale_byte(float amax) { // amax: finite, not negative
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - (127 + 8) + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (e < kLeastExp ? kLeastExp : e > kMostExp ? kMostExp : e) + 127;
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four features times 1 / 2^e as codes.  (The conversion rounds to nearest even, keeps NaN, and is not asked for more than 448.)
__device__ __forceinline__ uint32_t codes_of(float x0, float x1, float x2, float x3) {
    auto held = [](float x) { return fabsf(x) < INFINITY ? fminf(fmaxf(x, -kMostCode), kMostCode) : NAN; };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(held(x0), held(x1), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(held(x2), held(x3), w, true);
}

// Two codes of a word as two bf16, exactly.
template <bool UPPER>
__device__ __forceinline__ uint32_t bf16_of_codes(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, UPPER));
}
template <bool UPPER>
__device__ __forceinline__ f32x2 f32_of_codes(uint32_t codes, float scale) {
    return __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, UPPER));
}
// 16 bytes of features from codes: 8 (bf16, two words) or 4 (fp32, one).
__device__ __forceinline__ raw16 bf16_piece(uint32_t lower, uint32_t upper, float scale) {
    return raw16{bf16_of_codes<false>(lower, scale), bf16_of_codes<true>(lower, scale), bf16_of_codes<false>(upper, scale), bf16_of_codes<true>(upper, scale)};
}
__device__ __forceinline__ raw16 f32_piece(uint32_t codes, float scale) {
    const f32x2 a = f32_of_codes<false>(codes, scale), b = f32_of_codes<true>(codes, scale);
    return raw16{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
}

} // namespace mukv
