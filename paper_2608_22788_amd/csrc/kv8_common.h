// kv8_common.h -- the cache held in 8 bits: e4m3 codes in pages laid out as those
// of the bf16 cache ([num_pages][Hkv][16][D], one byte a value), and for each
// page and KV head a power of two for its keys and one for its values, as biased
// exponent bytes ([num_pages][Hkv][2], e8m0).  A value is code * 2^(byte - 127).
//
// Why powers of two.  The product of a code (4 significant bits) with one is
// exact in bf16, so that the conversion in front of a matrix product takes it
// along (one instruction for two values); and when a later token raises a page's
// power, the codes that the page holds already only move their exponents, so a
// value is rounded once (again only below 2^-6 of the power, where e4m3 is
// denormal).  A rounding is off by at most max(2^-4 of the value, 2^-10 of the
// power): values below 2^-10 of their page's power, beside one that is far larger,
// become zero.
#pragma once

#include "attn_common.h"

namespace tsattn {

constexpr int kLowestPower = 27, kHighestPower = 227;   // bytes that an append writes: 2^-100 .. 2^100
constexpr float kLargestCode = 448.0f;

// 2^(byte - 127), byte 1 .. 254.
__device__ __forceinline__ float power_of(int byte) { return __int_as_float(byte << 23); }

// The byte of the smallest power with amax <= 448 * power (amax finite), inside
// the range that is written.  448 is 1.75 * 2^8.
__device__ __forceinline__ int power_for(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int byte = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
    return min(max(byte, kLowestPower), kHighestPower);
}

// Four values times `inv` as codes, nearest even, saturating; what is infinite or
// NaN becomes the NaN code (e4m3 has no infinity).
__device__ __forceinline__ float code_value(float x, float inv) {
    return fabsf(x) < INFINITY ? __builtin_amdgcn_fmed3f(x * inv, -kLargestCode, kLargestCode) : __uint_as_float(0x7fc00000u);
}
__device__ __forceinline__ uint32_t pack_codes4(const float *x, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(code_value(x[0], inv), code_value(x[1], inv), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_value(x[2], inv), code_value(x[3], inv), w, true);
}
// Eight values over `power` as codes, nearest even, where none is larger than 448 times
// it, infinite or NaN: the conversion divides by the power itself.
typedef short s16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2_t codes8(const float x[8], float power) {
    s16x2_t w[2] = {};
#pragma unroll
    for (int i = 0; i < 2; i++) {
        w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], x[4 * i], x[4 * i + 1], power, false);
        w[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w[i], x[4 * i + 2], x[4 * i + 3], power, true);
    }
    return u32x2_t{__builtin_bit_cast(uint32_t, w[0]), __builtin_bit_cast(uint32_t, w[1])};
}
// Four codes times `factor` as codes.
__device__ __forceinline__ uint32_t scale_codes4(uint32_t w, float factor) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    const float x[4] = {lo[0], lo[1], hi[0], hi[1]};
    return pack_codes4(x, factor);
}

}  // namespace tsattn
