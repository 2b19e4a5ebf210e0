// FP8 E4M3 cache with a scale for each block of 16 tokens, KV head and part (K, V): how a scale follows from the values, and how
// codes move from one scale to a larger one.
//
// A scale is a power of two.  A float format has the same relative precision at every exponent, so nothing is lost against a scale
// of amax / 448 but up to one bit at the bottom of the range, and three things are gained: code * scale is a bf16 value exactly
// (the kernels that work on bf16 see what the cache stands for, without another rounding), v_cvt_scalef32_pk_bf16_fp8 applies
// it in the widening instruction itself, and a block whose scale grows keeps its codes' mantissas: going from scale s to 2^n s is
// exact but for codes that become subnormal, however often it happens while a block fills.
#pragma once
#include "internal.h"

namespace shiftattn {

// exponents of a scale: below 2^-100 nothing is worth keeping, above 2^119 a saturated code (448) would overflow
constexpr int kScaleExpMin = -100, kScaleExpMax = 119;

// bits of |x| of a finite x, 0 for an infinity or a NaN: maxima of these are maxima of magnitudes
__device__ inline uint32_t finite_magnitude(float x) {
    const uint32_t a = __float_as_uint(x) & 0x7FFFFFFFu;
    return a < 0x7F800000u ? a : 0u;
}

// least power of two s with top <= 448 s, 448 = 1.75 * 2^8: a mantissa beyond 1.75 carries into the exponent
__device__ inline float block_scale(uint32_t top) {
    int e = static_cast<int>((top + 0x1FFFFFu) >> 23) - 8;
    e = min(max(e, 127 + kScaleExpMin), 127 + kScaleExpMax);
    return __uint_as_float(static_cast<uint32_t>(e) << 23);
}

// four codes times ratio (a power of two below 1), rounded to the nearest code, ties to the even one
__device__ inline uint32_t rescale_codes(uint32_t codes, float ratio) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes), true);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * ratio, lo[1] * ratio, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * ratio, hi[1] * ratio, w, true);
    return static_cast<uint32_t>(w);
}

}  // namespace shiftattn
