// The 8-bit cache's element type: e4m3 codes and power-of-two scales.
#pragma once

#include "common.hpp"

namespace tf {

constexpr float kE4m3Max = 448.f;
// a page's scale stays in 2^-kScaleExp .. 2^kScaleExp
constexpr int kScaleExp = 64;

// The smallest power of two s with amax <= 448 s.  448 = 1.75 * 2^8, so for
// amax = m * 2^e it is 2^(e-8), one more where m > 1.75: exact, by integers.
__device__ __forceinline__ float pow2_scale(float amax) {
    const uint32_t u = __float_as_uint(amax);
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = min(max(e, -kScaleExp), kScaleExp);   // 0 and denormals land on the smallest
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// Two codes of a dword's lower (HI = false) or upper half as floats, exact.
typedef float f32pair __attribute__((ext_vector_type(2)));
template <bool HI>
__device__ __forceinline__ f32pair e4m3_pair(uint32_t w) {
    return __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HI);
}

// Held to +-448 with NaN kept: v_cvt would make NaN of what is larger.
__device__ __forceinline__ float e4m3_clamp(float x) { return x != x ? x : fminf(fmaxf(x, -kE4m3Max), kE4m3Max); }

// Four floats as codes, rounded to nearest even (the format's own precision:
// what the cache is for).
__device__ __forceinline__ uint32_t e4m3_quad(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(a), e4m3_clamp(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(c), e4m3_clamp(d), w, true);
}

// Four codes of scale `old` as codes of scale old / ratio.
__device__ __forceinline__ uint32_t e4m3_rescale(uint32_t w, float ratio) {
    const f32pair a = e4m3_pair<false>(w), b = e4m3_pair<true>(w);
    return e4m3_quad(a[0] * ratio, a[1] * ratio, b[0] * ratio, b[1] * ratio);
}

}  // namespace tf
