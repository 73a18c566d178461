// What the two kernels of attention over an 8-bit cache share.
#pragma once

#include <cfloat>

#include "serve_ptx.cuh"

namespace sas {
namespace {

// What takes a product of f16 queries and e4m3 keys to a score in log2 units: the row's factor times the page's key
// scale, kept within the normal numbers.  It underflows where queries of zeros or near it (2^-117) meet keys of zeros
// (2^-64), and 0 times a masked score's -infinity is NaN; the least normal number moves no score by more than 2^-90 (a
// product is below 2^15 448 d).  It overflows where both are large, and a product of 0 times infinity is NaN; the largest
// number leaves a product of 0 its score, 0, and the others past fp32's range.  NaN stays.
__device__ __forceinline__ float score_factor(float row, float page) {
    float f;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(f) : "f"(row * page), "f"(FLT_MIN));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(f) : "f"(f), "f"(FLT_MAX));
    return f;
}

// Sums of weights times values stand under a unit, a power of two, and go over to a page's value scale where the two are
// far apart (kScaleRange).  They would leave fp32 where a request has 2^120 and then a page of zeros' 2^-64, or falls in
// several steps, so a unit falls only as far as sums of up to `top` stay below 2^120.  Returns what the sums are
// multiplied by; `unit` becomes their new one.  A page whose scale stays far below the unit adds less than what the
// larger values' weights are rounded by.  A unit that rises takes sums along to 2^-149 of it, fp32's least number:
// where that factor is below kFarRise, which may be less than fp32 has, in two steps, the first one 2^-64.
constexpr float kFarRise = 7.888609052210118e-31f, kRiseStep = 5.421010862427522e-20f, kRiseRest = 18446744073709551616.f;   // 2^-100, 2^-64, 2^64
__device__ __forceinline__ float move_unit(float& unit, float scale, float top) {
    const int e = max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -6);   // top < 2^(e + 1)
    const float whole = unit / scale, most = __uint_as_float(static_cast<uint32_t>(127 + 119 - e) << 23);
    unit = top == 0.f || whole <= most ? scale : unit / most;
    return fminf(whole, most);
}
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) <= FLT_MAX ? fabsf(x) : 0.f; }

// Sums that leave the kernel or a warp before they are divided by the sum of weights (below 2^29: 2^21 keys, weights up
// to 2^8) may pass fp32 though the output does not, where scales are above kLargeScale: such ones, and their sum of weights,
// are made smaller by 2^kShrink, and the maximum that they are relative to is larger by as much.
constexpr float kLargeScale = 1152921504606846976.f;   // 2^60
constexpr float kShrink = 40.f, kShrinkFactor = 9.094947017729282e-13f;   // 2^-40

}  // namespace
}  // namespace sas
