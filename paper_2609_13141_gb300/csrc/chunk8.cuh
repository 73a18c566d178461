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

}  // namespace
}  // namespace sas
