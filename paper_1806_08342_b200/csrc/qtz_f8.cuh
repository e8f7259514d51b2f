// Shared by the translation units of the 8-bit floating-point operators (e4m3 codes, a scale for each block of 128).
#pragma once

#include <stdint.h>

#include "qtz_half_util.cuh"
#include "qtz_internal.cuh"

constexpr int kF8Block = 128;                          // columns (of weights: rows, too) that share a scale
constexpr float kF8Top = 448.f;                        // largest e4m3 value
constexpr float kF8MinScale = 7.888609052210118e-31f;  // 2^-100: the scale of a block of zeros

namespace qtz_dev {

// Two e4m3 codes, the lower byte first: rounded to nearest even, values beyond 448 saturate, NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi)
{
    uint16_t v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(hi), "f"(lo));
    return v;
}

// Scale of a block whose largest magnitude is `top` (infinities and NaN left out).
__device__ __forceinline__ float f8_scale(float top) { return fmaxf(top / kF8Top, kF8MinScale); }

__device__ __forceinline__ float load_real(const void* p, int64_t i, int ftype)
{
    if (ftype == QTZ_F32) return static_cast<const float*>(p)[i];
    if (ftype == QTZ_F16) return __half2float(static_cast<const __half*>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

}  // namespace qtz_dev

static inline bool qtz_is_real(int32_t ftype) { return ftype == QTZ_F32 || ftype == QTZ_F16 || ftype == QTZ_BF16; }
