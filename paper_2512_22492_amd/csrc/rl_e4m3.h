// rl_e4m3.h -- rounding to e4m3 codes, as the appends store them (gfx950).
// Internal header.
#pragma once

#include "rl_common.h"

namespace rl_da {

// Two fp32 values to two e4m3 codes (round to nearest even) in the low 16 bits.
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b)
{
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
}

__device__ __forceinline__ float clamp448(float v)
{
    // comparisons, not fminf/fmaxf, so that a NaN passes through unchanged
    return v > 448.0f ? 448.0f : (v < -448.0f ? -448.0f : v);
}

}  // namespace rl_da
