// Numbers to e4m3: the scale of a block, and the conversion.
#pragma once
#include "seq_internal.h"

namespace xls {

static constexpr float E4M3_MAX = 448.f, MIN_SCALE = 1.17549435e-38f;

// The largest |x| as the bits of a float: the order of the bits is the order of the numbers, infinity and then NaN above them.
__device__ __forceinline__ unsigned magnitude(float x) { return __builtin_bit_cast(unsigned, x) & 0x7fffffffu; }
__device__ __forceinline__ float scale_of(unsigned most)
{
    const float s = __builtin_bit_cast(float, most) / E4M3_MAX;
    return s < MIN_SCALE ? MIN_SCALE : s;      // a NaN stays
}

__device__ __forceinline__ unsigned e4m3x4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

}  // namespace xls
