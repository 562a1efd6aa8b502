// Values of 4-bit tiles (TRE_MXFP4), for the kernels that read them back.
#pragma once

#include "tre_internal.h"

namespace tre {

// The eight values of four code bytes under a block's scale byte.  (The
// conversion takes its scale from the exponent field alone, so a field of 0 is
// 2^-127; of 255, NaN, it makes no use.)
__device__ inline void mx_values(uint32_t codes, int scale, float (&v)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float s = __uint_as_float(uint32_t(scale) << 23);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
    const float x[8] = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = scale == kMxNanScale ? __uint_as_float(0x7fc00000u) : x[i];
}

}  // namespace tre
