// 4-bit weights (moe_few.h): the two formats, as the kernels see them.
#pragma once

#include "../../include/moe_few.h"
#include "common.h"

namespace moe {

inline int64_t q4_scale_cols(int64_t cols, int group) { return (cols + group - 1) / group; }

#if defined(__HIP_DEVICE_COMPILE__)
// The scale of an FP4 group, 2^(s - 127), from its byte (0 stands for 2^-127 and is flushed).
__device__ __forceinline__ float fp4_scale(uint32_t s) { return __uint_as_float(s << 23); }

// Eight codes (a register) as fp32 values under one scale.
template <int kFormat>
__device__ __forceinline__ void q4_values(uint32_t codes, float scale, float v[8])
{
    if constexpr (kFormat == MOE_Q4_FP4) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
        const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
        v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = (float)((int)((codes >> (4 * i)) & 15u) - 8) * scale;
    }
}
#endif

}  // namespace moe
