// Device helpers of the attention kernels that read the paged cache (internal to the library).
#pragma once
#include "attn_common.h"

namespace bs {

// The largest value, the sum, of the four lanes that hold the slots of one query row.
__device__ inline float max_across_groups(float x)
{
    x = max_across_halves(x);
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_across_groups(float x)
{
    x = sum_across_halves(x);
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ inline void store_row4(__bf16 *to, float4 x)
{
    bf16x4 w;
    w[0] = (__bf16)x.x; w[1] = (__bf16)x.y; w[2] = (__bf16)x.z; w[3] = (__bf16)x.w;
    *reinterpret_cast<bf16x4 *>(to) = w;
}
__device__ inline void store_row4(float *to, float4 x) { *reinterpret_cast<float4 *>(to) = x; }

}  // namespace bs
