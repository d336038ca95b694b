// What follows a product's sums: activations on four values, and four neighbouring elements read and written.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "symar.h"

namespace symar {

// y / 2 (1 + tanh u) = y / (1 + exp(-2u)); the quotient's two units in the last place are far below the result's rounding
__device__ __forceinline__ float gate(float y, float two_u) { return __fdividef(y, 1.0f + expf(-two_u)); }
__device__ __forceinline__ void activate4(float (&y)[4], int act)
{
    if (act == SYMAR_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = y[i] < 0.0f ? 0.0f : y[i];
    } else if (act == SYMAR_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = 0.5f * y[i] * (1.0f + erff(y[i] * 0.70710678118654752f));
    } else if (act == SYMAR_ACT_GELU_TANH) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = gate(y[i], 1.5957691216057308f * (y[i] + 0.044715f * y[i] * y[i] * y[i]));
    } else if (act == SYMAR_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = gate(y[i], y[i]);
    }
}
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void load4(const float *p, float (&r)[4])
{
    const float4 v = *reinterpret_cast<const float4 *>(p);
    r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16 *p, float (&r)[4])
{
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    r[0] = __uint_as_float(v.x << 16); r[1] = __uint_as_float(v.x & 0xffff0000u);
    r[2] = __uint_as_float(v.y << 16); r[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void put4(float *p, const float (&r)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(r[0], r[1], r[2], r[3]); }
__device__ __forceinline__ void put4(__nv_bfloat16 *p, const float (&r)[4])
{
    __nv_bfloat162 lo = __floats2bfloat162_rn(r[0], r[1]), hi = __floats2bfloat162_rn(r[2], r[3]);
    *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<uint32_t *>(&lo), *reinterpret_cast<uint32_t *>(&hi));
}

}  // namespace symar
