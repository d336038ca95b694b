// Rows read and written eight elements a thread, bf16 or float32 as a call says.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace symar {

// Eight elements as they were read: packed pairs (bf16 in one load) or one a word.
struct Raw {
    uint32_t w[8];
};

// A thread's eight elements of a row of n: side by side from `first` on (kVec: rows on 16-byte boundaries, n and `first` multiples of
// eight), or every `step`th.
template <bool kVec>
__device__ __forceinline__ Raw read8(const void *p, bool wide, int first, int step, int n)
{
    Raw r;
    if (kVec) {
        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
        if (first < n) {
            const char *q = static_cast<const char *>(p) + (int64_t)first * (wide ? 4 : 2);
            lo = *reinterpret_cast<const uint4 *>(q);
            if (wide) hi = *reinterpret_cast<const uint4 *>(q + 16);
        }
        r.w[0] = lo.x; r.w[1] = lo.y; r.w[2] = lo.z; r.w[3] = lo.w;
        r.w[4] = hi.x; r.w[5] = hi.y; r.w[6] = hi.z; r.w[7] = hi.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = first + j * step;
            r.w[j] = 0;
            if (at < n) r.w[j] = wide ? static_cast<const uint32_t *>(p)[at] : (uint32_t) static_cast<const uint16_t *>(p)[at] << 16;
        }
    }
    return r;
}
template <bool kVec>
__device__ __forceinline__ void values(const Raw &r, bool wide, float (&v)[8])
{
    if (kVec && !wide) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[2 * j]     = __uint_as_float(r.w[j] << 16);
            v[2 * j + 1] = __uint_as_float(r.w[j] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(r.w[j]);
    }
}
template <bool kVec>
__device__ __forceinline__ void write8(void *p, bool wide, int first, int step, int n, const float *v)
{
    if (kVec) {
        if (first >= n) return;
        char *q = static_cast<char *>(p) + (int64_t)first * (wide ? 4 : 2);
        if (wide) {
            *reinterpret_cast<float4 *>(q)      = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(q + 16) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
                w[j] = *reinterpret_cast<uint32_t *>(&h);
            }
            *reinterpret_cast<uint4 *>(q) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = first + j * step;
            if (at >= n) continue;
            if (wide) static_cast<float *>(p)[at] = v[j];
            else static_cast<__nv_bfloat16 *>(p)[at] = __float2bfloat16_rn(v[j]);
        }
    }
}

}  // namespace symar
