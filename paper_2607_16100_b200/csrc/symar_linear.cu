// out_g = act(x_g w_g^T + bias_g) + residual_g, one matrix per rank (formulas in include/symar.h).
#include "symar_ops.h"

namespace symar {
namespace {

struct LinearArgs {
    const __nv_bfloat16 *x, *w, *bias;
    const void *residual;
    void       *out;
    int64_t x_ld, x_group, w_ld, w_group, bias_group, residual_ld, residual_group, out_ld, out_group;
    int     m, n, k, act, root;
};

__device__ __forceinline__ float activate(float y, int act)
{
    switch (act) {
        case SYMAR_ACT_RELU: return y < 0.0f ? 0.0f : y;
        case SYMAR_ACT_GELU: return 0.5f * y * (1.0f + erff(y * 0.70710678118654752f));
        case SYMAR_ACT_GELU_TANH: return 0.5f * y * (1.0f + tanhf(0.79788456080286536f * (y + 0.044715f * y * y * y)));
        case SYMAR_ACT_SILU: return y / (1.0f + expf(-y));
    }
    return y;
}
__device__ __forceinline__ float as_f32(float v) { return v; }
__device__ __forceinline__ float as_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

constexpr int kTile = 64, kStep = 16;

template <typename O>
__global__ void __launch_bounds__(256) linear_kernel(const LinearArgs a)
{
    __shared__ float xs[kStep][kTile + 1], ws[kStep][kTile + 1];
    const int g = blockIdx.z, m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
    const __nv_bfloat16 *x = a.x + g * a.x_group, *w = a.w + g * a.w_group;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < a.k; k0 += kStep) {
        for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
            const int r = i / kStep, k = k0 + i % kStep;
            xs[i % kStep][r] = m0 + r < a.m && k < a.k ? __bfloat162float(x[(int64_t)(m0 + r) * a.x_ld + k]) : 0.0f;
            ws[i % kStep][r] = n0 + r < a.n && k < a.k ? __bfloat162float(w[(int64_t)(n0 + r) * a.w_ld + k]) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < kStep; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[k][ty + 16 * i], ws[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
    const bool mine = a.root < 0 || a.root == g;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m >= a.m || n >= a.n) continue;
            float y = acc[i][j];
            if (mine && a.bias) y += __bfloat162float(a.bias[g * a.bias_group + n]);
            y = activate(y, a.act);
            if (mine && a.residual) y += as_f32(static_cast<const O *>(a.residual)[g * a.residual_group + m * a.residual_ld + n]);
            put(static_cast<O *>(a.out) + g * a.out_group + m * a.out_ld + n, y);
        }
}

}  // namespace
}  // namespace symar

using namespace symar;

extern "C" int symar_linear(const symar_linear_t *args, void *cuda_stream)
{
    if (!args) return SYMAR_ERR_INVAL;
    const symar_linear_t &p = *args;
    if (p.groups < 0 || p.m < 0 || p.n < 0 || p.k < 0 || p.act < SYMAR_ACT_NONE || p.act > SYMAR_ACT_SILU) return SYMAR_ERR_INVAL;
    if (p.out_dtype != SYMAR_F32 && p.out_dtype != SYMAR_BF16) return SYMAR_ERR_INVAL;
    if (p.root < -1 || (p.root >= p.groups && p.groups > 0)) return SYMAR_ERR_INVAL;
    if (p.groups > 65535) return SYMAR_ERR_UNSUPPORTED;
    if (p.groups == 0 || p.m == 0 || p.n == 0) return SYMAR_OK;
    const uintptr_t wide = p.out_dtype == SYMAR_F32 ? 4 : 2;
    if (!p.out || (p.k > 0 && (!p.x || !p.w))) return SYMAR_ERR_INVAL;
    if (((uintptr_t)p.x | (uintptr_t)p.w | (uintptr_t)p.bias) % 2 || ((uintptr_t)p.out | (uintptr_t)p.residual) % wide) return SYMAR_ERR_INVAL;
    if ((p.groups > 1 && p.out_group == 0) || (p.m > 1 && p.out_ld < p.n)) return SYMAR_ERR_INVAL;
    LinearArgs a{(const __nv_bfloat16 *)p.x, (const __nv_bfloat16 *)p.w, (const __nv_bfloat16 *)p.bias, p.residual, p.out,
                 p.x_ld, p.x_group, p.w_ld, p.w_group, p.bias_group, p.residual_ld, p.residual_group, p.out_ld, p.out_group,
                 p.m, p.n, p.k, p.act, p.root};
    const int mt = (p.m + kTile - 1) / kTile, nt = (p.n + kTile - 1) / kTile;
    if (mt > 65535) return SYMAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)nt, (unsigned)mt, (unsigned)p.groups);
    if (p.out_dtype == SYMAR_F32) linear_kernel<float><<<grid, 256, 0, (cudaStream_t)cuda_stream>>>(a);
    else linear_kernel<__nv_bfloat16><<<grid, 256, 0, (cudaStream_t)cuda_stream>>>(a);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_linear");
}
