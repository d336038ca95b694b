// out[t] = sum_j weight[t][j] y[row of (t, j)] + residual[t], for every rank (formulas in include/symar.h): the experts' rows back in the
// tokens' order.
//
// A thread has eight channels of one token and asks for up to eight of its rows at once; they are added in the order of
// the token's choices, so that results do not depend on anything else.  Bound by the rows' bytes.
#include "symar_eights.cuh"
#include "symar_ops.h"

namespace symar {
namespace {

struct CombineArgs {
    const void    *y, *residual;
    const int32_t *token_row;
    const float   *weights;
    void          *out;
    int64_t y_ld, y_group, residual_ld, residual_group, out_ld, out_group, cells;      // cells: tokens of all groups
    int     tokens, top_k, rows, n, root;
    int     y_wide, out_wide;
    int     lanes, parts;                  // threads of a token, and of how many blocks' worth each
};
constexpr int kMost = 1 << 30;              // channels: their last step ends below 2^31
constexpr int kThreads = 256, kAtOnce = 8;

template <bool kVec>
__global__ void __launch_bounds__(kThreads) combine_kernel(const __grid_constant__ CombineArgs a)
{
    wait_for_stream();
    // `lanes` threads have 8 * lanes channels of a token; a block has kThreads / lanes tokens, or a part of one
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / a.lanes) + threadIdx.x / a.lanes, cell = unit / a.parts;
    if (cell >= a.cells) return;
    const int g = (int)(cell / a.tokens), t = (int)(cell - (int64_t)g * a.tokens);
    const int i = (int)(unit - cell * a.parts) * a.lanes + (int)threadIdx.x % a.lanes, first = kVec ? 8 * i : i, step = a.lanes * a.parts;
    const int32_t *at = a.token_row + (int64_t)t * a.top_k;
    const float *w = a.weights ? a.weights + (int64_t)t * a.top_k : nullptr;
    const char *y = static_cast<const char *>(a.y) + g * a.y_group * (a.y_wide ? 4 : 2);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int j0 = 0; j0 < a.top_k; j0 += kAtOnce) {
        Raw   r[kAtOnce];
        float by[kAtOnce];
        bool  on[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int row = j0 + j < a.top_k ? at[j0 + j] : -1;
            on[j] = row >= 0 && row < a.rows;
            by[j] = on[j] && w ? w[j0 + j] : 1.0f;
            if (on[j]) r[j] = read8<kVec>(y + row * a.y_ld * (a.y_wide ? 4 : 2), a.y_wide, first, step, a.n);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (!on[j]) continue;
            float v[8];
            values<kVec>(r[j], a.y_wide, v);
#pragma unroll
            for (int c = 0; c < 8; ++c) sum[c] = fmaf(by[j], v[c], sum[c]);
        }
    }
    if (a.residual && (a.root < 0 || a.root == g)) {
        const char *p = static_cast<const char *>(a.residual) + (g * a.residual_group + t * a.residual_ld) * (a.out_wide ? 4 : 2);
        float v[8];
        values<kVec>(read8<kVec>(p, a.out_wide, first, step, a.n), a.out_wide, v);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] += v[c];
    }
    write8<kVec>(static_cast<char *>(a.out) + (g * a.out_group + t * a.out_ld) * (a.out_wide ? 4 : 2), a.out_wide, first, step, a.n, sum);
}

bool dtype_ok(int d) { return d == SYMAR_F32 || d == SYMAR_BF16; }

}  // namespace
}  // namespace symar

using namespace symar;

extern "C" int symar_combine(const symar_combine_t *args, void *cuda_stream)
{
    if (!args) return SYMAR_ERR_INVAL;
    const symar_combine_t &p = *args;
    if (p.groups < 0 || p.tokens < 0 || p.top_k < 0 || p.rows < 0 || p.n < 0 || !dtype_ok(p.dtype) || !dtype_ok(p.out_dtype)) return SYMAR_ERR_INVAL;
    if (p.root < -1 || (p.root >= p.groups && p.groups > 0)) return SYMAR_ERR_INVAL;
    const uintptr_t yw = p.dtype == SYMAR_F32 ? 4 : 2, ow = p.out_dtype == SYMAR_F32 ? 4 : 2;
    if ((uintptr_t)p.y % yw || ((uintptr_t)p.out | (uintptr_t)p.residual) % ow || ((uintptr_t)p.token_row | (uintptr_t)p.weights) % 4) return SYMAR_ERR_INVAL;
    const int64_t strides[6] = {p.y_ld, p.y_group, p.residual_ld, p.residual_group, p.out_ld, p.out_group};
    bool vec = ((uintptr_t)p.y | (uintptr_t)p.out | (uintptr_t)p.residual) % 16 == 0 && p.n % 8 == 0;
    for (int64_t s : strides) {
        if (s < 0) return SYMAR_ERR_INVAL;
        vec = vec && s % 8 == 0;
    }
    if (p.n > kMost) return SYMAR_ERR_UNSUPPORTED;
    if (p.groups == 0 || p.tokens == 0 || p.n == 0) return SYMAR_OK;
    if (!p.out || (p.top_k > 0 && (!p.token_row || (p.rows > 0 && !p.y)))) return SYMAR_ERR_INVAL;
    if (rows_meet(p.tokens, p.out_ld, p.groups, p.out_group, p.n)) return SYMAR_ERR_INVAL;
    CombineArgs a{};
    a.y = p.y;  a.y_ld = p.y_ld;  a.y_group = p.y_group;
    a.residual = p.residual;  a.residual_ld = p.residual_ld;  a.residual_group = p.residual_group;
    a.out = p.out;  a.out_ld = p.out_ld;  a.out_group = p.out_group;
    a.token_row = p.token_row;  a.weights = p.weights;
    a.cells = (int64_t)p.groups * p.tokens;
    a.tokens = p.tokens;  a.top_k = p.top_k;  a.rows = p.rows;  a.n = p.n;  a.root = p.root;
    a.y_wide = p.dtype == SYMAR_F32;  a.out_wide = p.out_dtype == SYMAR_F32;
    a.lanes = 1;
    while (a.lanes < kThreads && a.lanes * 8 < p.n) a.lanes *= 2;
    a.parts = (p.n + a.lanes * 8 - 1) / (a.lanes * 8);
    const int64_t per = kThreads / a.lanes, blocks = (a.cells * a.parts + per - 1) / per;
    if (blocks > 0x7fffffff) return SYMAR_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const cudaError_t e = vec ? launch_early(combine_kernel<true>, dim3((unsigned)blocks), kThreads, 0, s, a)
                              : launch_early(combine_kernel<false>, dim3((unsigned)blocks), kThreads, 0, s, a);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_combine");
}
