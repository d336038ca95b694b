// out[t] = sum_j weight[t][j] y[row of (t, j)] + residual[t], for every rank (formulas in include/symar.h): the experts' rows back in the
// tokens' order.
//
// A thread has eight channels of one token and asks for its pieces of up to eight rows at once; a token's rows are added in the order
// of its choices, so that results do not depend on anything else.  Bound by the rows' bytes: 8192 tokens x 4 rows x 4096 take 57.8 us for 333 MB
// (5.75 TB/s, 0.88 of the measured copy rate); rows on no 16-byte boundary (4097) 143 us, whose elements are read and written one by one.
#include "symar_eights.cuh"
#include "symar_ops.h"

namespace symar {
namespace {

struct CombineArgs {
    const void    *y, *residual;
    const int32_t *token_row;
    const float   *weights;
    void          *out;
    int64_t y_ld, y_group, residual_ld, residual_group, out_ld, out_group;
    int     tokens, top_k, rows, n, root;
    int     lanes, parts;                  // threads of a token (a power of two), and into how many blocks its channels are divided
};
constexpr int kMost = 1 << 30;              // channels: their last step ends below 2^31
constexpr int kThreads = 256;

// Blocks of a multiprocessor: more of them hide more of the two dependent trips to memory, until their registers no longer hold what is on its way (four
// rows a token: 8 blocks 57.8 us, 5 62, as many as 54 registers allow 67; eight rows 5 blocks 50.4, 6 53).
constexpr int blocks_for(bool vec, bool wide, int rows) { return !vec ? 6 : rows == 8 ? (wide ? 3 : 4) : rows == 4 ? (wide ? 5 : 8) : 6; }

// kY, kOut: y and the results are float32.  K: rows asked for at once.
template <bool kVec, bool kY, bool kOut, int K>
__global__ void __launch_bounds__(kThreads, blocks_for(kVec, kY, K)) combine_kernel(const __grid_constant__ CombineArgs a)
{
    wait_for_stream();
    // a token's channels are divided into `parts` of eight a thread; on no boundary a warp has 256 in a row, a thread every thirty-second of them
    constexpr int step = 32;
    const unsigned lanes = kVec ? a.lanes : 32, per = kThreads / lanes, unit = blockIdx.x * per + threadIdx.x / lanes;
    const unsigned block = kVec ? blockIdx.x / (unsigned)a.parts : 0, part = kVec ? blockIdx.x - block * a.parts : unit % (unsigned)a.parts;
    const int g = blockIdx.y, t = (int)(kVec ? block * per + threadIdx.x / lanes : unit / (unsigned)a.parts);
    if (t >= a.tokens) return;
    const int first = 8 * (int)(part * lanes) + (kVec ? 8 : 1) * (int)(threadIdx.x & (lanes - 1));
    const int32_t *at = a.token_row + (int64_t)t * a.top_k;
    const float *w = a.weights ? a.weights + (int64_t)t * a.top_k : nullptr;
    const char *y = static_cast<const char *>(a.y) + g * a.y_group * (kY ? 4 : 2);
    float sum[8] = {};
    for (int j0 = 0; j0 < a.top_k; j0 += K) {
        int   row[K];
        float by[K];
        Raw   r[K];
#pragma unroll
        for (int j = 0; j < K; ++j) {
            row[j] = j0 + j < a.top_k ? at[j0 + j] : -1;
            by[j]  = j0 + j < a.top_k && w ? w[j0 + j] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const bool on = (unsigned)row[j] < (unsigned)a.rows;
            by[j] = on ? by[j] : 0.0f;     // (and zeros times that)
            r[j] = read8<kVec>(y + (on ? row[j] : 0) * a.y_ld * (kY ? 4 : 2), kY, first, step, on ? a.n : 0);
        }
#pragma unroll
        for (int j = 0; j < K; ++j) {
            float v[8];
            values<kVec>(r[j], kY, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = fmaf(by[j], v[e], sum[e]);
        }
    }
    if (a.residual && (a.root < 0 || a.root == g)) {
        const char *res = static_cast<const char *>(a.residual) + (g * a.residual_group + t * a.residual_ld) * (kOut ? 4 : 2);
        float v[8];
        values<kVec>(read8<kVec>(res, kOut, first, step, a.n), kOut, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += v[e];
    }
    write8<kVec>(static_cast<char *>(a.out) + (g * a.out_group + t * a.out_ld) * (kOut ? 4 : 2), kOut, first, step, a.n, sum);
}
template <bool kVec, bool kY, bool kOut, int K>
cudaError_t launch(CombineArgs a, int groups, cudaStream_t s)
{
    a.lanes = kVec ? 1 : 32;
    while (kVec && a.lanes < kThreads && a.lanes * 8 < a.n) a.lanes *= 2;
    a.parts = (a.n + a.lanes * 8 - 1) / (a.lanes * 8);
    const int64_t per = kThreads / a.lanes, blocks = kVec ? (a.tokens + per - 1) / per * a.parts : ((int64_t)a.tokens * a.parts + per - 1) / per;
    return launch_early(combine_kernel<kVec, kY, kOut, K>, dim3((unsigned)blocks, (unsigned)groups), kThreads, 0, s, a);
}
template <bool kVec, bool kY, bool kOut>
cudaError_t launch_of(const CombineArgs &a, int groups, cudaStream_t s)
{
    if (a.top_k <= 2) return launch<kVec, kY, kOut, 2>(a, groups, s);
    if constexpr (kVec)
        if (a.top_k > 4) return launch<true, kY, kOut, 8>(a, groups, s);
    return launch<kVec, kY, kOut, 4>(a, groups, s);
}
template <bool kVec>
cudaError_t launch_as(const CombineArgs &a, int groups, bool y_wide, bool out_wide, cudaStream_t s)
{
    if (y_wide) return out_wide ? launch_of<kVec, true, true>(a, groups, s) : launch_of<kVec, true, false>(a, groups, s);
    return out_wide ? launch_of<kVec, false, true>(a, groups, s) : launch_of<kVec, false, false>(a, groups, s);
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
    if (p.n > kMost || p.groups > 65535 || (int64_t)p.tokens * ((p.n + 255) / 256) > 0x7fffffff) return SYMAR_ERR_UNSUPPORTED;
    if (p.groups == 0 || p.tokens == 0 || p.n == 0) return SYMAR_OK;
    if (!p.out || (p.top_k > 0 && (!p.token_row || (p.rows > 0 && !p.y)))) return SYMAR_ERR_INVAL;
    if (rows_meet(p.tokens, p.out_ld, p.groups, p.out_group, p.n)) return SYMAR_ERR_INVAL;
    CombineArgs a{};
    a.y = p.y;  a.y_ld = p.y_ld;  a.y_group = p.y_group;
    a.residual = p.residual;  a.residual_ld = p.residual_ld;  a.residual_group = p.residual_group;
    a.out = p.out;  a.out_ld = p.out_ld;  a.out_group = p.out_group;
    a.token_row = p.token_row;  a.weights = p.weights;
    a.tokens = p.tokens;  a.top_k = p.top_k;  a.rows = p.rows;  a.n = p.n;  a.root = p.root;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const bool y_wide = p.dtype == SYMAR_F32, out_wide = p.out_dtype == SYMAR_F32;
    const cudaError_t e = vec ? launch_as<true>(a, p.groups, y_wide, out_wide, s) : launch_as<false>(a, p.groups, y_wide, out_wide, s);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_combine");
}
