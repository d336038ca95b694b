// What stands around an AllReduce in a decoder layer (formulas in include/symar.h): the block's result normed, gated, scaled and added to
// the residual stream, and the sum normed for the next block, in one pass over the rows.
//
// A row is read once, held in registers as binary32 through both norms and written once.  Sums go over a thread's own elements,
// then over the row's threads by shuffles and, where they are several warps, by shared memory; a layer norm takes the mean first
// and the squares of what is left after it, so that a large mean costs no digits.
#include "symar_eights.cuh"
#include "symar_ops.h"

namespace symar {
namespace {

struct Side {
    const void *weight, *bias;
    float eps;
    int   kind, wide, plus_one;            // wide: weight and bias are float32
};
struct NormArgs {
    const void *x, *residual, *gate;
    void       *residual_out, *out;
    int64_t x_ld, x_group, residual_ld, residual_group, residual_out_ld, residual_out_group, out_ld, out_group, gate_ld, gate_group;
    Side    after, before;
    float   scale, residual_scale;
    int     m, n, rows;
    int     x_wide, stream_wide, gate_step, gate_act;
};

// Where the eight elements of a thread's chunk c begin; on no 16-byte boundary they are T apart.
template <int T, bool kVec> __device__ __forceinline__ int first(int c, int i) { return kVec ? (c * T + i) * 8 : c * 8 * T + i; }

// Sum over a row's T threads, the same on every one of them; `room` is not in use by an earlier sum any more.
template <int T>
__device__ __forceinline__ float row_sum(float s, float *room)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (T == 32) return s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) room[warp] = s;
    __syncthreads();
    s = lane < T / 32 ? room[lane] : 0.0f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    return s;
}

template <int T, int C, bool kVec>
__device__ __forceinline__ void norm_row(float (&v)[C][8], const Side &s, const Raw &w0, const Raw &b0, int i, int n, float inv_n, float *room)
{
    if (s.kind == SYMAR_NORM_LAYER) {
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[c][j];                       // (elements beyond the row are zeros)
        const float mean = row_sum<T>(sum, room) * inv_n;
        room += 32;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = first<T, kVec>(c, i) + (kVec ? j : j * T) < n ? v[c][j] - mean : 0.0f;
    }
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(v[c][j], v[c][j], sum);
    const float by = 1.0f / sqrtf(fmaf(row_sum<T>(sum, room), inv_n, s.eps));
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] *= by;
        if (s.weight) {
            float w[8];
            values<kVec>(C == 1 ? w0 : read8<kVec>(s.weight, s.wide, first<T, kVec>(c, i), T, n), s.wide, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] *= s.plus_one ? 1.0f + w[j] : w[j];
        }
        if (s.bias) {
            float b[8];
            values<kVec>(C == 1 ? b0 : read8<kVec>(s.bias, s.wide, first<T, kVec>(c, i), T, n), s.wide, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] += b[j];
        }
    }
}
__device__ __forceinline__ float opened(float g, int act)
{
    if (act == SYMAR_GATE_SIGMOID) return 1.0f / (1.0f + expf(-g));
    return act == SYMAR_GATE_TANH ? tanhf(g) : g;
}

constexpr int kSmall = 8;                  // rows of a block where a warp has one

template <int T, int C, bool kVec>
__global__ void __launch_bounds__(T == 32 ? 32 * kSmall : T) norm_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float room[4 * 32];         // two sums of each norm
    wait_for_stream();
    const int row = T == 32 ? (int)blockIdx.x * kSmall + (int)(threadIdx.x >> 5) : (int)blockIdx.x;
    if (row >= a.rows) return;             // (a whole warp)
    const int i = T == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x, g = row / a.m, t = row - g * a.m, n = a.n;
    const float inv_n = 1.0f / (float)n;
    const char *x = static_cast<const char *>(a.x) + (g * a.x_group + t * a.x_ld) * (a.x_wide ? 4 : 2);
    const char *res = static_cast<const char *>(a.residual) + (g * a.residual_group + t * a.residual_ld) * (a.stream_wide ? 4 : 2);

    Raw in[C], old[C], none{}, wa = none, ba = none, wb = none, bb = none;
#pragma unroll
    for (int c = 0; c < C; ++c) in[c] = read8<kVec>(x, a.x_wide, first<T, kVec>(c, i), T, n);
    if (a.residual) {
#pragma unroll
        for (int c = 0; c < C; ++c) old[c] = read8<kVec>(res, a.stream_wide, first<T, kVec>(c, i), T, n);
    }
    if (C == 1) {                          // few rows: everything is asked for at once
        if (a.after.weight) wa = read8<kVec>(a.after.weight, a.after.wide, first<T, kVec>(0, i), T, n);
        if (a.after.bias) ba = read8<kVec>(a.after.bias, a.after.wide, first<T, kVec>(0, i), T, n);
        if (a.before.weight) wb = read8<kVec>(a.before.weight, a.before.wide, first<T, kVec>(0, i), T, n);
        if (a.before.bias) bb = read8<kVec>(a.before.bias, a.before.wide, first<T, kVec>(0, i), T, n);
    }
    float v[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) values<kVec>(in[c], a.x_wide, v[c]);
    if (a.after.kind != SYMAR_NORM_NONE) norm_row<T, C, kVec>(v, a.after, wa, ba, i, n, inv_n, room);
    if (a.gate) {
        const char *gate = static_cast<const char *>(a.gate) + (g * a.gate_group + t * a.gate_ld) * (a.x_wide ? 4 : 2);
        if (a.gate_step == 0) {
            const float by = a.scale * opened(a.x_wide ? *reinterpret_cast<const float *>(gate)
                                                       : __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(gate)), a.gate_act);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= by;
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float w[8];
                values<kVec>(read8<kVec>(gate, a.x_wide, first<T, kVec>(c, i), T, n), a.x_wide, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= a.scale * opened(w[j], a.gate_act);
            }
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] *= a.scale;
    }
    if (a.residual) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float h[8];
            values<kVec>(old[c], a.stream_wide, h);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = fmaf(a.residual_scale, h[j], v[c][j]);
        }
    }
    if (a.residual_out) {
        char *to = static_cast<char *>(a.residual_out) + (g * a.residual_out_group + t * a.residual_out_ld) * (a.stream_wide ? 4 : 2);
#pragma unroll
        for (int c = 0; c < C; ++c) write8<kVec>(to, a.stream_wide, first<T, kVec>(c, i), T, n, v[c]);
    }
    if (a.out) {
        norm_row<T, C, kVec>(v, a.before, wb, bb, i, n, inv_n, room + 64);
        char *to = static_cast<char *>(a.out) + (g * a.out_group + t * a.out_ld) * (a.x_wide ? 4 : 2);
#pragma unroll
        for (int c = 0; c < C; ++c) write8<kVec>(to, a.x_wide, first<T, kVec>(c, i), T, n, v[c]);
    }
}

template <int T, int C>
cudaError_t launch(const NormArgs &a, bool vec, cudaStream_t s)
{
    const unsigned blocks = T == 32 ? ((unsigned)a.rows + kSmall - 1) / kSmall : (unsigned)a.rows, threads = T == 32 ? 32 * kSmall : T;
    return vec ? launch_early(norm_kernel<T, C, true>, dim3(blocks), threads, 0, s, a) : launch_early(norm_kernel<T, C, false>, dim3(blocks), threads, 0, s, a);
}

bool dtype_ok(int d) { return d == SYMAR_F32 || d == SYMAR_BF16; }

}  // namespace
}  // namespace symar

using namespace symar;

extern "C" int symar_norm(const symar_norm_t *args, void *cuda_stream)
{
    if (!args) return SYMAR_ERR_INVAL;
    const symar_norm_t &p = *args;
    if (p.groups < 0 || p.m < 0 || p.n < 0 || !dtype_ok(p.dtype) || !dtype_ok(p.stream_dtype)) return SYMAR_ERR_INVAL;
    if (p.gate_act < SYMAR_GATE_NONE || p.gate_act > SYMAR_GATE_TANH || p.gate_step < 0 || p.gate_step > 1) return SYMAR_ERR_INVAL;
    const uintptr_t xw = p.dtype == SYMAR_F32 ? 4 : 2, sw = p.stream_dtype == SYMAR_F32 ? 4 : 2;
    uintptr_t at = (uintptr_t)p.x | (uintptr_t)p.out | (uintptr_t)(p.gate_step ? p.gate : nullptr), st = (uintptr_t)p.residual | (uintptr_t)p.residual_out;
    if ((at | (uintptr_t)p.gate) % xw || st % sw) return SYMAR_ERR_INVAL;
    bool vec = at % 16 == 0 && st % 16 == 0 && p.n % 8 == 0;
    const symar_norm_side_t *sides[2] = {&p.after, &p.before};
    for (const symar_norm_side_t *s : sides) {
        if (s->kind < SYMAR_NORM_NONE || s->kind > SYMAR_NORM_LAYER) return SYMAR_ERR_INVAL;
        if (s->kind == SYMAR_NORM_NONE) continue;
        if (!dtype_ok(s->dtype) || !(s->eps >= 0.0f) || s->eps > 3.0e38f || s->plus_one < 0 || s->plus_one > 1) return SYMAR_ERR_INVAL;
        const uintptr_t w = (uintptr_t)s->weight | (uintptr_t)s->bias;
        if (w % (s->dtype == SYMAR_F32 ? 4 : 2)) return SYMAR_ERR_INVAL;
        vec = vec && w % 16 == 0;
    }
    if (!(p.scale >= -3.0e38f && p.scale <= 3.0e38f && p.residual_scale >= -3.0e38f && p.residual_scale <= 3.0e38f)) return SYMAR_ERR_INVAL;
    const int64_t strides[10] = {p.x_ld, p.x_group, p.out_ld, p.out_group, p.gate_ld, p.gate_group,
                                 p.residual_ld, p.residual_group, p.residual_out_ld, p.residual_out_group};
    for (int i = 0; i < 10; ++i) {
        if (strides[i] < 0) return SYMAR_ERR_INVAL;
        if (!(p.gate_step == 0 && (i == 4 || i == 5))) vec = vec && strides[i] % 8 == 0;
    }
    if (p.n > SYMAR_NORM_MAX || (int64_t)p.groups * p.m > 0x7fffffff - kSmall) return SYMAR_ERR_UNSUPPORTED;
    if (p.groups == 0 || p.m == 0 || p.n == 0) return SYMAR_OK;
    if ((p.out == nullptr) != (p.before.kind == SYMAR_NORM_NONE)) return SYMAR_ERR_INVAL;
    if (!p.x || (!p.out && !p.residual_out)) return SYMAR_ERR_INVAL;
    if ((p.out && rows_meet(p.m, p.out_ld, p.groups, p.out_group, p.n)) ||
        (p.residual_out && rows_meet(p.m, p.residual_out_ld, p.groups, p.residual_out_group, p.n)))
        return SYMAR_ERR_INVAL;
    NormArgs a{};
    a.x = p.x;  a.x_ld = p.x_ld;  a.x_group = p.x_group;
    a.residual = p.residual;  a.residual_ld = p.residual_ld;  a.residual_group = p.residual_group;
    a.residual_out = p.residual_out;  a.residual_out_ld = p.residual_out_ld;  a.residual_out_group = p.residual_out_group;
    a.out = p.out;  a.out_ld = p.out_ld;  a.out_group = p.out_group;
    a.gate = p.gate;  a.gate_ld = p.gate_ld;  a.gate_group = p.gate_group;  a.gate_step = p.gate_step;  a.gate_act = p.gate_act;
    Side *to[2] = {&a.after, &a.before};
    for (int i = 0; i < 2; ++i) *to[i] = Side{sides[i]->weight, sides[i]->bias, sides[i]->eps, sides[i]->kind, sides[i]->dtype == SYMAR_F32, sides[i]->plus_one};
    a.scale = p.scale;  a.residual_scale = p.residual_scale;
    a.m = p.m;  a.n = p.n;  a.rows = p.groups * p.m;
    a.x_wide = p.dtype == SYMAR_F32;  a.stream_wide = p.stream_dtype == SYMAR_F32;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    // Few rows: as many threads as there are eights of a row, so that a row is one trip to memory; many: thirty-two elements a thread
    // and fewer threads to meet in a sum.
    const bool few = a.rows <= 296;
    cudaError_t e;
    if (a.n <= 256) e = launch<32, 1>(a, vec, s);
    else if (a.n <= 1024) e = few ? launch<128, 1>(a, vec, s) : launch<32, 4>(a, vec, s);
    else if (a.n <= 4096) e = few ? launch<512, 1>(a, vec, s) : launch<128, 4>(a, vec, s);
    else if (a.n <= 8192) e = few ? launch<1024, 1>(a, vec, s) : launch<256, 4>(a, vec, s);
    else if (a.n <= 16384) e = launch<512, 4>(a, vec, s);
    else e = launch<1024, 4>(a, vec, s);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_norm");
}
