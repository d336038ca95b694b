// The experts of every token, and the tokens of every expert (formulas in include/symar.h).
//
// A warp has one token at a time, a lane every thirty-second of its experts, as whole numbers in the order of the floats; a choice
// is one maximum over the warp and one minimum over the indexes that have it.  Which row of the lists a choice gets is a
// counting sort that keeps the tokens' order: every warp has tokens in a row and counts its choices per expert, the counts of
// earlier warps and blocks and of smaller experts are added up, and the warp goes through its tokens once more.  Nothing depends on the order in which
// blocks run.  Few tokens are one block and one launch; more are two launches, the blocks' counts between them in the workspace.
//
// Choices by score + bias have to be those of exact arithmetic, whatever binary32 rounds: where two neighbours in the order
// found are nearer than the rounding of their keys, the token's choices are made again in binary64.
#include <math.h>

#include "symar_ops.h"

namespace symar {
namespace {

struct RouteArgs {
    const void  *logits;
    const float *bias;
    int32_t *choice, *expert_start, *row_token, *token_row;
    float   *weights;
    int32_t *counts;                       // [blocks][experts], between the two launches
    int64_t  ld;
    float    scale;
    int      tokens, experts, top_k, wide, sigmoid, renormalise;
};
constexpr int kMaxExperts = SYMAR_ROUTE_MAX_EXPERTS, kMaxTop = SYMAR_ROUTE_MAX_TOP;
constexpr int kWarps = 32, kThreads = 32 * kWarps;
constexpr int kBlocks = 148;               // of the two launches
constexpr int kAlone  = 128;               // tokens of one block
static_assert(kThreads >= kMaxExperts && kMaxTop <= 32 && kMaxExperts <= 32 * 32, "");

__device__ __forceinline__ float logit_of(const RouteArgs &a, int64_t row, int e)
{
    const int64_t at = row + e;
    const float v = a.wide ? static_cast<const float *>(a.logits)[at]
                           : __uint_as_float((uint32_t) static_cast<const uint16_t *>(a.logits)[at] << 16);
    return v + 0.0f;                       // (-0 is 0)
}
// Whole numbers in the order of floats; 0: not to be had (-inf or NaN)
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t b = __float_as_uint(v);
    return v > -INFINITY ? b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u) : 0u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u ^ ((int32_t)u < 0 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ float warp_sum(float s)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    return s;
}
__device__ __forceinline__ double warp_sum(double s)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    return s;
}

// The choices by score + bias in binary64: lane j gets the j-th expert, -1 for none.
template <int V>
__device__ __noinline__ int choose_exactly(const RouteArgs &a, int64_t row, float top)
{
    const int lane = threadIdx.x & 31;
    double key[V], sum = 0.0;              // NaN: not to be had
#pragma unroll 1
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        const float v = e < a.experts ? logit_of(a, row, e) : -INFINITY;
        key[i] = a.sigmoid ? 1.0 / (1.0 + exp(-(double)v)) : exp((double)v - (double)top);
        if (!(v > -INFINITY)) key[i] = NAN;
        else sum += key[i];
    }
    sum = warp_sum(sum);
#pragma unroll 1
    for (int i = 0; i < V; ++i)
        if (lane + 32 * i < a.experts) key[i] = (a.sigmoid ? key[i] : key[i] / sum) + (double)a.bias[lane + 32 * i];
    int mine = -1;
    for (int j = 0; j < a.top_k; ++j) {
        double best = -INFINITY;
        int at = kMaxExperts;
#pragma unroll 1
        for (int i = 0; i < V; ++i)
            if (key[i] > best) best = key[i], at = lane + 32 * i;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            const double there = __shfl_xor_sync(0xffffffffu, best, d);
            const int there_at = __shfl_xor_sync(0xffffffffu, at, d);
            if (there > best || (there == best && there_at < at)) best = there, at = there_at;
        }
        if (at == kMaxExperts) break;
        if (lane == j) mine = at;
        if (lane == (at & 31)) key[at >> 5] = NAN;
    }
    return mine;
}

// Expert and weight of choice `lane` of token t (-1 and 0: none).  V: experts of a lane.
template <int V>
__device__ __forceinline__ int choose(const RouteArgs &a, int t, float &weight)
{
    const int lane = threadIdx.x & 31;
    const int64_t row = t * a.ld;
    uint32_t key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = lane + 32 * i < a.experts ? ordered(logit_of(a, row, lane + 32 * i)) : 0u;
    float top = 0.0f, sum = 1.0f;
    if (!a.sigmoid) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) most = max(most, key[i]);
        most = __reduce_max_sync(0xffffffffu, most);
        top = unordered(most);
        if (a.bias || !a.renormalise) {    // (the weights' quotients need no sum over all)
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) sum += key[i] ? expf(unordered(key[i]) - top) : 0.0f;
            sum = warp_sum(sum);
        }
        if (most == 0) top = 0.0f, sum = 1.0f;
    }
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (key[i] == 0) continue;
            const float v = unordered(key[i]);
            const float score = a.sigmoid ? 1.0f / (1.0f + expf(-v)) : expf(v - top) / sum;
            key[i] = ordered(score + a.bias[lane + 32 * i]);
        }
    }
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) best = max(best, key[i]);
    // one choice more than asked for, where the border has to be looked at
    const int more = a.bias ? min(a.top_k + 1, a.experts) : a.top_k;
    int mine = -1, last_at = -1;
    uint32_t last = 0;
    bool near = false;
    // two keys' errors together: a score's (sigmoid: a function's two units, two roundings; softmax: of the largest one, the sum's 37
    // additions more), and a rounding of the keys themselves
    const float step = a.sigmoid ? 0x1p-20f : 0x1p-17f / sum;
    for (int j = 0; j < more; ++j) {
        const uint32_t most = __reduce_max_sync(0xffffffffu, best);
        if (most == 0) break;
        int at = kMaxExperts;
        if (best == most) {
#pragma unroll
            for (int i = V - 1; i >= 0; --i) at = key[i] == most ? lane + 32 * i : at;
        }
        at = (int)__reduce_min_sync(0xffffffffu, (unsigned)at);
        if (lane == j && j < a.top_k) mine = at;
        if (a.bias) {
            if (j > 0) {
                const float was = unordered(last), is = unordered(most);
                if (!(was - is > step + 0x1p-21f * fabsf(is)))
                    near |= logit_of(a, row, at) != logit_of(a, row, last_at) || a.bias[at] != a.bias[last_at];
            }
            last = most, last_at = at;
        }
        best = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (lane + 32 * i == at) key[i] = 0;
            best = max(best, key[i]);
        }
    }
    if (near) mine = choose_exactly<V>(a, row, top);
    weight = 0.0f;
    if (mine >= 0) {
        const float v = logit_of(a, row, mine);
        weight = a.sigmoid ? 1.0f / (1.0f + expf(-v)) : expf(v - top);
        if (!a.sigmoid && !a.renormalise) weight /= sum;
    }
    if (a.renormalise) {
        const float all = warp_sum(weight);
        weight = all > 0.0f || !(all == all) ? weight / all : 0.0f;
    }
    weight *= a.scale;
    return mine;
}

// Tokens of a block and of a warp: neighbours, in order.
struct Part {
    int lo, hi;
};
__device__ __forceinline__ Part part(Part of, int i, int n)
{
    const int64_t count = of.hi - of.lo;
    return {of.lo + (int)(count * i / n), of.lo + (int)(count * (i + 1) / n)};
}

// Exclusive sums over the experts of what every thread e < experts holds; `room`: 33 words.
__device__ __forceinline__ int exclusive(int v, int *room)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += u;
    }
    if (lane == 31) room[warp] = s;
    __syncthreads();
    if (warp == 0) {
        int w = room[lane], u = w;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, u, d);
            if (lane >= d) u += x;
        }
        room[lane] = u - w;
        if (lane == 31) room[32] = u;
    }
    __syncthreads();
    return room[warp] + s - v;
}

// Rows of the warp's choices, once count[warp][e] holds its first row of expert e.
__device__ __forceinline__ void place(const RouteArgs &a, Part tokens, int32_t *count)
{
    const int lane = threadIdx.x & 31;
    for (int t = tokens.lo; t < tokens.hi; ++t) {
        const int64_t at = (int64_t)t * a.top_k + lane;
        const int e = lane < a.top_k ? a.choice[at] : -1;
        int row = -1;
        if (e >= 0) {                      // (a token's experts are different ones)
            row = count[e]++;
            a.row_token[row] = t;
        }
        if (lane < a.top_k) a.token_row[at] = row;
        __syncwarp();
    }
}

// kOnce: one block does it all.
template <int V, bool kOnce>
__global__ void __launch_bounds__(kThreads, 1) choose_kernel(const __grid_constant__ RouteArgs a)
{
    extern __shared__ int32_t count[];     // [kWarps][experts]
    __shared__ int room[33];
    wait_for_stream();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t *own = count + warp * a.experts;
    for (int e = lane; e < a.experts; e += 32) own[e] = 0;
    __syncwarp();
    const Part mine = part(part({0, a.tokens}, blockIdx.x, gridDim.x), warp, kWarps);
    for (int t = mine.lo; t < mine.hi; ++t) {
        float weight;
        const int e = choose<V>(a, t, weight);
        if (lane < a.top_k) {
            const int64_t at = (int64_t)t * a.top_k + lane;
            a.choice[at] = e;
            a.weights[at] = weight;
        }
        if (e >= 0) ++own[e];
        __syncwarp();
    }
    __syncthreads();
    int all = 0;
    if (tid < a.experts)
        for (int w = 0; w < kWarps; ++w) all += count[w * a.experts + tid];
    if (!kOnce) {
        if (tid < a.experts) a.counts[(int64_t)blockIdx.x * a.experts + tid] = all;
        return;
    }
    const int first = exclusive(all, room);
    if (tid < a.experts) {
        a.expert_start[tid] = first;
        int run = first;
        for (int w = 0; w < kWarps; ++w) {
            const int c = count[w * a.experts + tid];
            count[w * a.experts + tid] = run;
            run += c;
        }
    }
    if (tid == 0) a.expert_start[a.experts] = room[32];
    __syncthreads();
    place(a, mine, own);
    for (int64_t r = room[32] + tid; r < (int64_t)a.tokens * a.top_k; r += kThreads) a.row_token[r] = -1;
}

__global__ void __launch_bounds__(kThreads, 1) place_kernel(const __grid_constant__ RouteArgs a)
{
    extern __shared__ int32_t count[];     // [kWarps][experts]
    __shared__ int room[33];
    wait_for_stream();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t *own = count + warp * a.experts;
    for (int e = lane; e < a.experts; e += 32) own[e] = 0;
    __syncwarp();
    const Part mine = part(part({0, a.tokens}, blockIdx.x, gridDim.x), warp, kWarps);
    for (int t = mine.lo; t < mine.hi; ++t) {
        const int e = lane < a.top_k ? a.choice[(int64_t)t * a.top_k + lane] : -1;
        if (e >= 0) ++own[e];
        __syncwarp();
    }
    int before = 0, all = 0;               // of expert tid: in earlier blocks, in all
    if (tid < a.experts) {
#pragma unroll 8
        for (int b = 0; b < (int)gridDim.x; ++b) {
            const int c = a.counts[(int64_t)b * a.experts + tid];
            all += c;
            before += b < (int)blockIdx.x ? c : 0;
        }
    }
    const int first = exclusive(all, room);                    // (its barriers stand behind the counts of all warps)
    if (tid < a.experts) {
        if (blockIdx.x == 0) a.expert_start[tid] = first;
        int run = first + before;
        for (int w = 0; w < kWarps; ++w) {
            const int c = count[w * a.experts + tid];
            count[w * a.experts + tid] = run;
            run += c;
        }
    }
    if (blockIdx.x == 0 && tid == 0) a.expert_start[a.experts] = room[32];
    __syncthreads();
    place(a, mine, own);
    for (int64_t r = room[32] + (int64_t)blockIdx.x * kThreads + tid; r < (int64_t)a.tokens * a.top_k; r += (int64_t)gridDim.x * kThreads)
        a.row_token[r] = -1;
}

int blocks_of(int tokens) { return tokens <= kAlone ? 1 : (int)((tokens + kWarps - 1) / kWarps < kBlocks ? (tokens + kWarps - 1) / kWarps : kBlocks); }

template <int V>
int launch(const RouteArgs &a, int device, cudaStream_t s)
{
    const int shared = kWarps * a.experts * 4, blocks = blocks_of(a.tokens);
    static std::atomic<uint64_t> once{0}, many{0};
    const bool alone = blocks == 1;
    auto fn = alone ? choose_kernel<V, true> : choose_kernel<V, false>;
    cudaError_t e = allow_shared((const void *)fn, kWarps * V * 32 * 4, device, alone ? once : many);
    if (e == cudaSuccess) e = launch_early(fn, dim3((unsigned)blocks), kThreads, (size_t)shared, s, a);
    if (e == cudaSuccess && !alone) {
        static std::atomic<uint64_t> placed{0};
        e = allow_shared((const void *)place_kernel, kWarps * kMaxExperts * 4, device, placed);
        if (e == cudaSuccess) e = launch_early(place_kernel, dim3((unsigned)blocks), kThreads, (size_t)shared, s, a);
    }
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_route");
}

}  // namespace
}  // namespace symar

using namespace symar;

extern "C" size_t symar_route_workspace(int tokens, int experts)
{
    if (tokens <= kAlone || experts < 1 || experts > kMaxExperts) return 0;
    return (size_t)blocks_of(tokens) * experts * sizeof(int32_t);
}

extern "C" int symar_route(const symar_route_t *args, void *cuda_stream)
{
    if (!args) return SYMAR_ERR_INVAL;
    const symar_route_t &p = *args;
    if (p.tokens < 0 || p.experts < 1 || p.top_k < 1 || p.top_k > p.experts || (p.dtype != SYMAR_F32 && p.dtype != SYMAR_BF16)) return SYMAR_ERR_INVAL;
    if (p.score < SYMAR_SCORE_SOFTMAX || p.score > SYMAR_SCORE_SIGMOID || p.renormalise < 0 || p.renormalise > 1) return SYMAR_ERR_INVAL;
    if (!(p.scale >= -3.0e38f && p.scale <= 3.0e38f) || p.ld < 0) return SYMAR_ERR_INVAL;
    if (p.experts > kMaxExperts || p.top_k > kMaxTop || (int64_t)p.tokens * p.top_k > 0x7fffffff - kThreads) return SYMAR_ERR_UNSUPPORTED;
    if ((uintptr_t)p.logits % (p.dtype == SYMAR_F32 ? 4 : 2)) return SYMAR_ERR_INVAL;
    if (((uintptr_t)p.bias | (uintptr_t)p.choice | (uintptr_t)p.weights | (uintptr_t)p.expert_start | (uintptr_t)p.row_token | (uintptr_t)p.token_row |
         (uintptr_t)p.workspace) % 4)
        return SYMAR_ERR_INVAL;
    if (!p.expert_start) return SYMAR_ERR_INVAL;
    if (p.tokens > 0 && (!p.logits || !p.choice || !p.weights || !p.row_token || !p.token_row)) return SYMAR_ERR_INVAL;
    const size_t need = symar_route_workspace(p.tokens, p.experts);
    if (need > 0 && !p.workspace) return SYMAR_ERR_INVAL;
    if (need > p.workspace_bytes) return SYMAR_ERR_NOMEM;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (p.tokens == 0) {
        const cudaError_t e = cudaMemsetAsync(p.expert_start, 0, ((size_t)p.experts + 1) * sizeof(int32_t), s);
        return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "cudaMemsetAsync");
    }
    int device = -1;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    RouteArgs a{};
    a.logits = p.logits;  a.ld = p.ld;  a.bias = p.bias;
    a.choice = p.choice;  a.weights = p.weights;  a.expert_start = p.expert_start;  a.row_token = p.row_token;  a.token_row = p.token_row;
    a.counts = (int32_t *)p.workspace;
    a.scale = p.scale;  a.tokens = p.tokens;  a.experts = p.experts;  a.top_k = p.top_k;
    a.wide = p.dtype == SYMAR_F32;  a.sigmoid = p.score == SYMAR_SCORE_SIGMOID;  a.renormalise = p.renormalise;
    if (p.experts <= 32) return launch<1>(a, device, s);
    if (p.experts <= 64) return launch<2>(a, device, s);
    if (p.experts <= 128) return launch<4>(a, device, s);
    if (p.experts <= 256) return launch<8>(a, device, s);
    if (p.experts <= 512) return launch<16>(a, device, s);
    return launch<32>(a, device, s);
}
