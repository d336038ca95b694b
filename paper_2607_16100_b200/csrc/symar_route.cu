// The experts of every token, and the tokens of every expert (formulas in include/symar.h).
//
// A warp has one token at a time, a lane every thirty-second of its experts, as whole numbers in the order of the floats whose lowest
// bits give way to the expert's place in the lane.  A lane sorts its own; a choice is then the largest of the lanes' first ones.  Which row of the
// lists a choice gets is a counting sort that keeps the tokens' order: every warp has tokens in a row and counts its choices per expert, the counts
// of earlier warps and blocks and of smaller experts are added up, and the warp goes through its tokens once more.  Nothing depends on the order in
// which blocks run.  Few tokens are one block and one launch; more are two launches, the blocks' counts between them in the workspace.
//
// Choices have to be those of binary64, whatever binary32 rounds: where two neighbours in the order found, or the last choice and any expert
// behind it, are nearer than the rounding of their keys and not the same, the token's choices are made again in binary64.
//
// Bound by instructions and, with few tokens, by latency (B200, within a CUDA graph): 16384 tokens x 256 experts, top 8 of sigmoid + bias, take 27.2 us (about
// 20 and 7 for the two launches; 900 instructions of a warp a token, a third of them the eight choices), 64 x 128 9.2 us, one token 3.9 us.  A choice by
// two reductions over unsorted lanes took 1420 instructions (49 us), all doubts in binary64 over all experts 33 us.
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
    int      of_block, of_warp;            // tokens
};
constexpr int kMaxExperts = SYMAR_ROUTE_MAX_EXPERTS, kMaxTop = SYMAR_ROUTE_MAX_TOP;
constexpr int kWarps = 32, kThreads = 32 * kWarps;
constexpr int kBlocks = 148;               // of the two launches: the chip's multiprocessors (the workspace is asked for without a device)
constexpr int kAlone  = 64;                // tokens of one block: one launch costs the host half (64 x 128: 9.2 us alone, 8.1 in two)
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

// The choices in binary64, by score + bias or by logit: lane j gets the j-th expert, -1 for none.
template <int V>
__device__ __noinline__ int choose_exactly(const RouteArgs &a, int64_t row, float top)
{
    const int lane = threadIdx.x & 31;
    double key[V], sum = 0.0;              // NaN: not to be had
#pragma unroll 1
    for (int i = 0; i < V; ++i) {
        const int e = lane + 32 * i;
        const float v = e < a.experts ? logit_of(a, row, e) : -INFINITY;
        key[i] = !a.bias ? (double)v : a.sigmoid ? 1.0 / (1.0 + exp(-(double)v)) : exp((double)v - (double)top);
        if (!(v > -INFINITY)) key[i] = NAN;
        else sum += key[i];
    }
    if (a.bias) {
        sum = warp_sum(sum);
#pragma unroll 1
        for (int i = 0; i < V; ++i)
            if (lane + 32 * i < a.experts) key[i] = (a.sigmoid ? key[i] : key[i] / sum) + (double)a.bias[lane + 32 * i];
    }
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

// The weight of choice `lane` in binary64, divided by the largest chosen score first where only quotients count: those of scores below binary32's (or
// binary64's) range are numbers like others.  sum: a softmax's, of exp(logit - top).
__device__ __noinline__ float weigh_exactly(const RouteArgs &a, int64_t row, int mine, float top, float sum)
{
    const double x = mine >= 0 ? (double)logit_of(a, row, mine) : -INFINITY;
    double from = a.sigmoid ? 0.0 : (double)top;
    if (a.renormalise) {
        from = x;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) from = fmax(from, __shfl_xor_sync(0xffffffffu, from, d));
        if (a.sigmoid) from = fmin(from, 0.0);
    }
    double w = 0.0;                        // a sigmoid is exp(min(x, 0)) / (1 + exp(-|x|))
    if (mine >= 0) w = a.sigmoid ? exp(fmin(x, 0.0) - from) / (1.0 + exp(-fabs(x))) : exp(x - from);
    if (a.renormalise) w /= warp_sum(w);   // (called where there is a choice)
    else if (!a.sigmoid) w /= (double)sum;
    return (float)(w * (double)a.scale);
}

// The D largest of V keys in falling order, by Batcher's odd-even merges of D at a time.
template <int D>
__device__ __forceinline__ void sort_falling(uint32_t *key)
{
#pragma unroll
    for (int p = 1; p < D; p *= 2)
#pragma unroll
        for (int k = p; k >= 1; k /= 2)
#pragma unroll
            for (int j = k % p; j + k < D; j += 2 * k)
#pragma unroll
                for (int i = 0; i < k; ++i)
                    if (i + j + k < D && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
                        const uint32_t x = key[i + j], y = key[i + j + k];
                        key[i + j] = max(x, y), key[i + j + k] = min(x, y);
                    }
}
template <int V, int D>
__device__ __forceinline__ void largest(uint32_t (&key)[V])
{
    sort_falling<D>(key);
#pragma unroll
    for (int from = D; from < V; from += D) {
        sort_falling<D>(key + from);
        // the larger of the i-th largest here and the i-th smallest there are the D largest of both: they rise and fall, or fall and rise
#pragma unroll
        for (int i = 0; i < D; ++i) key[i] = max(key[i], key[from + D - 1 - i]);
#pragma unroll
        for (int k = D / 2; k >= 1; k /= 2)
#pragma unroll
            for (int i = 0; i < D; ++i)
                if ((i & k) == 0) {
                    const uint32_t x = key[i], y = key[i + k];
                    key[i] = max(x, y), key[i + k] = min(x, y);
                }
    }
}
__device__ __forceinline__ float fast_exp(float x)             // 2^-22, and 2^-23 |x|
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * 1.4426950408889634f));
    return y;
}
__device__ __forceinline__ float fast_inverse(float x)         // one unit
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Expert and weight of choice `lane` of token t (-1 and 0: none).  V: experts of a lane.
template <int V>
__device__ __forceinline__ int choose(const RouteArgs &a, int t, float &weight)
{
    constexpr int kDeep = V < 8 ? V : 8;   // experts of a lane that are looked at; a token that wants more of one is done in binary64
    constexpr uint32_t kPlace = V - 1;
    const int lane = threadIdx.x & 31;
    const int64_t row = t * a.ld;
    const int left = a.experts - lane;     // expert lane + 32 i is there where 32 i < left
    float v[V];
    if (a.wide) {
        const float *p = static_cast<const float *>(a.logits) + row + lane;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 32 * i < left ? p[32 * i] : -INFINITY;
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(a.logits) + row + lane;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 32 * i < left ? __uint_as_float((uint32_t)p[32 * i] << 16) : -INFINITY;
    }
    float top = 0.0f, sum = 1.0f;
    if (!a.sigmoid) {
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) most = fmaxf(most, v[i]);                 // (NaN counts as nothing)
        const uint32_t whole = __reduce_max_sync(0xffffffffu, ordered(most));
        top = whole ? unordered(whole) : 0.0f;
        if (a.bias || !a.renormalise) {    // (the weights' quotients need no sum over all)
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) sum += v[i] > -INFINITY ? expf(v[i] - top) : 0.0f;
            sum = warp_sum(sum);
            if (!whole) sum = 1.0f;
        }
    }
    uint32_t key[V];
    if (a.bias) {                          // (fast functions: what they round is in `step`)
        const float by = 1.0f / sum;
        const float *b = a.bias + lane;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float score = a.sigmoid ? fast_inverse(1.0f + fast_exp(-v[i])) : fast_exp(v[i] - top) * by;
            const float sought = 32 * i < left && v[i] > -INFINITY ? score + b[32 * i] : -INFINITY;
            key[i] = ordered(sought + 0.0f);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = ordered(v[i] + 0.0f);            // (-0 is 0)
    }
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = key[i] ? (key[i] & ~kPlace) | (kPlace - i) : 0u;
    largest<V, kDeep>(key);
    int mine = -1, deep = 0;               // choice `lane`; this lane's experts that were chosen
    // the next choice: its expert, and its key for the caller; -1 where nothing is left
    auto pick = [&](uint32_t &most) {
        most = __reduce_max_sync(0xffffffffu, key[0]);
        // (the same place in several lanes: the lowest lane's is the lowest index)
        const int winner = __ffs(__ballot_sync(0xffffffffu, key[0] == most)) - 1;
        const bool won = lane == winner && most != 0;
        deep += won;
#pragma unroll
        for (int i = 0; i + 1 < kDeep; ++i) key[i] = won ? key[i + 1] : key[i];
        key[kDeep - 1] = won ? 0u : key[kDeep - 1];
        return most ? winner + 32 * (int)(kPlace - (most & kPlace)) : -1;
    };
    // Two keys' errors together.  Of a sigmoid s, x its logit: s (1 - s) (2 + 1.2 |x|) units of the exponential, a unit of the sum and one of the quotient,
    // below 4 x 2^-23; of a softmax, p its largest score: p (2 + 1.2 |x|) with p |x| < 0.4 of it, 37 additions of the sum; then a rounding of the sum with
    // the bias, and the bits that the place takes.  Logits themselves are exact but for those bits.
    const float step = !a.bias ? 0.0f : a.sigmoid ? 0x1p-19f : 0x1p-17f / sum;
    auto apart = [&](uint32_t above, uint32_t below) {
        const float was = unordered(above & ~kPlace), is = unordered(below & ~kPlace);
        return was - is > step + (0x1p-21f + V * 0x1p-22f) * fmaxf(fabsf(was), fabsf(is));
    };
    uint32_t found = 0;
    for (int j = 0; j < a.top_k; ++j) {
        uint32_t most;
        const int at = pick(most);
        if (at < 0) break;
        if (lane == j) mine = at, found = most;
    }
    uint32_t under;
    const int behind = pick(under);        // the border has to be looked at
    const int next_at = __shfl_down_sync(0xffffffffu, mine, 1), other = lane == a.top_k - 1 ? behind : next_at;
    const uint32_t next = __shfl_down_sync(0xffffffffu, found, 1);
    const bool close = mine >= 0 && other >= 0 && lane < a.top_k && !apart(found, lane == a.top_k - 1 ? under : next);
    bool doubt = __any_sync(0xffffffffu, close || (kDeep < V && deep == kDeep));
    if (doubt) {
        // None where neighbours are the same, and all that is no further from the last choice than its error, too: a lane's experts that are left.
        auto unlike = [&](int x, int y) { return logit_of(a, row, x) != logit_of(a, row, y) || (a.bias && a.bias[x] != a.bias[y]); };
        bool differs = (close && unlike(mine, other)) || (kDeep < V && deep == kDeep);
        if (__shfl_sync(0xffffffffu, (int)close, a.top_k - 1)) {
            const int last_at = __shfl_sync(0xffffffffu, mine, a.top_k - 1);
            const uint32_t last = __shfl_sync(0xffffffffu, found, a.top_k - 1);
            int as_near = deep;
#pragma unroll
            for (int i = 0; i < kDeep; ++i)
                if (key[i] && !apart(last, key[i])) {
                    ++as_near;
                    differs = differs || unlike(lane + 32 * (int)(kPlace - (key[i] & kPlace)), last_at);
                }
            differs = differs || (kDeep < V && as_near == kDeep);      // (nobody knows what comes behind these)
        }
        doubt = __any_sync(0xffffffffu, differs);
    }
    if (doubt) {
        // Neighbours nearer than their errors: all that may be among the choices, in binary64.
        const uint32_t last = __shfl_sync(0xffffffffu, found, a.top_k - 1);
        int count = __popc(__ballot_sync(0xffffffffu, mine >= 0)), at = behind;
        uint32_t most = under;
        for (; at >= 0 && count < 32 && !apart(last, most); at = pick(most), ++count)
            if (lane == count) mine = at;
        if ((at >= 0 && !apart(last, most)) || (kDeep < V && __any_sync(0xffffffffu, deep == kDeep))) {
            mine = choose_exactly<V>(a, row, top);
        } else {
            double exact = -INFINITY, all = 0.0;
            if (a.bias && !a.sigmoid) {
#pragma unroll 4
                for (int e = lane; e < a.experts; e += 32) {
                    const float l = logit_of(a, row, e);
                    all += l > -INFINITY ? exp((double)l - (double)top) : 0.0;
                }
                all = warp_sum(all);
            }
            if (mine >= 0) {
                exact = (double)logit_of(a, row, mine);
                if (a.bias) exact = a.sigmoid ? 1.0 / (1.0 + exp(-exact)) : exp(exact - (double)top) / all;
                if (a.bias) exact += (double)a.bias[mine];
            }
            int rank = 0, sorted = -1;
            for (int j = 0; j < count; ++j) {
                const double key_j = __shfl_sync(0xffffffffu, exact, j);
                const int at_j = __shfl_sync(0xffffffffu, mine, j);
                rank += key_j > exact || (key_j == exact && at_j < mine);
            }
            for (int j = 0; j < count; ++j) {
                const int rank_j = __shfl_sync(0xffffffffu, rank, j), at_j = __shfl_sync(0xffffffffu, mine, j);
                if (lane == rank_j) sorted = at_j;
            }
            mine = lane < a.top_k ? sorted : -1;
        }
    }
    weight = 0.0f;
    if (mine >= 0) {
        const float logit = logit_of(a, row, mine);
        weight = a.sigmoid ? 1.0f / (1.0f + expf(-logit)) : expf(logit - top);
        if (!a.sigmoid && !a.renormalise) weight /= sum;
    }
    if (__any_sync(0xffffffffu, mine >= 0 && weight < 0x1p-100f)) {      // (its last digits, or all of it, may be below what binary32 holds)
        weight = weigh_exactly(a, row, mine, top, sum);
        return mine;
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
__device__ __forceinline__ Part part(Part of, int i, int size)
{
    const int lo = (int)min((int64_t)of.lo + (int64_t)i * size, (int64_t)of.hi);
    return {lo, (int)min((int64_t)lo + size, (int64_t)of.hi)};
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

// kOnce: one block does it all.  Otherwise a choice's place among those of its block and expert goes to token_row, for place_kernel.
template <int V, bool kOnce>
__global__ void __launch_bounds__(kThreads, 1) choose_kernel(const __grid_constant__ RouteArgs a)
{
    extern __shared__ int32_t count[];     // [kWarps][experts]
    __shared__ int room[33];
    constexpr int kKept = 4;               // tokens whose choices stay in registers
    wait_for_stream();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    int32_t *own = count + warp * a.experts;
    for (int e = lane; e < a.experts; e += 32) own[e] = 0;
    __syncwarp();
    const Part mine = part(part({0, a.tokens}, blockIdx.x, a.of_block), warp, a.of_warp);
    int kept[kKept];
    auto take = [&](int t) {
        float weight;
        const int e = choose<V>(a, t, weight);
        if (lane < a.top_k) {
            const int64_t at = (int64_t)t * a.top_k + lane;
            a.choice[at] = e;
            a.weights[at] = weight;
        }
        if (e >= 0) ++own[e];              // (a token's experts are different ones)
        __syncwarp();
        return e;
    };
#pragma unroll
    for (int u = 0; u < kKept; ++u) kept[u] = -1;
    for (int t = mine.lo; t < mine.hi; ++t) {
        const int e = take(t);
#pragma unroll
        for (int u = 0; u < kKept; ++u) kept[u] = t - mine.lo == u ? e : kept[u];
    }
    __syncthreads();
    // count[w][e]: the choices of expert e by warps before w
    int all = 0;
    if (tid < a.experts) {
#pragma unroll 8
        for (int w = 0; w < kWarps; ++w) {
            const int c = count[w * a.experts + tid];
            count[w * a.experts + tid] = all;
            all += c;
        }
    }
    int *base = count + kWarps * a.experts;
    int total = 0;
    if (kOnce) {
        const int first = exclusive(all, room);
        total = room[32];
        if (tid < a.experts) a.expert_start[tid] = base[tid] = first;
        if (tid == 0) a.expert_start[a.experts] = total;
    } else {
        if (tid < a.experts) a.counts[(int64_t)blockIdx.x * a.experts + tid] = all;
    }
    __syncthreads();
    for (int t = mine.lo; t < mine.hi; ++t) {
        const int64_t at = (int64_t)t * a.top_k + lane;
        int e = -1, row = -1;
        if (t - mine.lo < kKept) {
#pragma unroll
            for (int u = 0; u < kKept; ++u) e = t - mine.lo == u ? kept[u] : e;
        } else if (lane < a.top_k) {
            e = a.choice[at];
        }
        if (e >= 0) {
            row = own[e]++;
            if (kOnce) a.row_token[row += base[e]] = t;
        }
        if (lane < a.top_k) a.token_row[at] = row;
        __syncwarp();
    }
    if (kOnce)
        for (int64_t r = total + tid; r < (int64_t)a.tokens * a.top_k; r += kThreads) a.row_token[r] = -1;
}

__global__ void __launch_bounds__(kThreads, 1) place_kernel(const __grid_constant__ RouteArgs a)
{
    __shared__ int room[33];
    __shared__ int base[kMaxExperts], part_all[kThreads], part_before[kThreads];
    wait_for_stream();
    const int tid = threadIdx.x;
    // several threads an expert: each has every so-manyth block's counts
    int wide = 32;
    while (wide < a.experts) wide *= 2;
    const int e = tid & (wide - 1), shares = kThreads / wide;
    int before = 0, all = 0;               // choices of expert e in earlier blocks, and in all
    if (e < a.experts) {
#pragma unroll 8
        for (int b = tid / wide; b < (int)gridDim.x; b += shares) {
            const int c = a.counts[(int64_t)b * a.experts + e];
            all += c;
            before += b < (int)blockIdx.x ? c : 0;
        }
    }
    part_all[tid] = all, part_before[tid] = before;
    __syncthreads();
    all = before = 0;
    if (tid < a.experts)
        for (int q = 0; q < shares; ++q) all += part_all[tid + q * wide], before += part_before[tid + q * wide];
    const int first = exclusive(all, room);
    if (tid < a.experts) {
        base[tid] = first + before;
        if (blockIdx.x == 0) a.expert_start[tid] = first;
    }
    if (blockIdx.x == 0 && tid == 0) a.expert_start[a.experts] = room[32];
    __syncthreads();
    const Part tokens = part({0, a.tokens}, blockIdx.x, a.of_block);
    const int hi = tokens.hi * a.top_k;    // (below 2^31 with a block's threads more)
    for (int at = tokens.lo * a.top_k + tid; at < hi; at += kThreads) {
        const int expert = a.choice[at];
        if (expert < 0) continue;
        const int row = base[expert] + a.token_row[at];
        a.token_row[at] = row;
        a.row_token[row] = (int)((unsigned)at / (unsigned)a.top_k);
    }
    for (int64_t r = room[32] + (int64_t)blockIdx.x * kThreads + tid; r < (int64_t)a.tokens * a.top_k; r += (int64_t)gridDim.x * kThreads)
        a.row_token[r] = -1;
}

// Tokens of a block: as many for each of its warps.
int tokens_of(int tokens)
{
    if (tokens <= kAlone) return tokens;
    const int each = (int)(((int64_t)tokens + kBlocks * kWarps - 1) / (kBlocks * kWarps));
    return each * kWarps;
}
int blocks_of(int tokens) { return (int)(((int64_t)tokens + tokens_of(tokens) - 1) / tokens_of(tokens)); }

template <int V>
int launch(RouteArgs a, int device, cudaStream_t s)
{
    a.of_block = tokens_of(a.tokens);
    a.of_warp = (a.of_block + kWarps - 1) / kWarps;
    const int shared = (kWarps + 1) * a.experts * 4, blocks = blocks_of(a.tokens);
    static std::atomic<uint64_t> once{0}, many{0};
    const bool alone = blocks == 1;
    auto fn = alone ? choose_kernel<V, true> : choose_kernel<V, false>;
    cudaError_t e = allow_shared((const void *)fn, (kWarps + 1) * V * 32 * 4, device, alone ? once : many);
    if (e == cudaSuccess) e = launch_early(fn, dim3((unsigned)blocks), kThreads, (size_t)shared, s, a);
    if (e == cudaSuccess && !alone) e = launch_early(place_kernel, dim3((unsigned)blocks), kThreads, 0, s, a);
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
