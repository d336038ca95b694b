// out_g = act(x_g w_g^T + bias_g) + residual_g, one matrix per rank (formulas in include/symar.h), on the fifth
// generation's tensor cores.
//
// The weights are the 128 rows of every matrix instruction and the tokens its columns, 16 to 256 of them: with one
// token or a few, as in a decode step, every instruction still uses all 128 lanes and the kernel is a stream of the
// weights; with many it is an ordinary product of 128 x 256 tiles.  A block is one producer (the copy engine
// fills a ring of 64-wide slices of both operands), one thread that issues the products, and eight warps that take
// finished accumulators out of tensor memory, where the next tile is already being summed in the other half.
// Where tiles are fewer than half the multiprocessors, clusters of two to eight blocks share a tile's k and add their parts up over
// distributed shared memory in rank order (clusters of three left multiprocessors without one: 52 us instead of 37 for the odd case below).
//
// Bound and measured (B200, times within a CUDA graph).  Few tokens: the weights' bytes; 8 x 4 x 8192 x 1024 takes 25.3 us for 135 MB,
// 5.3 TB/s (0.81 of the measured copy rate; the ring of ten stages holds 200 KB a multiprocessor in flight, the rest is
// the start and the cluster's sum); 1 x 1024 x 1024 4.9 us, launch and latency.  Many: the tensor cores; 4096 x 8192 x 8192 takes 395 us,
// 1390 TFLOP/s (0.85 of the measured 1640; a library product 354), with bias, tanh-GELU and residual 450 us: the
// epilogue's 33 M values are 55 us of work for eight warps and only partly hidden.  float32 results 610-680 us: their sums leave
// the tensor cores every 128 products (see kChunk).  Rows on no 16-byte boundary: 2 x 333 x 1003 x 2049 takes 35.4 us where k = 2048 takes 13.9; the
// eight loading warps issue most of a slice's 7600 instructions, to shift and join its 2048 pieces (these kernels spill 24 to 120 bytes at 96 registers; the
// others nothing).
#include <type_traits>

#include "symar_ops.h"
#include "symar_rows.h"
#include "symar_tc.cuh"

namespace symar {
namespace {

struct LinearArgs {
    const __nv_bfloat16 *x, *w, *bias;
    const void *residual;
    void       *out;
    int64_t x_ld, x_group, w_ld, w_group, bias_group, residual_ld, residual_group, out_ld, out_group;
    int     m, n, k, act, root;
    int     n_tiles, m_tiles, tiles;       // of 128 channels, of NT tokens, of all groups
    int     split;                         // blocks of a cluster that share a tile's k
    int     vec_out, vec_res;              // four results at a time: rows on boundaries of four elements
    unsigned *status;
};

constexpr int kRows = 128;                 // channels of a tile; a stage has kSlice of k: 128 bytes, one swizzled row
constexpr int kMaxSplit = 8;
constexpr int kMostRows = 0x7fffffff - 511;          // of m, n and k: the tile or slice that holds the last one ends below 2^31

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 peer_load4(uint32_t addr, int rank)
{
    uint32_t there;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(there) : "memory");
    return v;
}
__device__ __forceinline__ void results_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

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

// What follows the sums: four neighbouring channels of one token, from `n` on (fewer at the row's end).
template <typename O> struct Four;
template <> struct Four<float> { float4 v; };
template <> struct Four<__nv_bfloat16> { uint2 v; };
struct Channels {
    float bias[4];
    int   n, count, add;             // add: this group takes bias and residual
};
__device__ __forceinline__ Channels channels_of(const LinearArgs &a, int g, int n)
{
    Channels c;
    c.n     = n;
    c.count = max(0, min(4, a.n - n));
    c.add   = a.root < 0 || a.root == g;
#pragma unroll
    for (int i = 0; i < 4; ++i) c.bias[i] = c.add && a.bias && i < c.count ? __bfloat162float(a.bias[g * a.bias_group + n + i]) : 0.0f;
    return c;
}
template <typename O>
__device__ __forceinline__ Four<O> residual4(const LinearArgs &a, const Channels &c, int g, int token)
{
    Four<O> r{};
    if (c.add && a.residual && c.count > 0) {
        const O *p = static_cast<const O *>(a.residual) + g * a.residual_group + token * a.residual_ld + c.n;
        if (a.vec_res && c.count == 4) {
            r = *reinterpret_cast<const Four<O> *>(p);
        } else {
            O h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = i < c.count ? p[i] : O(0.0f);
            r = *reinterpret_cast<const Four<O> *>(h);
        }
    }
    return r;
}
__device__ __forceinline__ void before_residual(const LinearArgs &a, const Channels &c, float4 &sum)
{
    float y[4] = {sum.x + c.bias[0], sum.y + c.bias[1], sum.z + c.bias[2], sum.w + c.bias[3]};
    activate4(y, a.act);
    sum = make_float4(y[0], y[1], y[2], y[3]);
}
template <typename O>
__device__ __forceinline__ void store4(const LinearArgs &a, const Channels &c, int g, int token, float4 v, const Four<O> &res)
{
    if (c.count == 0) return;
    float y[4] = {v.x, v.y, v.z, v.w};
    if (c.add && a.residual) {
        float r[4];
        load4(reinterpret_cast<const O *>(&res), r);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += r[i];
    }
    O *p = static_cast<O *>(a.out) + g * a.out_group + token * a.out_ld + c.n;
    if (a.vec_out && c.count == 4) {
        put4(p, y);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < c.count) put(p + i, y[i]);
    }
}
// `count` (at most 8 N) tokens from `token` on whose sums lie in shared memory, one in eight of them this warp's: bias and activation
// in a loop that is there once, then residuals, which were asked for before, and stores.
template <typename O, int N>
__device__ __forceinline__ void residuals_of(const LinearArgs &a, const Channels &c, int g, int token, int count, int w, Four<O> (&res)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (w + 8 * i < count) res[i] = residual4<O>(a, c, g, token + w + 8 * i);
}
template <typename O, int N>
__device__ __forceinline__ void finish(const LinearArgs &a, const Channels &c, int g, int token, int count, int w, float *sums, const Four<O> (&res)[N])
{
    float4 *mine = reinterpret_cast<float4 *>(sums);          // this lane's four channels of the first token
    if (a.act != SYMAR_ACT_NONE) {
#pragma unroll 2
        for (int t = w; t < count; t += 8) before_residual(a, c, mine[t * (kRows / 4)]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int t = w + 8 * i;
        if (t < count) {
            float4 v = mine[t * (kRows / 4)];
            if (a.act == SYMAR_ACT_NONE) v = make_float4(v.x + c.bias[0], v.y + c.bias[1], v.z + c.bias[2], v.w + c.bias[3]);
            store4<O>(a, c, g, token + t, v, res[i]);
        }
    }
}

// ---- rows on no 16-byte boundary ----
// Eight neighbouring lanes hold the eight aligned 16-byte pieces that a slice of a row begins in; the slice's own eight
// pieces start `shift` bytes into them.  A lane takes the missing end of its piece from its neighbour, the eighth from the
// first lane's piece of the next slice, which is on its way by then; so every piece is loaded once.
__device__ __noinline__ uint4 edge_piece(uintptr_t at, Span s)
{
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (at + 2 * i >= s.lo && at + 2 * i + 2 <= s.hi) w[i >> 1] |= (uint32_t)*reinterpret_cast<const uint16_t *>(at + 2 * i) << ((i & 1) * 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// (predicated, not a branch: the loads of all rows go out one after the other)
__device__ __forceinline__ uint4 load_if(uintptr_t at, bool on)
{
    uint4 v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                 "@p ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(at), "r"((int)on));
    return v;
}
// Piece c of a slice of each of N rows (of the first `split` of operand s0, the others of s1) where the row exists and the piece holds
// some of its k elements; pieces that lie in the operand in part are put together element by element.
template <int N>
__device__ __forceinline__ void pieces(uint4 (&v)[N], const uintptr_t (&at)[N], const int (&kind)[N], int k, int slice, int c, int split, Span s0, Span s1)
{
    const bool on = piece_wanted(k, slice, c);
    const int64_t byte = (int64_t)slice * 128 + c * 16;
    bool rest = false;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const bool want = on && (kind[j] & 16), whole = piece_whole(at[j] + byte, kind[j], j < split ? s0 : s1);
        v[j] = load_if(at[j] + byte, want && whole);
        rest |= want && !whole;
    }
    if (rest) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (on && (kind[j] & 16) && !piece_whole(at[j] + byte, kind[j], j < split ? s0 : s1)) v[j] = edge_piece(at[j] + byte, j < split ? s0 : s1);
    }
}
__device__ __forceinline__ uint4 joined(const uint4 &u, const uint4 &next, int shift, int c, int lane)
{
    const int from = c < 7 ? lane + 1 : lane - 7;
    uint32_t w[8] = {u.x, u.y, u.z, u.w, 0, 0, 0, 0};
    w[4] = __shfl_sync(0xffffffffu, c == 0 ? next.x : u.x, from);
    w[5] = __shfl_sync(0xffffffffu, c == 0 ? next.y : u.y, from);
    w[6] = __shfl_sync(0xffffffffu, c == 0 ? next.z : u.z, from);
    w[7] = __shfl_sync(0xffffffffu, c == 0 ? next.w : u.w, from);
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = shift & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = shift & 4 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (shift & 2) * 8);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// zeros from element `count` on
__device__ __forceinline__ uint4 cut(uint4 v, int count)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = count >= 2 * i + 2 ? w[i] : (count == 2 * i + 1 ? w[i] & 0xffffu : 0u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int NT, bool kWide, bool kTma>
struct Shape {
    static constexpr int kThreads = kTma ? 384 : 640;             // without the copy engine eight more warps load
    static constexpr int kA = kRows * kSlice * 2, kB = NT * kSlice * 2, kStage = kA + kB;
    // float32 results leave the registers all at once, bf16 results 32 tokens at a time in two buffers
    static constexpr int kStep  = NT < 32 ? NT : 32;
    static constexpr int kHold  = (kWide ? NT : 2 * kStep) * kRows * 4;
    static constexpr int kStages = (224 * 1024 - kHold) / kStage < 10 ? (224 * 1024 - kHold) / kStage : 10;
    static constexpr int kBytes = kStages * kStage + kHold + 1024;      // (the ring starts on a 1 KiB boundary)
    static constexpr int kCols  = 2 * NT < 32 ? 32 : 2 * NT;      // two accumulators
};
// Slices that a float32 result sums in the tensor cores at a time, whose additions truncate.  Error of the result (2-norm, of its own) at k = 1024, 8192,
// 32768, and time of 4096 x 8192 x 8192: two slices 1.3, 1.5, 1.9 x 10^-7, 610 us; four 2.3, 2.4, 2.6, 538; eight 2.3, 4.8, 4.8, 504; all of k 2.3, 21, 91, 480.
// A plain float32 product: 2.5, 9.5, 23.  (Partial sums of ranks are added up further; two is the nearest to one rounding, 0.3.)
constexpr int kChunk = 2;

// kWide: float32 results (and the sums of 128 products added up in registers)
template <int NT, bool kWide, bool kTma>
__global__ void __launch_bounds__(Shape<NT, kWide, kTma>::kThreads, 1)
linear_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const LinearArgs a)
{
    using S = Shape<NT, kWide, kTma>;
    using O = typename std::conditional<kWide, float, __nv_bfloat16>::type;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 4];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    unsigned char *ring = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    float *hold = reinterpret_cast<float *>(ring + S::kStages * S::kStage);
    const uint32_t ring_addr = smem_addr(ring);
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            bar_init(full + 8 * i, kTma ? 1 : 256);
            bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(acc_full + 8 * i, 1);
            bar_init(acc_empty + 8 * i, 256);
        }
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(S::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = tmem_at;

    wait_for_stream();
    // This block's slices of every one of its tiles: all of k, or its part where a cluster shares the tile.
    const int slices = (a.k + kSlice - 1) / kSlice, rank = a.split > 1 ? (int)blockIdx.x % a.split : 0;
    const int k_lo = (int)((int64_t)slices * rank / a.split), k_hi = (int)((int64_t)slices * (rank + 1) / a.split);
    const int first = (int)blockIdx.x / a.split, step = (int)gridDim.x / a.split;
    // up to sixteen tiles of tokens run through a column of weights before the next: at one time few weights and all
    // of their tokens are read, from L2 after the first
    auto place = [&](int tile, int &g, int &m0, int &n0) {
        const int per = a.n_tiles * a.m_tiles;
        g = tile / per;
        int i = tile - g * per;
        const int band = 16 * a.n_tiles, b = i / band, wide = min(16, a.m_tiles - 16 * b);
        i -= b * band;
        m0 = (16 * b + i % wide) * NT;
        n0 = i / wide * kRows;
    };

    if (kTma && warp == 0 && elected()) {
        // ---- producer: one thread ----
        int st = 0, round = 0;
        for (int tile = first; tile < a.tiles; tile += step) {
            int g, m0, n0;
            place(tile, g, m0, n0);
            for (int ks = k_lo; ks < k_hi; ++ks) {
                if (round > 0 && !bar_wait(empty + 8 * st, (round - 1) & 1, &failed)) goto done;
                const uint32_t at = ring_addr + st * S::kStage, bar = full + 8 * st;
                bar_expect(bar, S::kStage);
                tma_load(at, &wmap, ks * kSlice, n0, a.w_group ? g : 0, bar);
                tma_load(at + S::kA, &xmap, ks * kSlice, m0, a.x_group ? g : 0, bar);
                if (++st == S::kStages) st = 0, ++round;
            }
        }
    } else if (!kTma && warp >= 12) {
        // ---- producer: eight warps; a thread has one piece of every thirty-second row ----
        constexpr int kOf = kTma ? 1 : 4 + (NT + 31) / 32;
        int st = 0, round = 0;
        const int c = tid & 7, r = (tid - 384) >> 3;
        for (int tile = first; tile < a.tiles && k_lo < k_hi; tile += step) {
            int g, m0, n0;
            place(tile, g, m0, n0);
            const uintptr_t w = (uintptr_t)(a.w + g * a.w_group), x = (uintptr_t)(a.x + g * a.x_group);
            const Span ws{w, w + ((int64_t)(a.n - 1) * a.w_ld + a.k) * 2}, xs{x, x + ((int64_t)(a.m - 1) * a.x_ld + a.k) * 2};
            const uintptr_t w_row = w + (int64_t)(n0 + r) * a.w_ld * 2, x_row = x + (int64_t)(m0 + r) * a.x_ld * 2;
            uintptr_t at[kOf];                         // the aligned piece that the row begins in
            int kind[kOf];
#pragma unroll
            for (int j = 0; j < kOf; ++j) {
                const uintptr_t row = j < 4 ? w_row + j * 64 * a.w_ld : x_row + (j - 4) * 64 * a.x_ld;
                const int i = j < 4 ? n0 + r + 32 * j : m0 + r + 32 * (j - 4), rows = j < 4 ? a.n : a.m;
                at[j]   = row & ~(uintptr_t)15;
                kind[j] = row_kind(row, i < rows && (j < 4 || r + 32 * (j - 4) < NT), a.k, j < 4 ? ws : xs);
            }
            uint4 u[kOf], next[kOf];
            pieces<kOf>(u, at, kind, a.k, k_lo, c, 4, ws, xs);
            pieces<kOf>(next, at, kind, a.k, k_lo + 1, c, 4, ws, xs);
#pragma unroll 2            // (the pieces on their way change places with those in hand without a copy, which would wait for them)
            for (int ks = k_lo; ks < k_hi; ++ks) {
                const int left = a.k - ks * kSlice - c * 8;
                if (round > 0 && !warp_wait(empty + 8 * st, (round - 1) & 1, &failed)) goto done;
                unsigned char *dst = ring + st * S::kStage;
#pragma unroll
                for (int j = 0; j < kOf; ++j) {
                    uint4 v = joined(u[j], next[j], kind[j], c, lane);
                    if (left < 8) v = cut(v, left);
                    const int to = j < 4 ? r + 32 * j : r + 32 * (j - 4);
                    if (j < 4 || to < NT) *reinterpret_cast<uint4 *>(dst + (j < 4 ? 0 : S::kA) + to * 128 + ((c ^ (to & 7)) << 4)) = v;
                    u[j] = next[j];
                }
                // asked for a whole slice before they are joined (of the block's last slice's neighbour the slice after has no use)
                pieces<kOf>(next, at, kind, a.k, ks + 1 < k_hi ? ks + 2 : slices + 1, c, 4, ws, xs);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                bar_arrive(full + 8 * st);
                if (++st == S::kStages) st = 0, ++round;
            }
        }
    } else if (warp == 1 && elected()) {
        // ---- products: one thread ----
        constexpr uint32_t kHow = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NT / 8) << 17) | ((uint32_t)(kRows / 16) << 24);
        int st = 0, round = 0;
        uint32_t turn = 0;                              // accumulators filled so far
        for (int tile = first; tile < a.tiles; tile += step) {
            for (int ks = k_lo; ks < k_hi;) {
                const int to = kWide ? min(ks + kChunk, k_hi) : k_hi;
                const uint32_t buf = turn & 1, acc = tmem + buf * NT;
                if (turn >= 2 && !bar_wait(acc_empty + 8 * buf, ((turn >> 1) - 1) & 1, &failed)) goto done;
                tc_after();
                for (uint32_t add = 0; ks < to; ++ks, add = 1) {
                    if (!bar_wait(full + 8 * st, round & 1, &failed)) goto done;
                    tc_after();
                    const uint64_t w = operand(ring_addr + st * S::kStage), x = operand(ring_addr + st * S::kStage + S::kA);
                    product(acc, w, x, kHow, add);
#pragma unroll
                    for (int i = 1; i < kSlice / 16; ++i) product(acc, w + 2 * i, x + 2 * i, kHow, 1);
                    commit(empty + 8 * st);
                    if (++st == S::kStages) st = 0, ++round;
                }
                commit(acc_full + 8 * buf);
                ++turn;
            }
        }
    } else if (warp >= 4 && warp < 12) {
        // ---- results: out of tensor memory a thread holds one channel of many tokens; by way of shared memory it gets four
        // channels of one token, which are neighbours in `out` (and the code of an activation is there once)
        const int quarter = warp & 3, side = (warp - 4) >> 2, ew = warp - 4, ch = quarter * 32 + lane;   // a quarter's channels: two warps, half of the tokens each
        const uint32_t lanes = (uint32_t)quarter << 21;
        const bool parts = k_hi > k_lo;
        float *part = reinterpret_cast<float *>(ring);               // [token][channel] of a shared tile: the ring is not in use any more
        uint32_t turn = 0;
        for (int tile = first; tile < a.tiles; tile += step) {
            int g, m0, n0;
            place(tile, g, m0, n0);
            const int tokens = min(NT, a.m - m0);
            if (kWide) {
                constexpr int kOwn = kWide ? (NT < 32 ? 16 : NT / 2) : 1;     // (of 16 tokens one half of the warps holds all)
                const int col = NT < 32 ? 0 : side * kOwn;
                float sum[kOwn];
#pragma unroll
                for (int i = 0; i < kOwn; ++i) sum[i] = 0.0f;
                for (int ks = k_lo; ks < k_hi; ks += kChunk, ++turn) {
                    const uint32_t buf = turn & 1;
                    (void)warp_wait(acc_full + 8 * buf, (turn >> 1) & 1, &failed);     // (given up: on with what is there, the barriers count all)
                    tc_after();
#pragma unroll
                    for (int c0 = 0; c0 < kOwn; c0 += 16) {
                        float v[16];
                        acc_load16(tmem + lanes + buf * NT + col + c0, v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[kWide ? c0 + i : 0] += v[i];
                    }
                    tc_before();
                    bar_arrive(acc_empty + 8 * buf);
                }
                float *to = a.split > 1 ? part : hold;
                if (NT >= 32 || side == 0) {
#pragma unroll
                    for (int i = 0; i < kOwn; ++i) to[(col + i) * kRows + ch] = sum[i];
                }
                if (a.split == 1) {
                    results_sync();
                    const Channels c = channels_of(a, g, n0 + 4 * lane);
                    Four<O> res[4];
#pragma unroll 1
                    for (int t0 = 0; t0 < tokens; t0 += 32) {
                        const int count = min(32, tokens - t0);
                        residuals_of<O>(a, c, g, m0 + t0, count, ew, res);
                        finish<O>(a, c, g, m0 + t0, count, ew, hold + t0 * kRows + 4 * lane, res);
                    }
                    results_sync();
                }
            } else {
                const uint32_t buf = turn & 1;
                const Channels c = channels_of(a, g, n0 + 4 * lane);
                Four<O> res[S::kStep / 8];
                if (a.split == 1) residuals_of<O>(a, c, g, m0, min(S::kStep, tokens), ew, res);
                if (parts) {
                    (void)warp_wait(acc_full + 8 * buf, (turn >> 1) & 1, &failed);     // (given up: on with what is there, the barriers count all)
                    tc_after();
                }
#pragma unroll 1
                for (int c0 = 0; c0 < tokens; c0 += S::kStep) {
                    float *to = a.split > 1 ? part + c0 * kRows : hold + ((c0 / S::kStep) & 1) * S::kStep * kRows;
                    const int col = S::kStep < 32 ? 0 : side * 16;              // a half of the warps takes sixteen of the tokens
                    float v[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = 0.0f;
                    if (parts) acc_load16(tmem + lanes + buf * NT + c0 + col, v);
                    if (c0 + S::kStep >= tokens && parts) {          // the accumulator is free for the tile after the next
                        tc_before();
                        bar_arrive(acc_empty + 8 * buf);
                    }
                    if (S::kStep == 32 || side == 0) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) to[(col + i) * kRows + ch] = v[i];
                    }
                    if (a.split == 1) {
                        results_sync();      // one barrier a step: the other buffer was read before its last writer came here
                        const int count = min(S::kStep, tokens - c0);
                        finish<O>(a, c, g, m0 + c0, count, ew, to + 4 * lane, res);
                        residuals_of<O>(a, c, g, m0 + c0 + S::kStep, min(S::kStep, tokens - c0 - S::kStep), ew, res);
                    }
                }
                // a next tile's first step may be this tile's last buffer
                if (a.split == 1) results_sync();
                if (parts) ++turn;
            }
        }
    }
done:
    __syncwarp();
    if (a.split > 1) {
        // ---- the cluster's parts of the tile: block r sums tokens r, r + split, ... over the blocks in order ----
        cluster_sync();
        int g, m0, n0;
        place(first, g, m0, n0);
        const int tokens = min(NT, a.m - m0);
        const Channels c = channels_of(a, g, n0 + 4 * lane);
#pragma unroll 2
        for (int t = rank + a.split * warp; t < tokens; t += a.split * (S::kThreads / 32)) {
            const Four<O> res = residual4<O>(a, c, g, m0 + t);
            const uint32_t at = ring_addr + (t * kRows + 4 * lane) * 4;
            float4 v[kMaxSplit], y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int r = 0; r < kMaxSplit; ++r) v[r] = r < a.split ? peer_load4(at, r) : y;
#pragma unroll
            for (int r = 0; r < kMaxSplit; ++r) {
                y.x += v[r].x; y.y += v[r].y; y.z += v[r].z; y.w += v[r].w;
            }
            before_residual(a, c, y);
            store4<O>(a, c, g, m0 + t, y, res);
        }
        cluster_sync();                                   // no block leaves while its part may be read
    }
    tc_before();
    __syncthreads();
    if (failed) {
        // copies and products may still be in flight: give them time to end before the memory is let go
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        if (tid == 0 && a.status) atomicCAS(a.status, 0u, (unsigned)SYMAR_ERR_TIMEOUT);
        __syncthreads();
    }
    tc_after();
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kCols) : "memory");
}

// ---- host ---------------------------------------------------------------------------------
using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
EncodeFn encoder()
{
    static EncodeFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

// Rows that the copy engine can read: on 16-byte boundaries, rows that do not overlap.
bool engine_rows(const void *p, int64_t ld, int64_t group, int rows, int groups, int k)
{
    return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && group % 8 == 0 && group >= 0 && (rows == 1 || ld >= k) && ld < (1ll << 38) &&
           group < (1ll << 38) && k > 0 && (groups == 1 || group == 0 || group >= 8);
}
bool encode(CUtensorMap *map, const void *p, int64_t ld, int64_t group, int rows, int groups, int k, int box)
{
    const bool shared = group == 0 || groups == 1;
    if (ld < 8) ld = (k + 7) / 8 * 8;                    // one row: the stride is never used
    const cuuint64_t dims[3]    = {(cuuint64_t)k, (cuuint64_t)rows, (cuuint64_t)(shared ? 1 : groups)};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(shared ? ld : group) * 2};
    const cuuint32_t boxes[3] = {kSlice, (cuuint32_t)box, 1}, ones[3] = {1, 1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dims, strides, boxes, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Device {
    int sms = 0, id = -1;
};
int device_info(Device *d)
{
    static std::atomic<int> known[64];                   // multiprocessors; 0: not asked yet (by any thread)
    cudaError_t e = cudaGetDevice(&d->id);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    const bool slot = d->id >= 0 && d->id < 64;
    if (slot && (d->sms = known[d->id].load(std::memory_order_relaxed)) > 0) return SYMAR_OK;
    e = cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, d->id);
    if (e != cudaSuccess) return cuda_fail(e, "cudaDeviceGetAttribute");
    if (slot) known[d->id].store(d->sms, std::memory_order_relaxed);
    return SYMAR_OK;
}

template <int NT, bool kWide, bool kTma>
int launch(LinearArgs a, const CUtensorMap &wmap, const CUtensorMap &xmap, int groups, const Device &d, cudaStream_t stream)
{
    using S = Shape<NT, kWide, kTma>;
    auto fn = linear_kernel<NT, kWide, kTma>;
    a.n_tiles = (a.n + kRows - 1) / kRows;
    a.m_tiles = (a.m + NT - 1) / NT;
    const int64_t tiles = (int64_t)a.n_tiles * a.m_tiles * groups;
    if (tiles > 0x3fffffff) return SYMAR_ERR_UNSUPPORTED;
    a.tiles = (int)tiles;
    const int slices = (a.k + kSlice - 1) / kSlice;
    a.split = 1;
    while (a.split < kMaxSplit && tiles * a.split * 2 <= d.sms && slices >= a.split * 4 && NT * kRows * 4 <= S::kStages * S::kStage) a.split *= 2;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_shared((const void *)fn, S::kBytes, d.id, allowed);
    if (e != cudaSuccess) return cuda_fail(e, "symar_linear");
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    cfg.gridDim  = dim3((unsigned)(a.split > 1 ? tiles * a.split : (tiles < d.sms ? tiles : d.sms)));
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kBytes;
    cfg.stream   = stream;
    cfg.attrs    = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // (see wait_for_stream)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (a.split > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)a.split;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    e = cudaLaunchKernelEx(&cfg, fn, wmap, xmap, a);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_linear");
}

template <int NT>
int launch_as(const LinearArgs &a, int groups, const Device &d, bool wide, bool engine, cudaStream_t s)
{
    constexpr bool kBoth = NT <= 128;              // float32 results: the sums of a wider tile do not fit a thread's registers
    constexpr int  kByHand = NT > 128 ? 128 : NT;    // nor do the pieces of its rows where the block's threads load them
    CUtensorMap wmap{}, xmap{};
    engine = engine && encoder() && encode(&wmap, a.w, a.w_ld, a.w_group, a.n, groups, a.k, kRows) &&
             encode(&xmap, a.x, a.x_ld, a.x_group, a.m, groups, a.k, NT);
    if (wide && kBoth) return engine ? launch<NT, kBoth, true>(a, wmap, xmap, groups, d, s) : launch<kByHand, kBoth, false>(a, wmap, xmap, groups, d, s);
    return engine ? launch<NT, false, true>(a, wmap, xmap, groups, d, s) : launch<kByHand, false, false>(a, wmap, xmap, groups, d, s);
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
    if (p.m > kMostRows || p.n > kMostRows || p.k > kMostRows) return SYMAR_ERR_UNSUPPORTED;
    if ((uintptr_t)p.status % 4) return SYMAR_ERR_INVAL;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    auto clear = [&] {
        const cudaError_t e = p.status ? cudaMemsetAsync(p.status, 0, sizeof(unsigned), s) : cudaSuccess;
        return e == cudaSuccess ? (int)SYMAR_OK : cuda_fail(e, "cudaMemsetAsync");
    };
    if (p.groups == 0 || p.m == 0 || p.n == 0) return clear();
    const uintptr_t width = p.out_dtype == SYMAR_F32 ? 4 : 2;
    if (!p.out || (p.k > 0 && (!p.x || !p.w))) return SYMAR_ERR_INVAL;
    if (((uintptr_t)p.x | (uintptr_t)p.w | (uintptr_t)p.bias) % 2 || ((uintptr_t)p.out | (uintptr_t)p.residual) % width) return SYMAR_ERR_INVAL;
    if (p.x_ld < 0 || p.x_group < 0 || p.w_ld < 0 || p.w_group < 0 || p.bias_group < 0 || p.residual_ld < 0 || p.residual_group < 0 ||
        p.out_ld < 0 || p.out_group < 0 || rows_meet(p.m, p.out_ld, p.groups, p.out_group, p.n))
        return SYMAR_ERR_INVAL;
    Device d;
    int rc = device_info(&d);
    if (rc == SYMAR_OK) rc = clear();
    if (rc != SYMAR_OK) return rc;
    LinearArgs a{};
    a.x = (const __nv_bfloat16 *)p.x;  a.x_ld = p.x_ld;  a.x_group = p.groups > 1 ? p.x_group : 0;
    a.w = (const __nv_bfloat16 *)p.w;  a.w_ld = p.w_ld;  a.w_group = p.groups > 1 ? p.w_group : 0;
    a.bias = (const __nv_bfloat16 *)p.bias;  a.bias_group = p.bias_group;
    a.residual = p.residual;  a.residual_ld = p.residual_ld;  a.residual_group = p.residual_group;
    a.out = p.out;  a.out_ld = p.out_ld;  a.out_group = p.out_group;
    a.vec_out = ((uintptr_t)p.out % (4 * width) == 0) && p.out_ld % 4 == 0 && p.out_group % 4 == 0;
    a.vec_res = ((uintptr_t)p.residual % (4 * width) == 0) && p.residual_ld % 4 == 0 && p.residual_group % 4 == 0;
    a.m = p.m;  a.n = p.n;  a.k = p.k;  a.act = p.act;  a.root = p.root;  a.status = p.status;
    const bool engine = engine_rows(p.x, p.x_ld, a.x_group, p.m, p.groups, p.k) && engine_rows(p.w, p.w_ld, a.w_group, p.n, p.groups, p.k);
    const bool wide = p.out_dtype == SYMAR_F32;
    // Tokens of a tile: as few columns as hold them all, 256 at most (128 for float32 results, whose sums are registers).
    // Fewer would read the weights again; where tiles are few, clusters share their k instead.
    int nt = 16;
    while (nt < (wide ? 128 : 256) && nt < p.m) nt *= 2;
    switch (nt) {
        case 16: return launch_as<16>(a, p.groups, d, wide, engine, s);
        case 32: return launch_as<32>(a, p.groups, d, wide, engine, s);
        case 64: return launch_as<64>(a, p.groups, d, wide, engine, s);
        case 128: return launch_as<128>(a, p.groups, d, wide, engine, s);
    }
    return launch_as<256>(a, p.groups, d, false, engine, s);
}
