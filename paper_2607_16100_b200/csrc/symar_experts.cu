// One product per expert over the rows of the tokens that chose it, for every rank (formulas in include/symar.h), on the fifth
// generation's tensor cores.
//
// As in symar_linear.cu the weights are the 128 rows of every matrix instruction and the tokens its columns, so that experts with a token
// or two still use all lanes.  Of a tile's 128 weights' rows 64 are the gate's and 64 up's where the activation is gated: both halves
// of a result meet in one block.  How many rows an expert has is known on the device only: every block counts the
// experts' tiles for itself and takes every so-many-th of them; the instruction's columns and what is copied of the tokens go with what a
// tile has, in sixteens.  Four more warps gather the tokens' rows straight into the ring; only pairs of blocks (below) have them put in order beforehand.
//
// A block: one warp fills a ring of 64-wide slices of both operands, one thread issues the products, eight warps take finished accumulators
// out of tensor memory while the next tile is summed in its other half.  Many rows an expert go to pairs of blocks, few tiles over a long k to clusters that
// share it.
//
// Bound and measured (B200, within a CUDA graph).  A few tokens: the weights' bytes; one token's eight experts of 2 x 768 x 2048 take 14.6 us for 50 MB (a start of
// 6 us, then 6 TB/s), 64 tokens on four ranks of 64 experts of 2048 x 352 63 us for 376 MB (5.95 TB/s, 0.91 of the measured copy rate).  Many: the tensor cores (75% of the
// cycles in 212 us of pair_kernel), the experts' uneven numbers of rows (a fifth of it), and putting rows in order.  Small ragged products: the start, a tile's
// epilogue and two rounds of tiles (333 tokens, 7 experts of 1003 x 520 on two ranks, GELU and float32 results: 23.5 us).
#include <type_traits>

#include "symar_act.cuh"
#include "symar_maps.h"
#include "symar_ops.h"
#include "symar_tc.cuh"

namespace symar {
namespace {

struct ExpertsArgs {
    const __nv_bfloat16 *bias, *x;         // (x: where its rows are gathered)
    const int32_t *expert_start, *row_token;
    void    *out;
    int64_t  x_ld, x_group, bias_expert, bias_group, out_ld, out_group;
    int      groups, experts, rows, x_rows, n, k, act, gated;
    int      x_shared, w_shared;           // one for all groups
    int      n_tiles;                      // of 128 channels, or 64 gated ones
    int      vec_out;
    int      split;                        // blocks of a cluster that share a tile's k
    unsigned *status;
};

constexpr int kRows = 128, kHalf = 64, kSlice = 64;
constexpr int kMaxExperts = SYMAR_EXPERTS_MAX;
constexpr int kLoaders = 128;                // threads that gather rows
constexpr int kChunk = 2;                  // slices that a float32 result sums in the tensor cores at a time (see symar_linear.cu).  A bf16 result sums all of its
                                           // block's slices there: its own rounding hides what truncating additions lose (k = 4096: 0.00166 of the result off 64 bits with
                                           // either, 0.2% more of its elements rounded the other way)
constexpr int kBand  = 16;                 // tiles of tokens that run through a column of weights before the next
constexpr int kStep  = 32;                 // tokens that leave the accumulator at a time

__device__ __forceinline__ void results_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ void tma_load4(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
// sixteen bytes of which the first `count` are read and the rest are zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint32_t count)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(count) : "memory");
}
// An arrival of this thread once all its copies so far have landed.
__device__ __forceinline__ void copies_arrive(uint32_t bar)
{
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
// What other threads' copies have written, seen by the tensor cores behind this.
__device__ __forceinline__ void copies_seen() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- clusters ----
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank)
{
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
    return there;
}
// (An address of at_rank.  What it orders is tensor memory alone, by tcgen05's own fences; a release of what the thread has stored would wait for
// its results on their way.)
__device__ __forceinline__ void far_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// A thread's wait for what other blocks of its cluster do
__device__ __forceinline__ bool pair_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ bool pair_wait(uint32_t bar, uint32_t parity, volatile int *failed)
{
    const uint64_t t0 = now_ns();
    for (int i = 1;; ++i) {
        if (pair_try(bar, parity)) return true;
        if (i % 256 == 0 && (*failed || now_ns() - t0 > kWaitNs)) {
            *failed = 1;
            return false;
        }
    }
}
// The same for a whole warp: all its lanes go on, or none.
__device__ __forceinline__ bool pair_warp_wait(uint32_t bar, uint32_t parity, volatile int *failed)
{
    const uint64_t t0 = now_ns();
#pragma unroll 1
    for (int i = 1;; ++i) {
        if (__all_sync(0xffffffffu, pair_try(bar, parity))) return true;
        if (i % 256 == 0 && __any_sync(0xffffffffu, *failed || now_ns() - t0 > kWaitNs)) {
            *failed = 1;
            return false;
        }
    }
}
// (What the block has read of its shared memory is read before: the others may write there again.)
__device__ __forceinline__ void used_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// a word into another block's shared memory (addresses of at_rank), counted by that block's barrier
__device__ __forceinline__ void far_store(uint32_t at, float v, uint32_t bar)
{
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(at), "r"(__float_as_uint(v)), "r"(bar) : "memory");
}

// rows of one copy of a tile's tokens
constexpr int box_of(int nt) { return nt == 64 ? 32 : nt == 128 ? 128 : nt / 2; }

template <int NT, bool kWide, bool kGather, bool kSplit>
struct Shape {
    static constexpr int kThreads = 384 + (kGather ? kLoaders : 0);
    static constexpr int kA = kRows * kSlice * 2, kB = NT * kSlice * 2, kStage = kA + kB;
    static constexpr int kBox  = box_of(NT);
    static constexpr int kHold = (kSplit ? NT : kStep) * kRows * 4;
    static constexpr int kStages = (212 * 1024 - kHold) / kStage;
    static constexpr int kBytes = kStages * kStage + kHold + 1024;      // (the ring starts on a 1 KiB boundary)
    static constexpr int kCols  = 2 * NT;                               // two accumulators
};

// The experts' rows and tiles: first[e] is expert e's first row, tiles[e] the tiles of at most NT rows of the experts before it.
struct Plan {
    int first[kMaxExperts + 1], tiles[kMaxExperts + 1];
};
// by one warp: starts that fall or leave 0 .. rows are brought into order
__device__ __forceinline__ void make_plan(Plan &p, const int32_t *start, int experts, int rows, int nt)
{
    const int lane = threadIdx.x & 31;
    constexpr int kAtOnce = 4;             // loads on their way
    int most = 0, tiles = 0;               // so far
    for (int e0 = 0; e0 <= experts; e0 += 32 * kAtOnce) {
        int v[kAtOnce];
#pragma unroll
        for (int c = 0; c < kAtOnce; ++c) v[c] = e0 + 32 * c + lane <= experts ? max(0, min(start[e0 + 32 * c + lane], rows)) : 0;
#pragma unroll
        for (int c = 0; c < kAtOnce; ++c) {
            const int e = e0 + 32 * c + lane;
            if (e - lane > experts) break;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, v[c], d);
                if (lane >= d) v[c] = max(v[c], u);
            }
            v[c] = max(v[c], most);
            int before = __shfl_up_sync(0xffffffffu, v[c], 1);
            if (lane == 0) before = most;
            // tiles of expert e - 1, which ends here
            int t = e > 0 && e <= experts ? (v[c] - before + nt - 1) / nt : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, t, d);
                if (lane >= d) t += u;
            }
            t += tiles;
            if (e <= experts) p.first[e] = v[c], p.tiles[e] = t;
            most = __shfl_sync(0xffffffffu, v[c], 31), tiles = __shfl_sync(0xffffffffu, t, 31);
        }
    }
}

// An expert's tiles are of one size, in 32s: its last one's weights would cost as much for a few rows as for many.
__device__ __forceinline__ int tile_size(int rows, int m_tiles) { return ((rows + m_tiles - 1) / m_tiles + 31) & ~31; }

struct Tile {
    int g, e, row, count, n0;              // its rows, of one expert, and its first channel
};
// (tiles of `channels` results)
__device__ __forceinline__ Tile tile_of(const Plan &p, const ExpertsArgs &a, int tile, int channels)
{
    Tile t;
    const int per = p.tiles[a.experts] * a.n_tiles;
    t.g = tile / per;
    int i = tile - t.g * per;
    const int m = i / a.n_tiles;           // the last expert whose tiles begin at or before
    int lo = 0, hi = a.experts - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.tiles[mid] <= m) lo = mid;
        else hi = mid - 1;
    }
    t.e = lo;
    const int m_tiles = p.tiles[lo + 1] - p.tiles[lo];
    i -= p.tiles[lo] * a.n_tiles;
    const int b = i / (kBand * a.n_tiles), wide = min(kBand, m_tiles - kBand * b);
    i -= b * kBand * a.n_tiles;
    const int rows = p.first[t.e + 1] - p.first[t.e], size = tile_size(rows, m_tiles), m0 = (kBand * b + i % wide) * size;
    t.row   = p.first[t.e] + m0;
    t.count = min(size, rows - m0);
    t.n0    = i / wide * channels;
    return t;
}

// A thread's four channels: neighbours, or (rows on no boundary, where a warp's stores are to lie side by side) as many apart as there are threads to a
// token.  What the tile's rows share of them:
struct Channels {
    float bias[4], up_bias[4];
    int   in, step, n, count;              // the first one in the tile, to the next, the first one of all, how many there are
};
__device__ __forceinline__ Channels channels_of(const ExpertsArgs &a, const Tile &t, int lane)
{
    Channels c;
    const int threads = a.gated ? 16 : 32, i = lane & (threads - 1);
    c.step  = a.vec_out ? 1 : threads;
    c.in    = a.vec_out ? 4 * i : i;
    c.n     = t.n0 + c.in;
    c.count = max(0, min(4, (a.n - c.n + c.step - 1) / c.step));
    const __nv_bfloat16 *b = a.bias ? a.bias + t.g * a.bias_group + t.e * a.bias_expert : nullptr;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c.bias[j]    = b && j < c.count ? __bfloat162float(b[c.n + j * c.step]) : 0.0f;
        c.up_bias[j] = b && a.gated && j < c.count ? __bfloat162float(b[a.n + c.n + j * c.step]) : 0.0f;
    }
    return c;
}
// (vec_out: rows and n on boundaries of four elements, so all four channels are there or none)
template <typename O>
__device__ __forceinline__ void store(const ExpertsArgs &a, const Channels &c, int g, int row, const float (&y)[4])
{
    O *p = static_cast<O *>(a.out) + g * a.out_group + row * a.out_ld + c.n;
    if (a.vec_out) {
        if (c.count == 4) put4(p, y);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < c.count) put(p + j * c.step, y[j]);
    }
}
__device__ __forceinline__ float4 held4(const float *row, const Channels &c)
{
    if (c.step == 1) return *reinterpret_cast<const float4 *>(row + c.in);
    return make_float4(row[c.in], row[c.in + c.step], row[c.in + 2 * c.step], row[c.in + 3 * c.step]);
}
// What follows the sums of four channels of a tile's token.
template <typename O>
__device__ __forceinline__ void finish_row(const ExpertsArgs &a, const Tile &t, const Channels &c, int token, float4 sum, float4 up)
{
    float y[4] = {sum.x + c.bias[0], sum.y + c.bias[1], sum.z + c.bias[2], sum.w + c.bias[3]};
    activate4(y, a.act);
    if (a.gated) {
        y[0] *= up.x + c.up_bias[0]; y[1] *= up.y + c.up_bias[1]; y[2] *= up.z + c.up_bias[2]; y[3] *= up.w + c.up_bias[3];
    }
    store<O>(a, c, t.g, t.row + token, y);
}
// 32 tokens from c0 on of a tile: out of tensor memory a thread holds one weights' row of many tokens; by way of shared memory it gets four
// neighbouring channels of one token, and up's beside the gate's.
template <typename O>
__device__ __forceinline__ void finish(const ExpertsArgs &a, const Tile &t, const Channels &c, int c0, const float (&v)[16], float *hold, int ew, int side,
                                       int ch, int lane)
{
    const int per = a.gated ? 2 : 1;       // tokens that a warp finishes at once
#pragma unroll
    for (int i = 0; i < 16; ++i) hold[(16 * side + i) * kRows + ch] = v[i];
    results_sync();
    const int count = min(kStep, t.count - c0);
    for (int i = ew * per + (a.gated ? lane >> 4 : 0); i < count; i += 8 * per) {
        const float4 y = held4(hold + i * kRows, c);
        finish_row<O>(a, t, c, c0 + i, y, a.gated ? held4(hold + i * kRows + kHalf, c) : y);
    }
    __syncwarp();                          // (halves of a warp may have had different numbers of tokens; in results_sync itself it costs 3% of a decode batch)
    results_sync();
}

template <int NT, bool kWide, bool kGather, bool kSplit>
__global__ void __launch_bounds__(Shape<NT, kWide, kGather, kSplit>::kThreads, 1)
experts_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ ExpertsArgs a)
{
    using S = Shape<NT, kWide, kGather, kSplit>;
    using O = typename std::conditional<kWide, float, __nv_bfloat16>::type;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Plan plan;
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 6];
    __shared__ uint32_t tmem_at;
    __shared__ int failed, bad;
    unsigned char *ring = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    float *hold = reinterpret_cast<float *>(ring + S::kStages * S::kStage);
    const uint32_t ring_addr = smem_addr(ring);
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 16;
    const uint32_t parts_here = acc_empty + 16, parts_used = parts_here + 8;      // of a tile that several blocks share
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            bar_init(full + 8 * i, kGather ? 1 + kLoaders : 1);
            bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(acc_full + 8 * i, 1);
            bar_init(acc_empty + 8 * i, 256);
        }
        bar_init(parts_here, 1);
        bar_init(parts_used, kSplit ? a.split : 1);
        failed = bad = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 32 && a.k > 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
        if (!kGather) asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(S::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    wait_for_stream();
    if (warp == 3) make_plan(plan, a.expert_start, a.experts, a.rows, NT);
    tc_before();
    if (kSplit) {
        __syncwarp();
        cluster_sync();                    // the other blocks' barriers are there
    } else {
        __syncthreads();
    }
    tc_after();
    const uint32_t tmem = tmem_at;
    const int channels = a.gated ? kHalf : kRows, slices = (a.k + kSlice - 1) / kSlice, tiles = a.groups * plan.tiles[a.experts] * a.n_tiles;
    // this block's slices of every one of its tiles: all of k, or its part where a cluster shares the tile
    const int rank = kSplit ? (int)blockIdx.x % a.split : 0, first = kSplit ? (int)blockIdx.x / a.split : (int)blockIdx.x;
    const int step = kSplit ? (int)gridDim.x / a.split : (int)gridDim.x;
    const int k_lo = kSplit ? (int)((int64_t)slices * rank / a.split) : 0, k_hi = kSplit ? (int)((int64_t)slices * (rank + 1) / a.split) : slices;

    if (warp == 0 && elected()) {
        // ---- producer: one thread.  A copy's own cost counts beside its bytes: one for the tokens, two where half of a small tile's are wanted (boxes of 32
        // rows: 303 us instead of 203 for 16384 rows x 2048 x 4096; two boxes instead of one for 128 rows 13.3 instead of 9.9 us for 1000 x 128 x 520), and no
        // gathering by the copy engine (four rows an instruction: 1090 instead of 203 us).  The weights' two halves in one copy of five axes were slower (15.0 us).
        int st = 0, round = 0;
        for (int tile = first; tile < tiles && slices > 0; tile += step) {
            const Tile t = tile_of(plan, a, tile, channels);
            const int second = t.n0 + (a.gated ? a.n : kHalf), wg = a.w_shared ? 0 : t.g, xg = a.x_shared ? 0 : t.g;
            const bool two = NT > S::kBox && t.count > S::kBox;
            for (int ks = k_lo; ks < k_hi; ++ks) {
                if (round > 0 && !bar_wait(empty + 8 * st, (round - 1) & 1, &failed)) goto done;
                const uint32_t at = ring_addr + st * S::kStage, bar = full + 8 * st;
                bar_expect(bar, S::kA + (kGather ? 0 : two ? S::kB : S::kBox * kSlice * 2));
                tma_load4(at, &wmap, ks * kSlice, t.n0, t.e, wg, bar);
                tma_load4(at + S::kA / 2, &wmap, ks * kSlice, second, t.e, wg, bar);
                if (!kGather) tma_load(at + S::kA, &xmap, ks * kSlice, t.row, xg, bar);
                if (!kGather && two) tma_load(at + S::kA + S::kBox * kSlice * 2, &xmap, ks * kSlice, t.row + S::kBox, xg, bar);
                if (++st == S::kStages) st = 0, ++round;
            }
        }
    } else if (kGather && warp >= 12) {
        // ---- gathered rows: four warps; a thread has one piece of every sixteenth row.  The copies themselves arrive at the stage's barrier; the
        // fence that shows them to the tensor cores is behind the wait for it, as here it would wait for all copies on their way.
        constexpr int kOf = kGather ? NT / 16 : 1;
        const int c = tid & 7, r = (tid - 384) >> 3;
        int st = 0, round = 0;
        Tile t{};
        int token[kOf], next[kOf];                       // of this tile's rows and, asked for a tile ahead, of the next one's
        auto tokens_of = [&](int tile) {
            if (tile >= tiles) return;
            t = tile_of(plan, a, tile, channels);
#pragma unroll
            for (int j = 0; j < kOf; ++j) next[j] = r + 16 * j < t.count ? a.row_token[t.row + r + 16 * j] : -1;      // (columns behind the last are zeros)
        };
        tokens_of(first);
        for (int tile = first; tile < tiles && slices > 0; tile += step) {
            const __nv_bfloat16 *x = a.x + (a.x_shared ? 0 : t.g * a.x_group);
            const int cols = (t.count + 15) & ~15;
#pragma unroll
            for (int j = 0; j < kOf; ++j) {
                token[j] = next[j];
                if (r + 16 * j < t.count && (uint32_t)token[j] >= (uint32_t)a.x_rows) token[j] = -1, bad = 1;
            }
            tokens_of(tile + step);
            for (int ks = k_lo; ks < k_hi; ++ks) {
                if (round > 0 && !warp_wait(empty + 8 * st, (round - 1) & 1, &failed)) goto done;
                const int k0 = ks * kSlice + c * 8;
                const uint32_t count = (uint32_t)max(0, min(8, a.k - k0)) * 2, dst = ring_addr + st * S::kStage + S::kA + r * 128 + ((c ^ (r & 7)) << 4);
#pragma unroll
                for (int j = 0; j < kOf; ++j) {
                    if (16 * j >= cols) break;
                    const bool on = token[j] >= 0 && count > 0;
                    copy16(dst + j * 16 * 128, on ? x + (int64_t)token[j] * a.x_ld + k0 : a.x, on ? count : 0);
                }
                copies_arrive(full + 8 * st);
                if (++st == S::kStages) st = 0, ++round;
            }
        }
    } else if (warp == 1 && elected()) {
        // ---- products: one thread ----
        constexpr uint32_t kHow = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kRows / 16) << 24);
        int st = 0, round = 0;
        uint32_t turn = 0;                              // accumulators filled so far
        for (int tile = first; tile < tiles; tile += step) {
            const uint32_t how = kHow | (uint32_t)((tile_of(plan, a, tile, channels).count + 15) / 16 * 2) << 17;
            for (int ks = k_lo; ks < k_hi;) {
                const int to = kWide ? min(ks + kChunk, k_hi) : k_hi;
                const uint32_t buf = turn & 1, acc = tmem + buf * NT;
                if (turn >= 2 && !bar_wait(acc_empty + 8 * buf, ((turn >> 1) - 1) & 1, &failed)) goto done;
                tc_after();
                for (uint32_t add = 0; ks < to; ++ks, add = 1) {
                    if (!bar_wait(full + 8 * st, round & 1, &failed)) goto done;
                    if (kGather) copies_seen();
                    tc_after();
                    const uint64_t w = operand(ring_addr + st * S::kStage), x = operand(ring_addr + st * S::kStage + S::kA);
                    product(acc, w, x, how, add);
#pragma unroll
                    for (int i = 1; i < kSlice / 16; ++i) product(acc, w + 2 * i, x + 2 * i, how, 1);
                    commit(empty + 8 * st);
                    if (++st == S::kStages) st = 0, ++round;
                }
                commit(acc_full + 8 * buf);
                ++turn;
            }
        }
    } else if (warp >= 4 && warp < 12) {
        // ---- results ----
        const int quarter = warp & 3, side = (warp - 4) >> 2, ew = warp - 4, ch = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)quarter << 21;
        uint32_t turn = 0, shared_tiles = 0;
        bool whole = true;                 // no wait for other blocks gave up: nothing more is sent or expected then, their barriers may be a phase behind
        for (int tile = first; tile < tiles; tile += step) {
            const Tile t = tile_of(plan, a, tile, channels);
            const Channels c = channels_of(a, t, lane);
            constexpr int kOwn = kWide ? NT / 2 : 1;
            float sum[kOwn];
            if (kWide) {
#pragma unroll
                for (int i = 0; i < kOwn; ++i) sum[i] = 0.0f;
                for (int ks = k_lo; ks < k_hi; ks += kChunk, ++turn) {
                    const uint32_t buf = turn & 1;
                    (void)warp_wait(acc_full + 8 * buf, (turn >> 1) & 1, &failed);     // (given up: on with what is there, the barriers count all)
                    tc_after();
#pragma unroll
                    for (int c0 = 0; c0 < kOwn; c0 += 16) {
                        if (2 * c0 + 16 * side >= t.count) continue;
                        float v[16];
                        acc_load16(tmem + lanes + buf * NT + 2 * c0 + 16 * side, v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[kWide ? c0 + i : 0] += v[i];
                    }
                    tc_before();
                    bar_arrive(acc_empty + 8 * buf);
                }
            } else if (slices > 0) {
                (void)warp_wait(acc_full + 8 * (turn & 1), (turn >> 1) & 1, &failed);
                tc_after();
            }
            if (kSplit && shared_tiles > 0) whole &= pair_warp_wait(parts_used, (shared_tiles - 1) & 1, &failed);   // every block has used its parts of the tile before
#pragma unroll
            for (int c0 = 0; c0 < NT; c0 += kStep) {
                if (c0 >= t.count) break;
                float v[16];
                if (kWide) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = sum[kWide ? c0 / 2 + i : 0];
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = 0.0f;
                    if (slices > 0 && c0 + 16 * side < t.count) acc_load16(tmem + lanes + (turn & 1) * NT + c0 + 16 * side, v);
                    if (slices > 0 && c0 + kStep >= t.count) {       // the accumulator is free for the tile after the next
                        tc_before();
                        bar_arrive(acc_empty + 8 * (turn & 1));
                    }
                }
                if (kSplit) {
                    // token i's sums are added up by block i % split, as its token i / split
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int token = c0 + 16 * side + i, to = token % a.split;
                        if (token >= t.count || !whole) break;
                        far_store(at_rank(smem_addr(hold + ((token / a.split) * a.split + rank) * kRows + ch), to), v[i], at_rank(parts_here, to));
                    }
                } else {
                    finish<O>(a, t, c, c0, v, hold, ew, side, ch, lane);
                }
            }
            if (kSplit) {
                const int own = (t.count - rank + a.split - 1) / a.split;      // (0 or less: none)
                if (tid == 128 && whole) bar_expect(parts_here, (uint32_t)(max(own, 0) * a.split * kRows * 4));
                whole &= pair_warp_wait(parts_here, shared_tiles & 1, &failed);
                const int per = a.gated ? 2 : 1;
                for (int i = ew * per + (a.gated ? lane >> 4 : 0); i < own; i += 8 * per) {
                    float4 y4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f), u = y4;
                    for (int r = 0; r < a.split; ++r) {
                        const float *row = hold + (i * a.split + r) * kRows;
                        const float4 y = held4(row, c);
                        y4.x += y.x; y4.y += y.y; y4.z += y.z; y4.w += y.w;
                        if (a.gated) {
                            const float4 w = held4(row + kHalf, c);
                            u.x += w.x; u.y += w.y; u.z += w.z; u.w += w.w;
                        }
                    }
                    finish_row<O>(a, t, c, rank + i * a.split, y4, u);
                }
                __syncwarp();
                results_sync();
                if (tid < 128 + a.split) used_arrive(at_rank(parts_used, (uint32_t)(tid - 128)));
                ++shared_tiles;
            }
            if (!kWide && slices > 0) ++turn;
        }
        if (kSplit && shared_tiles > 0) (void)pair_warp_wait(parts_used, (shared_tiles - 1) & 1, &failed);
    }
done:
    __syncwarp();
    tc_before();
    __syncthreads();
    if (failed) {
        // copies and products may still be in flight: give them time to end before the memory is let go
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        __syncthreads();
    }
    if (kSplit) {
        __syncwarp();
        cluster_sync();                    // no block's memory is in use any more
    }
    if (tid == 0 && a.status && (failed || bad)) atomicCAS(a.status, 0u, (unsigned)(failed ? SYMAR_ERR_TIMEOUT : SYMAR_ERR_INVAL));
    tc_after();
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kCols) : "memory");
}

// ---- pairs of multiprocessors -------------------------------------------------------------
// With many rows an expert, a cluster of two blocks has a tile of 256 weights' rows and up to 256 tokens: each block holds its 128 weights' rows and
// half of the tokens, both read both halves of the tokens, and the first block's thread issues the products of both.  A block's copies are a third
// fewer for the same products.  Rows by token are put in order by a kernel of their own first: gathered into the ring as above they come at 40 bytes a
// cycle at best (16384 rows x 2 x 1024 x 4096 of 32 experts: 304 us with four gathering warps a block, 250 with the rows in order beforehand, of
// which that takes 35; 215 where they are in order already, 177 for four experts of 4096 rows each: 1550 TFLOP/s).
__device__ __forceinline__ void pair_load3(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load4(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_product(uint32_t acc, uint64_t a, uint64_t b, uint32_t how, uint32_t add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(acc),
                 "l"(a), "l"(b), "r"(how), "r"(add) : "memory");
}
__device__ __forceinline__ void pair_commit(uint32_t bar)      // (the barrier at this address in both blocks)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}

constexpr int kPair = 256;                 // tokens of a pair's tile
struct PairShape {
    static constexpr int kA = kRows * kSlice * 2, kB = kPair / 2 * kSlice * 2, kStage = kA + kB, kHold = kStep * kRows * 4;
    static constexpr int kStages = (212 * 1024 - kHold) / kStage;
    static constexpr int kBytes = kStages * kStage + kHold + 1024;
};

__global__ void __launch_bounds__(384, 1)
pair_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const __grid_constant__ ExpertsArgs a)
{
    using S = PairShape;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Plan plan;
    __shared__ __align__(8) uint64_t bars[2 * S::kStages + 4];
    __shared__ uint32_t tmem_at;
    __shared__ int failed;
    unsigned char *ring = smem_raw + ((1024 - (smem_addr(smem_raw) & 1023)) & 1023);
    float *hold = reinterpret_cast<float *>(ring + S::kStages * S::kStage);
    const uint32_t ring_addr = smem_addr(ring);
    const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, acc_full = empty + 8 * S::kStages, acc_empty = acc_full + 16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const uint32_t full0 = at_rank(full, 0), acc_empty0 = at_rank(acc_empty, 0);       // the barriers that the products wait for are the first block's

    if (tid == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            bar_init(full + 8 * i, 1);
            bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(acc_full + 8 * i, 1);
            bar_init(acc_empty + 8 * i, 2 * 8);
        }
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_at)), "n"(2 * kPair) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    wait_for_stream();
    if (warp == 3) make_plan(plan, a.expert_start, a.experts, a.rows, kPair);
    __syncwarp();
    tc_before();
    cluster_sync();                        // the other block's barriers are there
    tc_after();
    const uint32_t tmem = tmem_at;
    const int own = a.gated ? kHalf : kRows, channels = 2 * own, slices = (a.k + kSlice - 1) / kSlice, tiles = a.groups * plan.tiles[a.experts] * a.n_tiles;
    const int first = (int)blockIdx.x / 2, step = (int)gridDim.x / 2;

    if (warp == 0 && elected()) {
        // ---- producer: one thread of each block ----
        int st = 0, round = 0;
        for (int tile = first; tile < tiles && slices > 0; tile += step) {
            const Tile t = tile_of(plan, a, tile, channels);
            const int half = ((t.count + 31) & ~31) / 2, n0 = t.n0 + (int)rank * own, second = n0 + (a.gated ? a.n : kHalf);
            const int wg = a.w_shared ? 0 : t.g, xg = a.x_shared ? 0 : t.g;
            for (int ks = 0; ks < slices; ++ks) {
                if (round > 0 && !bar_wait(empty + 8 * st, (round - 1) & 1, &failed)) goto done;
                const uint32_t at = ring_addr + st * S::kStage, bar = full0 + 8 * st;
                if (rank == 0) bar_expect(full + 8 * st, 2 * S::kStage);
                pair_load4(at, &wmap, ks * kSlice, n0, t.e, wg, bar);
                pair_load4(at + S::kA / 2, &wmap, ks * kSlice, second, t.e, wg, bar);
                pair_load3(at + S::kA, &xmap, ks * kSlice, t.row + (int)rank * half, xg, bar);
                if (++st == S::kStages) st = 0, ++round;
            }
        }
        for (int i = 0; i < S::kStages; ++i) {           // the products' last arrivals, which come from the other block, find this one there
            if (round > 0 && !bar_wait(empty + 8 * st, (round - 1) & 1, &failed)) goto done;
            if (++st == S::kStages) st = 0, ++round;
        }
    } else if (warp == 1 && rank == 0 && elected()) {
        // ---- products of both blocks: one thread ----
        constexpr uint32_t kHow = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(2 * kRows / 16) << 24);
        int st = 0, round = 0;
        uint32_t turn = 0;                              // accumulators filled so far
        for (int tile = first; tile < tiles && slices > 0; tile += step) {
            const uint32_t how = kHow | (uint32_t)((tile_of(plan, a, tile, channels).count + 31) / 32 * 4) << 17;
            const uint32_t buf = turn & 1, acc = tmem + buf * kPair;
            if (turn >= 2 && !pair_wait(acc_empty + 8 * buf, ((turn >> 1) - 1) & 1, &failed)) goto done;
            tc_after();
            for (int ks = 0; ks < slices; ++ks) {
                if (!pair_wait(full + 8 * st, round & 1, &failed)) goto done;
                tc_after();
                const uint64_t w = operand(ring_addr + st * S::kStage), x = operand(ring_addr + st * S::kStage + S::kA);
#pragma unroll
                for (int i = 0; i < kSlice / 16; ++i) pair_product(acc, w + 2 * i, x + 2 * i, how, ks > 0 || i > 0);
                pair_commit(empty + 8 * st);
                if (++st == S::kStages) st = 0, ++round;
            }
            pair_commit(acc_full + 8 * buf);
            ++turn;
        }
    } else if (warp >= 4 && warp < 12) {
        // ---- results: this block's weights' rows, all tokens ----
        const int quarter = warp & 3, side = (warp - 4) >> 2, ew = warp - 4, ch = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)quarter << 21;
        uint32_t turn = 0;
        for (int tile = first; tile < tiles; tile += step) {
            Tile t = tile_of(plan, a, tile, channels);
            t.n0 += (int)rank * own;
            const Channels c = channels_of(a, t, lane);
            if (slices > 0) {
                (void)warp_wait(acc_full + 8 * (turn & 1), (turn >> 1) & 1, &failed);     // (given up: on with what is there, the barriers count all)
                tc_after();
            }
#pragma unroll 1
            for (int c0 = 0; c0 < t.count; c0 += kStep) {
                float v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = 0.0f;
                if (slices > 0 && c0 + 16 * side < t.count) acc_load16(tmem + lanes + (turn & 1) * kPair + c0 + 16 * side, v);
                if (slices > 0 && c0 + kStep >= t.count) {       // the accumulator is free for the tile after the next
                    tc_before();
                    __syncwarp();
                    if (lane == 0) far_arrive(acc_empty0 + 8 * (turn & 1));
                }
                finish<__nv_bfloat16>(a, t, c, c0, v, hold, ew, side, ch, lane);
            }
            if (slices > 0) ++turn;
        }
    }
done:
    __syncwarp();
    if (failed) {
        // copies and products may still be in flight: give them time to end before the memory is let go
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    }
    __syncwarp();
    tc_before();
    cluster_sync();                        // neither block's memory is in use any more
    tc_after();
    if (tid == 0 && a.status && failed) atomicCAS(a.status, 0u, (unsigned)SYMAR_ERR_TIMEOUT);
    if (warp == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(2 * kPair) : "memory");
}

// Rows of x in the lists' order: sixteen bytes a thread and step; rows of nobody are left out.
struct GatherArgs {
    const unsigned char *x;
    unsigned char       *out;              // [groups][rows][pieces of 16 bytes]
    const int32_t *expert_start, *row_token;
    int64_t   x_ld, x_group;               // bytes
    int       experts, rows, x_rows, groups, k, pieces;
    unsigned *status;
};
constexpr int kGatherThreads = 256;

__global__ void __launch_bounds__(kGatherThreads) gather_kernel(const __grid_constant__ GatherArgs a)
{
    wait_for_stream();
    const int lane = threadIdx.x & 31;
    const int from = max(0, min(a.expert_start[0], a.rows));
    int count = 0;                         // rows of somebody, from there on (see make_plan)
    for (int e = lane; e <= a.experts; e += 32) count = max(count, a.expert_start[e]);
    count = max(0, min(__reduce_max_sync(0xffffffffu, count), a.rows) - from);
    // a warp's unit: 128 pieces of a row, four of them a lane
    const int parts = (a.pieces + 127) / 128, whole = a.k / 8;
    const int64_t units = (int64_t)a.groups * count * parts;
    for (int64_t i = (int64_t)blockIdx.x * (kGatherThreads / 32) + (threadIdx.x >> 5); i < units; i += (int64_t)(kGatherThreads / 32) * gridDim.x) {
        const int64_t cell = i / parts;
        const int c0 = (int)(i - cell * parts) * 128 + lane, g = (int)(cell / count), row = from + (int)(cell - (int64_t)g * count);
        const int token = a.row_token[row];
        const bool there = token >= 0 && token < a.x_rows;
        if (!there && c0 == 0 && a.status) atomicCAS(a.status, 0u, (unsigned)SYMAR_ERR_INVAL);
        const unsigned char *x = a.x + g * a.x_group + (there ? token : 0) * a.x_ld;
        uint4 *out = reinterpret_cast<uint4 *>(a.out) + ((int64_t)g * a.rows + row) * a.pieces;
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c0 + 32 * j < whole) v[j] = *reinterpret_cast<const uint4 *>(x + 16ll * (c0 + 32 * j));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c0 + 32 * j;
            if (c < whole) out[c] = there ? v[j] : make_uint4(0, 0, 0, 0);
            else if (c < a.pieces)             // the last one in part
                for (int e = 8 * c; e < a.k; ++e) reinterpret_cast<uint16_t *>(out)[e] = there ? reinterpret_cast<const uint16_t *>(x)[e] : 0;
        }
    }
}

// ---- host ---------------------------------------------------------------------------------
constexpr int kMost = 1 << 30;             // of rows, channels and k: what a tile adds stays below 2^31

// A map of 64-wide boxes over bf16 elements; axes of one element have any stride.
bool encode(CUtensorMap *map, const void *p, int axes, const int64_t *extent, const int64_t *stride, int box)
{
    cuuint64_t dims[4], bytes[3];
    const cuuint32_t boxes[4] = {kSlice, (cuuint32_t)box, 1, 1}, ones[4] = {1, 1, 1, 1};
    int64_t last = (extent[0] + 7) / 8 * 8;
    for (int i = 0; i < axes; ++i) {
        dims[i] = (cuuint64_t)extent[i];
        if (i == 0) continue;
        if (extent[i] > 1) last = stride[i];
        bytes[i - 1] = (cuuint64_t)last * 2;
    }
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, axes, const_cast<void *>(p), dims, bytes, boxes, ones,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Whether the copy engine can walk an axis: steps of 16 bytes, below 2^40 of them.
bool engine_axis(int64_t extent, int64_t stride) { return extent <= 1 || (stride >= 8 && stride % 8 == 0 && stride < (1ll << 39)); }

// Clusters of s blocks that run at once.  The chip's groups of multiprocessors are no multiples of eight: of sixteen clusters of eight two waited for the
// others (16 tiles over k = 4672 17.6 us instead of 9.4 for 14), so a few less are counted on.
int clusters_of(int sms, int s) { return s == 8 ? sms / 8 * 3 / 4 : s == 4 ? sms / 4 * 9 / 10 : sms / s; }
template <int NT, bool kWide, bool kGather, bool kSplit>
int launch(const ExpertsArgs &a, int tiles, const CUtensorMap &wmap, const CUtensorMap &xmap, const Device &d, cudaStream_t stream)
{
    using S = Shape<NT, kWide, kGather, kSplit>;
    auto fn = experts_kernel<NT, kWide, kGather, kSplit>;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_shared((const void *)fn, S::kBytes, d.id, allowed);
    if (e != cudaSuccess) return cuda_fail(e, "symar_experts");
    const int most = clusters_of(d.sms, a.split);
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    cfg.gridDim  = dim3((unsigned)(a.split * (tiles < most ? tiles : most)));
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kBytes;
    cfg.stream   = stream;
    cfg.attrs    = attr;
    cfg.numAttrs = kSplit ? 2 : 1;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // (see wait_for_stream)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    e = cudaLaunchKernelEx(&cfg, fn, wmap, xmap, a);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_experts");
}
// Blocks that share a tile's k, where tiles are few: what a multiprocessor does then in slices, an exchange of parts counted as four.
int split_of(int tiles, int slices, int sms)
{
    int best = 1;
    int64_t least = (int64_t)((tiles + sms - 1) / sms) * (slices + 1);
    for (int s = 2; s <= 8; s *= 2) {
        const int clusters = clusters_of(sms, s);
        const int64_t cost = (int64_t)((tiles + clusters - 1) / clusters) * ((slices + s - 1) / s + 4);
        if (slices >= 2 * s && cost < least) least = cost, best = s;
    }
    return best;
}
template <int NT, bool kWide>
int launch_as(ExpertsArgs a, const CUtensorMap &wmap, const CUtensorMap &xmap, const Device &d, cudaStream_t s)
{
    const int64_t used = a.experts < a.rows ? a.experts : a.rows, tiles = (int64_t)a.groups * a.n_tiles * (a.rows / NT + used);      // at most
    if (tiles > kMost || (int64_t)a.n_tiles * kBand > kMost) return SYMAR_ERR_UNSUPPORTED;
    a.split = 1;
    if constexpr (NT == 64) {
        a.split = split_of((int)tiles, (a.k + kSlice - 1) / kSlice, d.sms);
        if (a.split > 1)
            return a.row_token ? launch<NT, kWide, true, true>(a, (int)tiles, wmap, xmap, d, s) : launch<NT, kWide, false, true>(a, (int)tiles, wmap, xmap, d, s);
    }
    return a.row_token ? launch<NT, kWide, true, false>(a, (int)tiles, wmap, xmap, d, s) : launch<NT, kWide, false, false>(a, (int)tiles, wmap, xmap, d, s);
}

int launch_pair(ExpertsArgs a, const CUtensorMap &wmap, const CUtensorMap &xmap, const Device &d, cudaStream_t stream)
{
    a.n_tiles = (a.n_tiles + 1) / 2;       // of both blocks' channels
    const int64_t used = a.experts < a.rows ? a.experts : a.rows, tiles = (int64_t)a.groups * a.n_tiles * (a.rows / kPair + used);      // at most
    if (tiles > kMost || (int64_t)a.n_tiles * kBand > kMost) return SYMAR_ERR_UNSUPPORTED;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_shared((const void *)pair_kernel, PairShape::kBytes, d.id, allowed);
    if (e != cudaSuccess) return cuda_fail(e, "symar_experts");
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2];
    cfg.gridDim  = dim3((unsigned)(2 * (tiles < d.sms / 2 ? tiles : d.sms / 2)));
    cfg.blockDim = dim3(384);
    cfg.dynamicSmemBytes = PairShape::kBytes;
    cfg.stream   = stream;
    cfg.attrs    = attr;
    cfg.numAttrs = 2;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;       // (see wait_for_stream)
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    e = cudaLaunchKernelEx(&cfg, pair_kernel, wmap, xmap, a);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_experts");
}

// Tokens of a tile, by what an expert has of them on average: few leave room for more weights on their way, many read them less often (64 or 128 with 32 experts of
// 2 x 1024 x 4096: 25 rows each 96.6 and 100 us, 50 rows 118 and 111).  Pairs take many rows where their tiles are enough for all multiprocessors (a product's start costs
// them 3 us more: 1000 rows x 128 x 520 of seven experts 13.3 us instead of 9.9; with 1003 channels on two ranks 17.9 instead of 19.3) and the gathering beforehand is
// little beside the products (75 rows each of k = 4096: 112 us instead of 123, of k = 1024 25.3 instead of 22.9).  148 is the chip's number of multiprocessors: the
// workspace goes by the same rule and is asked for by sizes alone, without a device.
int tile_tokens(const symar_experts_t &p)
{
    const int64_t used = p.experts < p.rows ? p.experts : p.rows, each = used > 0 ? p.rows / used : 0;
    const int64_t tiles = (int64_t)p.groups * (p.gated ? (p.n + kHalf - 1) / kHalf : (p.n + kRows - 1) / kRows) * (p.rows / kPair + used);
    if (each <= 32) return 64;
    return each <= (p.k < 2048 ? 96 : 48) || tiles < 148 || p.out_dtype == SYMAR_F32 ? 128 : kPair;
}
bool in_order_first(const symar_experts_t &p) { return p.row_token && p.k > 0 && tile_tokens(p) == kPair; }
int64_t pieces_of(int k) { return ((int64_t)k + 7) / 8; }

}  // namespace
}  // namespace symar

using namespace symar;

extern "C" size_t symar_experts_workspace(const symar_experts_t *p)
{
    if (!p || p->groups <= 0 || p->experts <= 0 || p->rows <= 0 || p->n <= 0 || p->k <= 0 || !in_order_first(*p)) return 0;
    const int64_t groups = p->groups > 1 && p->x_group != 0 ? p->groups : 1;
    const __int128 bytes = (__int128)groups * p->rows * pieces_of(p->k) * 16;
    return bytes < ((__int128)1 << 62) ? (size_t)bytes : (size_t)1 << 62;
}

extern "C" int symar_experts(const symar_experts_t *args, void *cuda_stream)
{
    if (!args) return SYMAR_ERR_INVAL;
    const symar_experts_t &p = *args;
    if (p.groups < 0 || p.experts < 0 || p.rows < 0 || p.x_rows < 0 || p.n < 0 || p.k < 0 || p.act < SYMAR_ACT_NONE || p.act > SYMAR_ACT_SILU ||
        p.gated < 0 || p.gated > 1 || (p.out_dtype != SYMAR_F32 && p.out_dtype != SYMAR_BF16) || (uintptr_t)p.status % 4)
        return SYMAR_ERR_INVAL;
    if (p.experts > kMaxExperts || p.rows > kMost || p.x_rows > kMost || p.n > kMost || p.k > kMost) return SYMAR_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    auto clear = [&] {
        const cudaError_t e = p.status ? cudaMemsetAsync(p.status, 0, sizeof(unsigned), s) : cudaSuccess;
        return e == cudaSuccess ? (int)SYMAR_OK : cuda_fail(e, "cudaMemsetAsync");
    };
    if (p.groups == 0 || p.experts == 0 || p.rows == 0 || p.n == 0) return clear();
    const uintptr_t width = p.out_dtype == SYMAR_F32 ? 4 : 2;
    if (!p.out || !p.expert_start || (p.k > 0 && (!p.x || !p.w || p.x_rows == 0))) return SYMAR_ERR_INVAL;
    if (((uintptr_t)p.x | (uintptr_t)p.w | (uintptr_t)p.bias) % 2 || (uintptr_t)p.out % width || ((uintptr_t)p.expert_start | (uintptr_t)p.row_token) % 4)
        return SYMAR_ERR_INVAL;
    if (!p.row_token && p.x_rows < p.rows) return SYMAR_ERR_INVAL;
    if (p.x_ld < 0 || p.x_group < 0 || p.w_ld < 0 || p.w_expert < 0 || p.w_group < 0 || p.bias_expert < 0 || p.bias_group < 0 || p.out_ld < 0 ||
        p.out_group < 0 || rows_meet(p.rows, p.out_ld, p.groups, p.out_group, p.n))
        return SYMAR_ERR_INVAL;
    Device d;
    ExpertsArgs a{};
    a.bias = (const __nv_bfloat16 *)p.bias;  a.bias_expert = p.bias_expert;  a.bias_group = p.bias_group;
    a.x = (const __nv_bfloat16 *)p.x;  a.x_ld = p.x_ld;  a.x_group = p.x_group;
    a.expert_start = p.expert_start;  a.row_token = p.row_token;
    a.out = p.out;  a.out_ld = p.out_ld;  a.out_group = p.out_group;
    a.groups = p.groups;  a.experts = p.experts;  a.rows = p.rows;  a.x_rows = p.x_rows;
    a.n = p.n;  a.k = p.k;  a.act = p.act;  a.gated = p.gated;
    a.x_shared = p.groups == 1 || p.x_group == 0;
    a.w_shared = p.groups == 1 || p.w_group == 0;
    a.n_tiles = p.gated ? (p.n + kHalf - 1) / kHalf : (p.n + kRows - 1) / kRows;
    a.vec_out = (uintptr_t)p.out % (4 * width) == 0 && p.out_ld % 4 == 0 && p.out_group % 4 == 0 && p.n % 4 == 0;
    a.status = p.status;
    CUtensorMap wmap{}, xmap{};
    const bool wide = p.out_dtype == SYMAR_F32, first = in_order_first(p);
    const int nt = tile_tokens(p);
    GatherArgs ga{};
    if (p.k > 0) {
        const int64_t w_rows = (int64_t)p.n * (p.gated ? 2 : 1);
        const int64_t w_extent[4] = {p.k, w_rows, p.experts, a.w_shared ? 1 : p.groups}, w_stride[4] = {1, p.w_ld, p.w_expert, p.w_group};
        int64_t x_extent[3] = {p.k, p.x_rows, a.x_shared ? 1 : p.groups}, x_stride[3] = {1, p.x_ld, p.x_group};
        bool ok = encoder() && ((uintptr_t)p.x | (uintptr_t)p.w) % 16 == 0;
        for (int i = 1; i < 4; ++i) ok = ok && engine_axis(w_extent[i], w_stride[i]);
        for (int i = 1; i < 3; ++i) ok = ok && engine_axis(x_extent[i], x_stride[i]);
        if (!ok) return SYMAR_ERR_UNSUPPORTED;
        const void *x = p.x;
        if (first) {
            const size_t need = symar_experts_workspace(&p);
            if (!p.workspace || (uintptr_t)p.workspace % 16) return SYMAR_ERR_INVAL;
            if (p.workspace_bytes < need) return SYMAR_ERR_NOMEM;
            ga = GatherArgs{(const unsigned char *)p.x, (unsigned char *)p.workspace, p.expert_start, p.row_token, 2 * p.x_ld, 2 * p.x_group, p.experts, p.rows,
                            p.x_rows, (int)x_extent[2], p.k, (int)pieces_of(p.k), p.status};
            x = p.workspace;
            x_extent[1] = p.rows, x_stride[1] = 8 * pieces_of(p.k), x_stride[2] = x_stride[1] * p.rows;
            ok = x_stride[2] < (1ll << 39);
        }
        if (ok && (!p.row_token || first)) ok = encode(&xmap, x, 3, x_extent, x_stride, box_of(nt));
        if (!ok || !encode(&wmap, p.w, 4, w_extent, w_stride, kHalf)) return SYMAR_ERR_UNSUPPORTED;
    }
    int rc = device_info(&d);
    if (rc == SYMAR_OK) rc = clear();
    if (rc != SYMAR_OK) return rc;
    if (nt == 64) return wide ? launch_as<64, true>(a, wmap, xmap, d, s) : launch_as<64, false>(a, wmap, xmap, d, s);
    if (nt == 128) return wide ? launch_as<128, true>(a, wmap, xmap, d, s) : launch_as<128, false>(a, wmap, xmap, d, s);
    if (first) {
        const int64_t blocks = ((int64_t)ga.groups * ga.rows * ((ga.pieces + 127) / 128) + kGatherThreads / 32 - 1) / (kGatherThreads / 32), most = 8ll * d.sms;
        const cudaError_t e = launch_early(gather_kernel, dim3((unsigned)(blocks < most ? blocks : most)), kGatherThreads, 0, s, ga);
        if (e != cudaSuccess) return cuda_fail(e, "symar_experts");
    }
    return launch_pair(a, wmap, xmap, d, s);
}
