// What stands around an AllReduce in a decoder layer (formulas in include/symar.h): the block's result normed, gated, scaled and added to
// the residual stream, and the sum normed for the next block, in one pass over the rows.
//
// A row is read once, held in registers as binary32 through both norms and written once.  Sums go over a thread's own elements,
// then over the row's threads by shuffles and, where they are several warps, by shared memory; a layer norm takes the mean first
// and the squares of what is left after it, so that a large mean costs no digits.
//
// Bound and measured (B200, within a CUDA graph).  A few rows: latency; one of 8192 takes 2.9 us, of which the launch is most.  Many long
// ones: bytes; 16384 x 8192 with norms on both sides and a gate a channel takes 200 us for 1.07 GB (5.4 TB/s, 0.82 of the measured copy rate), with the norm before
// the next block alone 188 us, 16384 x 4096 of float32 189 and 175 us; what keeps it from the copy's rate is the row's chain of two sums among half the warps a multiprocessor could have.  Short
// ones: instructions and their latency (61% of the issue slots at 44% of the warps); 73728 heads of 128 out of rows of 20 take 12.9 us (2.9 TB/s), of
// float32 16.5.  Rows on no 16-byte boundary: the same (50% at 40%), as every element is read and written by itself; 1501 x 2049, two layer norms with bias
// and a float32 stream, takes 19.9 us where 2048 takes 17.7.
#include <type_traits>

#include "symar_eights.cuh"
#include "symar_maps.h"
#include "symar_norm_side.h"
#include "symar_ops.h"
#include "symar_tc.cuh"

namespace symar {
namespace {

struct NormArgs {
    const void *x, *residual, *gate;
    void       *residual_out, *out;
    int64_t x_ld, x_group, residual_ld, residual_group, residual_out_ld, residual_out_group, out_ld, out_group, gate_ld, gate_group;
    Side    after, before;
    float   scale, residual_scale;
    int     m, n, rows;
    int     x_wide, stream_wide, gate_step, gate_act;
    unsigned *status;
};

// A row's share of one thread: C chunks of eight elements.  Where chunk c begins; in rows on no 16-byte boundary its elements are T apart.
template <bool kVec> __device__ __forceinline__ int first(int c, int i, int T) { return kVec ? (c * T + i) * 8 : c * 8 * T + i; }
template <bool kVec> __device__ __forceinline__ bool inside(int c, int j, int i, int T, int n) { return first<kVec>(c, i, T) + (kVec ? j : j * T) < n; }

__device__ __forceinline__ float lanes_sum(float s, int lanes)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
        if (d < lanes) s += __shfl_xor_sync(0xffffffffu, s, d);
    return s;
}
// Sums over a row's threads, the same on every one of them: L lanes of a warp, or T threads (whole warps) that meet at a barrier.  No two sums of a row
// use the same room.
template <int L> struct LanesSum {
    __device__ __forceinline__ float operator()(float s, int) const { return lanes_sum(s, L); }
};
struct ThreadsSum {
    float *room;                           // [4][32]
    int    warps, warp, barrier;
    __device__ __forceinline__ float operator()(float s, int which) const
    {
        s = lanes_sum(s, 32);
        if (warps == 1) return s;
        const int lane = threadIdx.x & 31;
        if (lane == 0) room[32 * which + warp] = s;
        asm volatile("bar.sync %0, %1;" ::"r"(barrier), "r"(32 * warps) : "memory");
        return lanes_sum(lane < warps ? room[32 * which + lane] : 0.0f, 32);       // (zeros behind the last: in every lane the same order)
    }
};

// A side's weights and biases of chunk c as a kernel has them at hand: read for this row (kRead: already), or held as floats for all rows, where biases,
// which few norms have, are read again.
template <int C, bool kVec, bool kRead> struct ReadVectors {
    Raw w[2][kRead ? C : 1], b[2][kRead ? C : 1];
    int i, T;
    __device__ __forceinline__ void read(const Side &s, int side, int n)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (s.weight) w[side][c] = read8<kVec>(s.weight, s.wide, first<kVec>(c, i, T), T, n);
            if (s.bias) b[side][c] = read8<kVec>(s.bias, s.wide, first<kVec>(c, i, T), T, n);
        }
    }
    __device__ __forceinline__ void weight(const Side &s, int side, int c, int n, float (&f)[8]) const
    {
        values<kVec>(kRead ? w[side][kRead ? c : 0] : read8<kVec>(s.weight, s.wide, first<kVec>(c, i, T), T, n), s.wide, f);
        const float plus = s.plus_one ? 1.0f : 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] += plus;
    }
    __device__ __forceinline__ void bias(const Side &s, int side, int c, int n, float (&f)[8]) const
    {
        values<kVec>(kRead ? b[side][kRead ? c : 0] : read8<kVec>(s.bias, s.wide, first<kVec>(c, i, T), T, n), s.wide, f);
    }
};
template <int C, bool kVec> struct HeldVectors {
    float w[2][C][8];
    int   i, T;
    __device__ __forceinline__ void hold(const Side &s, int side, int n)
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (!s.weight) continue;
            values<kVec>(read8<kVec>(s.weight, s.wide, first<kVec>(c, i, T), T, n), s.wide, w[side][c]);
            const float plus = s.plus_one ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[side][c][j] += plus;
        }
    }
    __device__ __forceinline__ void weight(const Side &, int side, int c, int, float (&f)[8]) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = w[side][c][j];
    }
    __device__ __forceinline__ void bias(const Side &s, int, int c, int n, float (&f)[8]) const
    {
        values<kVec>(read8<kVec>(s.bias, s.wide, first<kVec>(c, i, T), T, n), s.wide, f);
    }
};

template <int C, bool kVec, typename Vectors, typename Sum>
__device__ __forceinline__ void norm_row(float (&v)[C][8], const Side &s, int side, const Vectors &vectors, int i, int T, int n, float inv_n, const Sum &sum)
{
    if (s.kind == SYMAR_NORM_LAYER) {
        float all = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) all += v[c][j];                       // (elements beyond the row are zeros)
        const float mean = sum(all, 2 * side + 1) * inv_n;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = inside<kVec>(c, j, i, T, n) ? v[c][j] - mean : 0.0f;
    }
    float all = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) all = fmaf(v[c][j], v[c][j], all);
    const float by = 1.0f / sqrtf(fmaf(sum(all, 2 * side), inv_n, s.eps));
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] *= by;
        if (s.weight) {
            float w[8];
            vectors.weight(s, side, c, n, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] *= w[j];
        }
        if (s.bias) {
            float b[8];
            vectors.bias(s, side, c, n, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] += b[j];
        }
    }
}
__device__ __forceinline__ void open8(float (&g)[8], int act)
{
    if (act == SYMAR_GATE_SIGMOID) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.0f / (1.0f + expf(-g[j]));
    } else if (act == SYMAR_GATE_TANH) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = tanhf(g[j]);
    }
}
template <typename P> __device__ __forceinline__ P *moved(P *p, int64_t elements, bool wide)
{
    return (P *)((char *)p + elements * (wide ? 4 : 2));
}
// A row's gate where it is one number, times the scale
__device__ __forceinline__ float row_gate(const NormArgs &a, int g, int t)
{
    if (!a.gate || a.gate_step) return a.scale;
    const void *p = moved(a.gate, g * a.gate_group + t * a.gate_ld, a.x_wide);
    float v = a.x_wide ? *static_cast<const float *>(p) : __bfloat162float(*static_cast<const __nv_bfloat16 *>(p));
    if (a.gate_act == SYMAR_GATE_SIGMOID) v = 1.0f / (1.0f + expf(-v));
    else if (a.gate_act == SYMAR_GATE_TANH) v = tanhf(v);
    return a.scale * v;
}
struct Gate {
    const void *p;                         // a row's channels, where there is a gate for each
    bool        wide;
    int         act;
    float       scale;
};
// One row from what in(c), old(c) give of x and residual to what is stored where it is to be kept.  `by`: row_gate(), of gates that are one number.
// kX, kStream: x and the stream are float32.
template <int C, bool kVec, bool kX, bool kStream, typename Vectors, typename Sum, typename In, typename Old>
__device__ __forceinline__ void do_row(const NormArgs &a, const In &in, const Old &old, const Vectors &vectors, const Gate &gate, float by, int g, int t, bool keep,
                                       int i, int T, float inv_n, const Sum &sum)
{
    const int n = a.n;
    float v[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) values<kVec>(in(c), kX, v[c]);
    if (a.after.kind != SYMAR_NORM_NONE) norm_row<C, kVec>(v, a.after, 0, vectors, i, T, n, inv_n, sum);
    if (a.gate && a.gate_step) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float w[8];
            values<kVec>(read8<kVec>(gate.p, gate.wide, first<kVec>(c, i, T), T, n), gate.wide, w);
            open8(w, gate.act);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] *= gate.scale * w[j];
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] *= by;
    }
    if (a.residual) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float h[8];
            values<kVec>(old(c), kStream, h);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = fmaf(a.residual_scale, h[j], v[c][j]);
        }
    }
    if (a.residual_out && keep) {
        void *to = moved(a.residual_out, g * a.residual_out_group + t * a.residual_out_ld, kStream);
#pragma unroll
        for (int c = 0; c < C; ++c) write8<kVec>(to, kStream, first<kVec>(c, i, T), T, n, v[c]);
    }
    if (a.out) {
        norm_row<C, kVec>(v, a.before, 1, vectors, i, T, n, inv_n, sum);
        if (!keep) return;
        void *to = moved(a.out, g * a.out_group + t * a.out_ld, kX);
#pragma unroll
        for (int c = 0; c < C; ++c) write8<kVec>(to, kX, first<kVec>(c, i, T), T, n, v[c]);
    }
}

// ---- a block has a row: few rows, and long ones on no boundary ----
// kT: threads of a block (0: as launched; on no boundary elements a known number apart need no arithmetic for each address).
template <int C, int kT, bool kX, bool kStream>
__global__ void __launch_bounds__(kT ? kT : 1024, kT && kT <= 256 ? 1024 / (kT ? kT : 1) : 1) row_kernel(const __grid_constant__ NormArgs a)
{
    constexpr bool kVec = kT == 0;
    __shared__ float room[4 * 32];
    wait_for_stream();
    const int T = kT ? kT : blockDim.x, i = threadIdx.x, row = blockIdx.x, g = row / a.m, t = row - g * a.m;
    const void *x = moved(a.x, g * a.x_group + t * a.x_ld, kX);
    Raw in[C], old[C] = {};
#pragma unroll
    for (int c = 0; c < C; ++c) in[c] = read8<kVec>(x, kX, first<kVec>(c, i, T), T, a.n);
    if (a.residual) {
        const void *h = moved(a.residual, g * a.residual_group + t * a.residual_ld, kStream);
#pragma unroll
        for (int c = 0; c < C; ++c) old[c] = read8<kVec>(h, kStream, first<kVec>(c, i, T), T, a.n);
    }
    ReadVectors<C, kVec, C == 1> vectors;  // (one trip to memory where registers allow it)
    vectors.i = i, vectors.T = T;
    if constexpr (C == 1) vectors.read(a.after, 0, a.n), vectors.read(a.before, 1, a.n);
    const float by = row_gate(a, g, t);
    do_row<C, kVec, kX, kStream>(a, [&](int c) { return in[c]; }, [&](int c) { return old[c]; }, vectors,
                                 Gate{moved(a.gate, g * a.gate_group + t * a.gate_ld, kX), kX, a.gate_act, a.scale}, by, g, t, true, i, T, 1.0f / (float)a.n, ThreadsSum{room, T / 32, i >> 5, 0});
}

// ---- L lanes of a warp have a row: short rows, U of them asked for before the first is computed ----
constexpr int kShortThreads = 256;

template <int L, int C, int U, bool kVec, bool kX, bool kStream>
__global__ void __launch_bounds__(kShortThreads, C == 1 ? 4 : C == 2 ? 3 : 2) short_kernel(const __grid_constant__ NormArgs a)
{
    wait_for_stream();
    const int i = (int)threadIdx.x % L, slot = (int)(blockIdx.x * kShortThreads + threadIdx.x) / L, slots = (int)gridDim.x * (kShortThreads / L);
    const float inv_n = 1.0f / (float)a.n;
    typename std::conditional<C == 1, HeldVectors<C, kVec>, ReadVectors<C, kVec, false>>::type vectors;
    vectors.i = i, vectors.T = L;
    if constexpr (C == 1) vectors.hold(a.after, 0, a.n), vectors.hold(a.before, 1, a.n);
    for (int64_t row0 = (int64_t)(slot / (32 / L)) * (32 / L) * U; row0 < a.rows; row0 += (int64_t)slots * U) {      // (whole warps go on together)
        Raw in[U][C], old[U][C] = {};
        int g[U], t[U];
        float by[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (rows behind the last read the last one's and are not stored)
            const int row = (int)min(row0 + u * (32 / L) + slot % (32 / L), (int64_t)a.rows - 1);
            g[u] = row / a.m, t[u] = row - g[u] * a.m;
            const void *x = moved(a.x, g[u] * a.x_group + t[u] * a.x_ld, kX);
#pragma unroll
            for (int c = 0; c < C; ++c) in[u][c] = read8<kVec>(x, kX, first<kVec>(c, i, L), L, a.n);
            if (a.residual) {
                const void *h = moved(a.residual, g[u] * a.residual_group + t[u] * a.residual_ld, kStream);
#pragma unroll
                for (int c = 0; c < C; ++c) old[u][c] = read8<kVec>(h, kStream, first<kVec>(c, i, L), L, a.n);
            }
            by[u] = row_gate(a, g[u], t[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            do_row<C, kVec, kX, kStream>(a, [&](int c) { return in[u][c]; }, [&](int c) { return old[u][c]; }, vectors,
                                         Gate{moved(a.gate, g[u] * a.gate_group + t[u] * a.gate_ld, kX), kX, a.gate_act, a.scale}, by[u], g[u], t[u],
                                         row0 + u * (32 / L) + slot % (32 / L) < a.rows, i, L, inv_n, LanesSum<L>{});
    }
}

// ---- many long rows: a block for each multiprocessor, whose groups of threads have a row each; the copy engine brings a group's next rows into its
// slots of shared memory meanwhile, so that reading never waits for the sums.  Weights and gates that all rows share lie in shared memory too. ----
struct Ring {
    int T, groups, slots;                  // threads of a group; groups; a group's slots
    int x_bytes, old_bytes, gate_bytes;    // of a row in a slot: x, residual, gate (0: not in it)
    int held;                              // bytes of what all rows share
};
constexpr int kRingThreads = 512, kRingRoom = 208 * 1024 - 32, kMaxSlots = 8, kMaxGroups = 15, kRingMost = 32 * kRingThreads;

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// eight values at a place in shared memory
__device__ __forceinline__ void shared8(const unsigned char *p, bool wide, float (&v)[8])
{
    const uint4 lo = *reinterpret_cast<const uint4 *>(p);
    Raw r;
    r.w[0] = lo.x; r.w[1] = lo.y; r.w[2] = lo.z; r.w[3] = lo.w;
    if (wide) {
        const uint4 hi = *reinterpret_cast<const uint4 *>(p + 16);
        r.w[4] = hi.x; r.w[5] = hi.y; r.w[6] = hi.z; r.w[7] = hi.w;
    }
    values<true>(r, wide, v);
}
// A vector that all rows share, in shared memory from this thread's first element on.
struct Held {
    int there, at, wide, step;             // step: bytes from a chunk to the next
};

// A thread has four chunks of eight elements: what it does once a row is then little beside what it does for every element, and that is
// what this kernel is made of (the row kernel's code in its place, sixteen elements a thread: 57 instructions an element and 275 us
// for 16384 x 8192 with two norms).
template <bool kX, bool kStream>
__global__ void __launch_bounds__(kRingThreads, 1) ring_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ Ring ring)
{
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(8) uint64_t bars[kMaxGroups * kMaxSlots];
    __shared__ float room[kMaxGroups * 2 * 4 * 32];            // a row's four sums, of every second row
    __shared__ int failed;
    constexpr int C = 4, kZero = 32, kXB = kX ? 4 : 2, kSB = kStream ? 4 : 2;
    const int T = ring.T, group = (int)threadIdx.x / T, i = (int)threadIdx.x - group * T, n = a.n;
    if (threadIdx.x == 0) {
        for (int b = 0; b < ring.groups * ring.slots; ++b) bar_init(smem_addr(bars + b), 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    wait_for_stream();
    // chunks behind the row's end read zeros from the first 32 bytes, so that nothing branches
    if (threadIdx.x < kZero / 4) reinterpret_cast<uint32_t *>(smem)[threadIdx.x] = 0;
    int used = kZero;
    auto hold = [&](const void *p, bool wide) {
        const int width = wide ? 4 : 2, bytes = n * width, at = used;
        if (!p) return Held{0, 0, 0, 0};
        for (int b = 16 * (int)threadIdx.x; b < bytes; b += 16 * (int)blockDim.x)
            *reinterpret_cast<uint4 *>(smem + at + b) = *reinterpret_cast<const uint4 *>(static_cast<const char *>(p) + b);
        used += bytes;
        return Held{1, at + 8 * i * width, wide, 8 * T * width};
    };
    const Held w0 = hold(a.after.weight, a.after.wide), b0 = hold(a.after.bias, a.after.wide), w1 = hold(a.before.weight, a.before.wide),
               b1 = hold(a.before.bias, a.before.wide);
    Held gate{0, 0, 0, 0};
    if (a.gate && a.gate_step && !ring.gate_bytes) {           // with its function and the scale
        float *to = reinterpret_cast<float *>(smem + used);
        for (int c = 8 * (int)threadIdx.x; c < n; c += 8 * (int)blockDim.x) {
            float f[8];
            values<true>(read8<true>(a.gate, kX, c, 0, n), kX, f);
            open8(f, a.gate_act);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] *= a.scale;
            write8<true>(to, true, c, 0, n, f);
        }
        gate = Held{1, used + 32 * i, 1, 32 * T};
    }
    __syncthreads();
    const int slot_bytes = ring.x_bytes + ring.old_bytes + ring.gate_bytes, step = (int)gridDim.x * ring.groups;
    const int slots = kZero + ring.held + group * ring.slots * slot_bytes;
    const uint32_t bar0 = smem_addr(bars + group * ring.slots);
    const float inv_n = 1.0f / (float)n;
    auto ask = [&](int64_t row, int s) {   // (by one thread)
        if (row >= a.rows) return;
        const int g = (int)row / a.m, t = (int)row - g * a.m;
        const uint32_t to = smem_addr(smem) + slots + s * slot_bytes, bar = bar0 + 8 * s;
        bar_expect(bar, (uint32_t)slot_bytes);
        bulk_load(to, moved(a.x, g * a.x_group + t * a.x_ld, kX), ring.x_bytes, bar);
        if (ring.old_bytes) bulk_load(to + ring.x_bytes, moved(a.residual, g * a.residual_group + t * a.residual_ld, kStream), ring.old_bytes, bar);
        if (ring.gate_bytes) bulk_load(to + ring.x_bytes + ring.old_bytes, moved(a.gate, g * a.gate_group + t * a.gate_ld, kX), ring.gate_bytes, bar);
    };
    int64_t row = (int64_t)blockIdx.x * ring.groups + group;
    if (i == 0)
        for (int s = 0; s < ring.slots; ++s) ask(row + (int64_t)s * step, s);
    bool on[C];
#pragma unroll
    for (int c = 0; c < C; ++c) on[c] = (c * T + i) * 8 < n;

    float v[C][8];
    auto normed = [&](const Side &s, const Held &w, const Held &b, const ThreadsSum &sum, int which) {
        if (s.kind == SYMAR_NORM_LAYER) {
            float all = 0.0f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) all += v[c][j];                   // (elements beyond the row are zeros)
            const float mean = sum(all, which + 1) * inv_n;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = on[c] ? v[c][j] - mean : 0.0f;
        }
        float all = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) all = fmaf(v[c][j], v[c][j], all);
        const float by = 1.0f / sqrtf(fmaf(sum(all, which), inv_n, s.eps));
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] *= by;
            if (w.there) {
                float f[8];
                shared8(smem + (on[c] ? w.at + c * w.step : 0), w.wide, f);
                if (s.plus_one) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) f[j] += 1.0f;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= f[j];
            }
            if (b.there) {
                float f[8];
                shared8(smem + (on[c] ? b.at + c * b.step : 0), b.wide, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] += f[j];
            }
        }
    };
    auto gate_of = [&](int64_t r) { return r < a.rows ? row_gate(a, (int)r / a.m, (int)r % a.m) : 0.0f; };
    const bool row_gates = a.gate && !a.gate_step;
    float by = row_gates ? gate_of(row) : a.scale;
    uint32_t turn = 0;
    bool whole = true;                     // no wait gave up: nothing more is asked for then, as slots may still be written
    for (int s = 0, round = 0; row < a.rows; row += step, ++turn) {
        const float next = row_gates ? gate_of(row + step) : by;
        const int g = a.m == a.rows ? 0 : (int)row / a.m, t = (int)row - g * a.m;
        const ThreadsSum sum{room + (group * 2 + (turn & 1)) * 4 * 32, T / 32, i >> 5, 1 + group};
        whole &= warp_wait(bar0 + 8 * s, round & 1, &failed);  // (given up: on with what is there, the barriers count all)
        const int x = slots + s * slot_bytes + 8 * i * kXB, h = slots + s * slot_bytes + ring.x_bytes + 8 * i * kSB;
#pragma unroll
        for (int c = 0; c < C; ++c) shared8(smem + (on[c] ? x + c * 8 * T * kXB : 0), kX, v[c]);
        if (a.after.kind != SYMAR_NORM_NONE) normed(a.after, w0, b0, sum, 0);
        if (gate.there) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float f[8];
                shared8(smem + (on[c] ? gate.at + c * gate.step : 0), true, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= f[j];
            }
        } else if (ring.gate_bytes) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float f[8];
                shared8(smem + (on[c] ? x + ring.x_bytes + ring.old_bytes + c * 8 * T * kXB : 0), kX, f);
                open8(f, a.gate_act);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= a.scale * f[j];
            }
        } else if (by != 1.0f) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= by;
        }
        if (ring.old_bytes) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float f[8];
                shared8(smem + (on[c] ? h + c * 8 * T * kSB : 0), kStream, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = fmaf(a.residual_scale, f[j], v[c][j]);
            }
        }
        if (a.residual_out) {
            void *to = moved(a.residual_out, g * a.residual_out_group + t * a.residual_out_ld + 8 * i, kStream);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (on[c]) write8<true>(to, kStream, c * 8 * T, 0, n, v[c]);
        }
        if (a.out) {
            normed(a.before, w1, b1, sum, 2);
            void *to = moved(a.out, g * a.out_group + t * a.out_ld + 8 * i, kX);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (on[c]) write8<true>(to, kX, c * 8 * T, 0, n, v[c]);
        } else {
            asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(T) : "memory");
        }
        // all of the slot has been read before the row's last barrier
        if (i == 0 && whole) ask(row + (int64_t)ring.slots * step, s);
        if (++s == ring.slots) s = 0, ++round;
        by = next;
    }
    if (*static_cast<volatile int *>(&failed)) {
        // copies may still be on their way: give them time to end before the memory is let go
        for (int k = 0; k < 1000; ++k) __nanosleep(1000);
        if (i == 0 && a.status) atomicCAS(a.status, 0u, (unsigned)SYMAR_ERR_TIMEOUT);
    }
}

// How the ring divides shared memory; no group fits: T is 0.
Ring ring_of(const NormArgs &a)
{
    Ring r{};
    const int xw = a.x_wide ? 4 : 2;
    r.x_bytes = a.n * xw;
    r.old_bytes = a.residual ? a.n * (a.stream_wide ? 4 : 2) : 0;
    r.gate_bytes = a.gate && a.gate_step && (a.gate_ld != 0 || a.gate_group != 0) ? a.n * xw : 0;
    for (const Side *s : {&a.after, &a.before}) r.held += ((s->weight != nullptr) + (s->bias != nullptr)) * a.n * (s->wide ? 4 : 2);
    if (a.gate && a.gate_step && !r.gate_bytes) r.held += a.n * 4;
    if (r.held > kRingRoom) return r;
    const int threads = ((a.n + 31) / 32 + 31) / 32 * 32;
    for (int groups = kRingThreads / threads < kMaxGroups ? kRingThreads / threads : kMaxGroups; groups > 0; --groups) {
        const int slots = (kRingRoom - r.held) / (groups * (r.x_bytes + r.old_bytes + r.gate_bytes));
        if (slots < 2) continue;
        r.T = threads, r.groups = groups, r.slots = slots < kMaxSlots ? slots : kMaxSlots;
        break;
    }
    return r;
}
template <int L, int C, int U, bool kVec, bool kX, bool kStream>
cudaError_t launch_short(const NormArgs &a, const Device &d, cudaStream_t s)
{
    const int64_t blocks = ((int64_t)a.rows * L + kShortThreads * U - 1) / (kShortThreads * U), most = 8ll * d.sms;
    return launch_early(short_kernel<L, C, U, kVec, kX, kStream>, dim3((unsigned)(blocks < most ? blocks : most)), kShortThreads, 0, s, a);
}
template <bool kVec, bool kX, bool kStream>
cudaError_t launch(const NormArgs &a, const Device &d, cudaStream_t s)
{
    // Many long rows: more than what is resident at once of the row kernel (of 8192: 400 rows 12.5 us, in the ring 13.3; 800 rows 19.1 us, a row a block 25.8; of
    // 2048: 800 rows 6.8 and 6.0).  Many short ones: a block a row has idle threads, but is over sooner (1080 heads of 128 2.2 us, several a warp 2.9).
    const bool many = a.rows > 4 * d.sms;
    if (a.rows > 16 * d.sms && a.n <= (kVec ? 512 : 1024)) {
        if constexpr (kVec) {
            if (a.n <= 64) return launch_short<8, 1, 2, true, kX, kStream>(a, d, s);
            if (a.n <= 128) return launch_short<16, 1, 2, true, kX, kStream>(a, d, s);
            if (a.n <= 256) return launch_short<32, 1, 2, true, kX, kStream>(a, d, s);
            return launch_short<32, 2, 1, true, kX, kStream>(a, d, s);     // (16384 x 512, two norms and a gate: 20.4 us, in the ring 26.6)
        } else {
            return launch_short<32, 4, 1, false, kX, kStream>(a, d, s);
        }
    }
    // (16384 x 1024: 29.9 us, with a warp a row in registers 34.6)
    if (kVec && many && a.n > 512 && a.n <= kRingMost && (a.after.kind != SYMAR_NORM_NONE || a.before.kind != SYMAR_NORM_NONE)) {
        const Ring r = ring_of(a);
        if (r.T) {
            const int bytes = 32 + r.held + r.groups * r.slots * (r.x_bytes + r.old_bytes + r.gate_bytes);
            static std::atomic<uint64_t> allowed{0};
            const cudaError_t e = allow_shared((const void *)ring_kernel<kX, kStream>, kRingRoom + 32, d.id, allowed);
            return e != cudaSuccess ? e : launch_early(ring_kernel<kX, kStream>, dim3((unsigned)d.sms), (unsigned)(r.T * r.groups), (size_t)bytes, s, a, r);
        }
    }
    const dim3 rows((unsigned)a.rows);
    if constexpr (kVec) {
        // (of 16384, one row 6.0 us with sixteen elements a thread and 8.0 with thirty-two; 254 rows 14.7 and 12.9)
        const int chunks = a.n <= 8192 ? 1 : a.n <= 16384 && a.rows <= d.sms ? 2 : 4;
        const unsigned threads = (unsigned)(((a.n + 8 * chunks - 1) / (8 * chunks) + 31) / 32 * 32);
        if (chunks == 1) return launch_early(row_kernel<1, 0, kX, kStream>, rows, threads, 0, s, a);
        return chunks == 2 ? launch_early(row_kernel<2, 0, kX, kStream>, rows, threads, 0, s, a) : launch_early(row_kernel<4, 0, kX, kStream>, rows, threads, 0, s, a);
    } else {
        if (a.n <= 1024) return launch_early(row_kernel<1, 128, kX, kStream>, rows, 128, 0, s, a);
        // sixteen elements a thread, in as many warps as that takes (2049 in 160 threads 21.7 us, in 256 26.5)
        switch ((a.n + 511) / 512) {
            case 3: return launch_early(row_kernel<2, 96, kX, kStream>, rows, 96, 0, s, a);
            case 4: return launch_early(row_kernel<2, 128, kX, kStream>, rows, 128, 0, s, a);
            case 5: return launch_early(row_kernel<2, 160, kX, kStream>, rows, 160, 0, s, a);
            case 6: return launch_early(row_kernel<2, 192, kX, kStream>, rows, 192, 0, s, a);
            case 7: return launch_early(row_kernel<2, 224, kX, kStream>, rows, 224, 0, s, a);
            case 8: return launch_early(row_kernel<2, 256, kX, kStream>, rows, 256, 0, s, a);
        }
        if (a.n <= 8192) return launch_early(row_kernel<2, 512, kX, kStream>, rows, 512, 0, s, a);
        return launch_early(row_kernel<4, 1024, kX, kStream>, rows, 1024, 0, s, a);
    }
}
template <bool kVec>
cudaError_t launch_as(const NormArgs &a, const Device &d, cudaStream_t s)
{
    if (a.x_wide) return a.stream_wide ? launch<kVec, true, true>(a, d, s) : launch<kVec, true, false>(a, d, s);
    return a.stream_wide ? launch<kVec, false, true>(a, d, s) : launch<kVec, false, false>(a, d, s);
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
    if (p.gate_act < SYMAR_GATE_NONE || p.gate_act > SYMAR_GATE_TANH || p.gate_step < 0 || p.gate_step > 1 || (uintptr_t)p.status % 4) return SYMAR_ERR_INVAL;
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
    if (p.n > SYMAR_NORM_MAX || (int64_t)p.groups * p.m > 0x7fffffff) return SYMAR_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    auto clear = [&] {
        const cudaError_t e = p.status ? cudaMemsetAsync(p.status, 0, sizeof(unsigned), s) : cudaSuccess;
        return e == cudaSuccess ? (int)SYMAR_OK : cuda_fail(e, "cudaMemsetAsync");
    };
    if (p.groups == 0 || p.m == 0 || p.n == 0) return clear();
    if ((p.out == nullptr) != (p.before.kind == SYMAR_NORM_NONE)) return SYMAR_ERR_INVAL;
    if (!p.x || (!p.out && !p.residual_out)) return SYMAR_ERR_INVAL;
    if ((p.out && rows_meet(p.m, p.out_ld, p.groups, p.out_group, p.n)) ||
        (p.residual_out && rows_meet(p.m, p.residual_out_ld, p.groups, p.residual_out_group, p.n)) || (p.out && p.out == p.residual_out))
        return SYMAR_ERR_INVAL;
    NormArgs a{};
    a.x = p.x;  a.x_ld = p.x_ld;  a.x_group = p.x_group;
    a.residual = p.residual;  a.residual_ld = p.residual_ld;  a.residual_group = p.residual_group;
    a.residual_out = p.residual_out;  a.residual_out_ld = p.residual_out_ld;  a.residual_out_group = p.residual_out_group;
    a.out = p.out;  a.out_ld = p.out_ld;  a.out_group = p.out_group;
    a.gate = p.gate;  a.gate_ld = p.gate_ld;  a.gate_group = p.gate_group;  a.gate_step = p.gate_step;  a.gate_act = p.gate_act;
    a.after = side_of(p.after);  a.before = side_of(p.before);
    a.scale = p.scale;  a.residual_scale = p.residual_scale;
    a.m = p.m;  a.n = p.n;  a.rows = p.groups * p.m;
    a.x_wide = p.dtype == SYMAR_F32;  a.stream_wide = p.stream_dtype == SYMAR_F32;
    a.status = p.status;
    Device d;
    int rc = device_info(&d);
    if (rc == SYMAR_OK) rc = clear();
    if (rc != SYMAR_OK) return rc;
    const cudaError_t e = vec ? launch_as<true>(a, d, s) : launch_as<false>(a, d, s);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_norm");
}
