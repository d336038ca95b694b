// The paged 4-bit key/value cache: context, append with rotation, read-back, and the table of rotations.
// The formats and formulas are those stated in include/symar.h.
#include <cmath>
#include <cstring>
#include <new>

#include "symar_ops.h"

namespace symar {
namespace {

constexpr int kThreads   = 256;
constexpr int kMaxTokens = 16;      // tokens that one block of append or read takes

// ---- eight channels of a row, in binary32 ------------------------------------------
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> struct Eight;                 // eight channels as they lie in memory
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p, bool vec)
    {
        if (vec) a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        else a = make_float4(p[0], p[1], p[2], p[3]), b = make_float4(p[4], p[5], p[6], p[7]);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, bool vec)
    {
        if (vec) {
            a = *reinterpret_cast<const uint4 *>(p);
        } else {
            const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
            a = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
        }
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i]     = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
__device__ __forceinline__ void store8(float *p, bool vec, const float (&x)[8])
{
    if (vec) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = x[i];
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, bool vec, const float (&x)[8])
{
    if (vec) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<uint32_t *>(&h);
        }
        *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = __float2bfloat16_rn(x[i]);
    }
}

// ---- where a new token goes ---------------------------------------------------------
struct Place {
    int     seq, pos;       // pos < 0: an idle slot's token
    int64_t page;           // -1: nowhere
};

__device__ Place place_of(const KvView &c, const KvBatch &b, int *status, int token)
{
    Place p{token, -1, -1};
    if (b.token_start) {
        int lo = 0, hi = b.seqs;                      // first sequence whose tokens end beyond `token`
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (b.token_start[mid + 1] > token) hi = mid;
            else lo = mid + 1;
        }
        p.seq = lo;
        if (lo >= b.seqs || token < b.token_start[lo]) return p;      // a row of no sequence: behind the last, or before the first
        p.pos = b.lengths[lo] - (b.token_start[lo + 1] - token);
    } else {
        p.pos = b.lengths[token] - 1;
    }
    if (p.pos >= 0) p.page = kv_page_of(c, b, status, p.seq, p.pos);
    return p;
}

struct Rows {
    char   *p;
    int64_t ld, head;       // elements
    int     vec;            // 16-byte accesses allowed
};
struct AppendArgs {
    KvView  c;
    KvBatch b;
    Rows    q, qo, k, v;
    const float2 *table;
    int64_t table_rows;
    int     rot, interleaved, q_heads;
    int    *status;
    int     tokens_per_block;
    int     run;                 // query heads that a thread turns by the rotations it has loaded
    int     groups;              // of `run` query heads
    int     kv_blocks;           // blocks of the first kind (see append_kernel)
    uint32_t by_groups, by_heads;      // reciprocals: 2^32 / groups, 2^32 / (2 kv_heads), rounded up
};

// One unit is one head of one token: dim/8 lanes of a warp, eight channels each.  The channels that those of the half layout are
// turned with are read beside them (another lane of the warp reads them too), before any lane of the warp writes, so that q may be
// rotated in place.
__device__ __forceinline__ bool whole_chunk_pairs(int rot) { return (rot & 15) == 0; }
__device__ __forceinline__ int pair_of(int c0, int rot) { return c0 < (rot >> 1) ? c0 + (rot >> 1) : c0 - (rot >> 1); }
template <typename T>
__device__ __forceinline__ void rotate8(float (&x)[8], const Eight<T> &pair, const T *row, int c0, int rot, bool interleaved, const float2 *cs)
{
    if (c0 >= rot) return;
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ch = c0 + 2 * i;
            if (ch < rot) {
                const float2 t = __ldg(cs + (ch >> 1));
                const float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i]     = __fsub_rn(__fmul_rn(a, t.x), __fmul_rn(b, t.y));
                x[2 * i + 1] = __fadd_rn(__fmul_rn(b, t.x), __fmul_rn(a, t.y));
            }
        }
        return;
    }
    const int h = rot >> 1;
    float y[8];
    if (whole_chunk_pairs(rot)) {                      // the chunk lies in one half
        pair.get(y);
        const float4 *w = reinterpret_cast<const float4 *>(cs + (c0 < h ? c0 : c0 - h));
        const bool low = c0 < h;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float4 t;
            if (((uintptr_t)cs & 15) == 0) {
                t = __ldg(w + i);
            } else {
                const float2 u = __ldg(reinterpret_cast<const float2 *>(w + i)), v = __ldg(reinterpret_cast<const float2 *>(w + i) + 1);
                t = make_float4(u.x, u.y, v.x, v.y);
            }
            const float a0 = __fmul_rn(x[2 * i], t.x), b0 = __fmul_rn(y[2 * i], t.y);
            const float a1 = __fmul_rn(x[2 * i + 1], t.z), b1 = __fmul_rn(y[2 * i + 1], t.w);
            x[2 * i]     = low ? __fsub_rn(a0, b0) : __fadd_rn(a0, b0);
            x[2 * i + 1] = low ? __fsub_rn(a1, b1) : __fadd_rn(a1, b1);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int ch = c0 + i;
        y[i] = ch < rot ? to_f32(row[ch < h ? ch + h : ch - h]) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int ch = c0 + i;
        if (ch < rot) {
            const float2 t = __ldg(cs + (ch < h ? ch : ch - h));
            const float a = __fmul_rn(x[i], t.x), b = __fmul_rn(y[i], t.y);
            x[i] = ch < h ? __fsub_rn(a, b) : __fadd_rn(a, b);
        }
    }
}

// x rounded to a whole number, for |x| < 2^22: what lies below 1 in a sum with 1.5 * 2^23 is rounded away, ties to even
__device__ __forceinline__ float whole(float x) { return __fsub_rn(__fadd_rn(x, 12582912.0f), 12582912.0f); }

// Codes and word of a group of 64 channels held by eight neighbouring lanes.  Returns this lane's eight codes.
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t &word)
{
    float lo = 0.0f, hi = 0.0f, odd = 0.0f;            // odd: NaN once a value is not finite
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo  = fminf(lo, x[i]);
        hi  = fmaxf(hi, x[i]);
        odd = __fmaf_rn(x[i], 0.0f, odd);
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        lo  = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi  = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
        odd = __fadd_rn(odd, __shfl_xor_sync(0xffffffffu, odd, d));
    }
    const float fifteenth = 1.0f / 15.0f;
    const uint32_t bits = __float_as_uint(__fsub_rn(__fmul_rn(hi, fifteenth), __fmul_rn(lo, fifteenth))) & ~15u;
    const float s = __uint_as_float(bits);
    if (odd != odd) {
        word = 0x7fc00000u;
        return 0u;
    }
    if (!(s >= 1.17549435e-38f)) {
        word = 0u;
        return 0u;
    }
    const float inv = __fdiv_rn(1.0f, s);
    const float z   = whole(__fmul_rn(-lo, inv));
    word            = bits | (uint32_t)z;
    float half[2];                                     // four codes each: n0 + 16 n1 + 256 n2 + 4096 n3, exact
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 3; i >= 0; --i)
            sum = __fmaf_rn(sum, 16.0f, fminf(fmaxf(__fadd_rn(whole(__fmul_rn(x[4 * j + i], inv)), z), 0.0f), 15.0f));
        half[j] = __fadd_rn(sum, 8388608.0f);
    }
    return __byte_perm(__float_as_uint(half[0]), __float_as_uint(half[1]), 0x5410);
}

// n / d for n < 2^31 / d, by the reciprocal that the host rounded up
__device__ __forceinline__ int over(int n, uint32_t reciprocal) { return reciprocal ? (int)__umulhi((uint32_t)n, reciprocal) : n; }

// (a, b) turned by eight angles
__device__ __forceinline__ void turn8(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = a[i], y = b[i];
        a[i] = __fsub_rn(__fmul_rn(x, c[i]), __fmul_rn(y, s[i]));
        b[i] = __fadd_rn(__fmul_rn(y, c[i]), __fmul_rn(x, s[i]));
    }
}

// Queries of a block's tokens.  A thread has sixteen channels of `run` heads of one token: in the half layout eight and the eight
// that they are turned with, so that nothing is read twice and the eight rotations are loaded once for all its heads; in the interleaved
// layout sixteen neighbours.  Channels that are not turned go along in pairs of eights.
template <typename T>
__device__ __forceinline__ void queries(const AppendArgs &a, const Place *at, int first, int mine)
{
    const int lanes = a.c.dim / 16, shift = 31 - __clz(lanes), half = a.rot >> 4;      // half: threads of a head that turn something
    const int total = mine * a.groups * lanes;
    for (int u = (int)((blockIdx.y - (unsigned)a.kv_blocks) * kThreads + threadIdx.x); u < total; u += (int)(gridDim.y - (unsigned)a.kv_blocks) * kThreads) {
        const int j = u & (lanes - 1), tg = u >> shift, t = over(tg, a.by_groups), group = tg - t * a.groups;
        const Place p = at[t];
        const bool turn = a.table && p.pos >= 0 && p.pos < a.table_rows && j < half;
        const int c0 = a.interleaved ? 16 * j : (j < half ? 8 * j : a.rot + 16 * (j - half));
        const int c1 = a.interleaved || j >= half ? c0 + 8 : c0 + (a.rot >> 1);
        float cs[8], sn[8];
        if (turn) {
            const float4 *w = reinterpret_cast<const float4 *>(a.table + (int64_t)p.pos * (a.rot >> 1) + 8 * j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 v = __ldg(w + i);
                cs[2 * i] = v.x; sn[2 * i] = v.y; cs[2 * i + 1] = v.z; sn[2 * i + 1] = v.w;
            }
        }
        if (a.table && p.pos >= a.table_rows && j == 0 && group == 0) kv_record(a.status, p.seq, p.pos);
        const T *src = reinterpret_cast<const T *>(a.q.p) + (int64_t)(first + t) * a.q.ld + (int64_t)(group * a.run) * a.q.head;
        T *dst       = reinterpret_cast<T *>(a.qo.p) + (int64_t)(first + t) * a.qo.ld + (int64_t)(group * a.run) * a.qo.head;
        const int heads = min(a.run, a.q_heads - group * a.run);
        constexpr int kAhead = sizeof(T) == 2 ? 2 : 1;             // heads whose loads are on their way at a time
        for (int h0 = 0; h0 < heads; h0 += kAhead, src += kAhead * a.q.head, dst += kAhead * a.qo.head) {
            Eight<T> u[kAhead], v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (h0 + i < heads) u[i].load(src + i * a.q.head + c0, a.q.vec), v[i].load(src + i * a.q.head + c1, a.q.vec);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (h0 + i >= heads) break;
                float x[8], y[8];
                u[i].get(x);
                v[i].get(y);
                if (turn && !a.interleaved) {
                    turn8(x, y, cs, sn);
                } else if (turn) {
                    float e[8], o[8];                  // the pairs' first and second channels
#pragma unroll
                    for (int l = 0; l < 4; ++l) e[l] = x[2 * l], o[l] = x[2 * l + 1], e[l + 4] = y[2 * l], o[l + 4] = y[2 * l + 1];
                    turn8(e, o, cs, sn);
#pragma unroll
                    for (int l = 0; l < 4; ++l) x[2 * l] = e[l], x[2 * l + 1] = o[l], y[2 * l] = e[l + 4], y[2 * l + 1] = o[l + 4];
                }
                store8(dst + i * a.qo.head + c0, a.qo.vec, x);
                store8(dst + i * a.qo.head + c1, a.qo.vec, y);
            }
        }
    }
}

// Bound: bytes.  16384 tokens of 64 query and 2 x 8 key/value heads of 128 in bf16: 631 MB in 145 us, 4.4 TB/s (0.67 of the measured copy
// rate); keys and values alone take 60 us.  64 tokens 3.4 us, one token 2.6 us: the trip
// from the lengths to the page table to the page.  Ragged prompts of float32 (5 x up to 1501): 15.7 us.  Paired queries of bf16 spill 32 bytes at 64
// registers a thread, of float32 4.
// Blocks with the first kv_blocks indexes in y store keys and values, the others turn queries.  (Where the queries' pairs do not come in
// eights, kPaired is false and every block does both, a head of a token like another.)
// (four blocks per multiprocessor: measured against three and five, with one, two or four heads' loads ahead)
template <typename T, bool kPaired>
__global__ void __launch_bounds__(kThreads, 4) append_kernel(const AppendArgs a)
{
    wait_for_stream();
    __shared__ Place at[kMaxTokens];
    const int first = (int)blockIdx.x * a.tokens_per_block;
    const int mine  = min(a.tokens_per_block, a.b.tokens - first);
    if ((int)threadIdx.x < mine) at[threadIdx.x] = place_of(a.c, a.b, a.status, first + threadIdx.x);
    __syncthreads();
    if (kPaired && (int)blockIdx.y >= a.kv_blocks) {
        queries<T>(a, at, first, mine);
        return;
    }

    const int lanes = a.c.dim / 8, shift = 31 - __clz(lanes), per_pass = kThreads / lanes;
    const int q_heads = kPaired ? 0 : a.q_heads, heads = q_heads + 2 * a.c.kv_heads, units = mine * heads;
    const int lane  = (int)threadIdx.x & (lanes - 1), c0 = lane * 8;
    struct Unit {
        Eight<T> x, pair;
        const T *row;
        int t, h;                                      // t < 0: none
    };
    auto fetch = [&](int u) {
        Unit f;
        f.t = u < units ? over(u, a.by_heads) : -1;
        if (f.t >= 0) {
            f.h = u - f.t * heads;
            const bool is_q = f.h < q_heads, is_k = !is_q && f.h < q_heads + a.c.kv_heads;
            const Rows &r   = is_q ? a.q : (is_k ? a.k : a.v);
            f.row = reinterpret_cast<const T *>(r.p) + (int64_t)(first + f.t) * r.ld + (int64_t)(is_q ? f.h : f.h - q_heads - (is_k ? 0 : a.c.kv_heads)) * r.head;
            f.x.load(f.row + c0, r.vec);
            if ((is_q || is_k) && !a.interleaved && c0 < a.rot && whole_chunk_pairs(a.rot)) f.pair.load(f.row + pair_of(c0, a.rot), r.vec);
        }
        return f;
    };
    // every warp makes the same number of trips: the shuffles and the barrier below take whole warps
    const int step = (kPaired ? a.kv_blocks : (int)gridDim.y) * per_pass, mine_at = (int)threadIdx.x >> shift;
    Unit next = fetch((int)blockIdx.y * per_pass + mine_at);
    for (int u0 = (int)blockIdx.y * per_pass; u0 < units; u0 += step) {
        const Unit f = next;
        if (kPaired) next = fetch(u0 + step + mine_at);        // (q rotated in place: nothing of it is read ahead of a write)
        const bool on  = f.t >= 0, is_q = on && f.h < q_heads, is_k = on && !is_q && f.h < q_heads + a.c.kv_heads;
        const Place p  = at[on ? f.t : 0];
        float x[8] = {};
        if (on) {
            f.x.get(x);
            if ((is_q || is_k) && a.table && p.pos >= 0) {
                if (p.pos < a.table_rows) rotate8(x, f.pair, f.row, c0, a.rot, a.interleaved, a.table + (int64_t)p.pos * (a.rot >> 1));
                else if (lane == 0) kv_record(a.status, p.seq, p.pos);
            }
        }
        __syncwarp();
        if (is_q) store8(reinterpret_cast<T *>(a.qo.p) + (int64_t)(first + f.t) * a.qo.ld + (int64_t)f.h * a.qo.head + c0, a.qo.vec, x);
        uint32_t word, codes = quantise8(x, word);
        if (a.table && p.pos >= a.table_rows) word = 0x7fc00000u, codes = 0u;      // cannot be turned: NaN, not what the page held before
        if (on && !is_q && p.page >= 0) {
            const int hh = f.h - q_heads - (is_k ? 0 : a.c.kv_heads), ps = 1 << a.c.page_shift, row = (is_k ? 0 : ps) + (p.pos & (ps - 1));
            unsigned char *base = a.c.pages + p.page * a.c.page_bytes + hh * a.c.head_bytes;
            *reinterpret_cast<uint32_t *>(base + row * (a.c.dim / 2) + lane * 4) = codes;
            if ((lane & 7) == 0) reinterpret_cast<uint32_t *>(base + ps * a.c.dim)[row * a.c.groups + (lane >> 3)] = word;
        }
        if (!kPaired) next = fetch(u0 + step + mine_at);
    }
}

struct ReadArgs {
    KvView  c;
    KvBatch b;
    Rows    k, v;
    int    *status;
    int     tokens_per_block;
    uint32_t by_heads;
};

// Bytes: 16384 tokens 24.5 us for 86 MB, 3.5 TB/s (0.54 of the measured copy rate); bound by the loads in flight, of which a thread has four
// bytes of codes and a word at a time.  One token 1.8 us.
template <typename T>
__global__ void __launch_bounds__(kThreads) read_kernel(const ReadArgs a)
{
    wait_for_stream();
    __shared__ Place at[kMaxTokens];
    const int first = (int)blockIdx.x * a.tokens_per_block;
    const int mine  = min(a.tokens_per_block, a.b.tokens - first);
    if ((int)threadIdx.x < mine) at[threadIdx.x] = place_of(a.c, a.b, a.status, first + threadIdx.x);
    __syncthreads();

    const int lanes = a.c.dim / 8, shift = 31 - __clz(lanes), per_pass = kThreads / lanes;
    const int heads = 2 * a.c.kv_heads, units = mine * heads, ps = 1 << a.c.page_shift;
    const int lane  = (int)threadIdx.x & (lanes - 1);
    for (int u = (int)blockIdx.y * per_pass + ((int)threadIdx.x >> shift); u < units; u += (int)gridDim.y * per_pass) {
        const int  t = over(u, a.by_heads), h = u - t * heads;
        const bool is_k = h < a.c.kv_heads;
        const int  hh   = is_k ? h : h - a.c.kv_heads;
        const Rows &r   = is_k ? a.k : a.v;
        if (!r.p) continue;
        const Place p = at[t];
        float x[8] = {};
        if (p.page >= 0) {
            const int at_row = (is_k ? 0 : ps) + (p.pos & (ps - 1));
            const unsigned char *base = a.c.pages + p.page * a.c.page_bytes + hh * a.c.head_bytes;
            const uint32_t codes = *reinterpret_cast<const uint32_t *>(base + at_row * (a.c.dim / 2) + lane * 4);
            const uint32_t word  = reinterpret_cast<const uint32_t *>(base + ps * a.c.dim)[at_row * a.c.groups + (lane >> 3)];
            const float s = kv_scale(word);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __fmul_rn((float)((int)(codes >> (4 * i) & 15u) - kv_zero(word)), s);
        }
        store8(reinterpret_cast<T *>(r.p) + (int64_t)(first + t) * r.ld + (int64_t)hh * r.head + lane * 8, r.vec, x);
    }
}

struct TableArgs {
    float2 *table;
    int64_t rows;
    int     half, kind;
    double  log2_base, inv_factor, original, low, high, magnitude;
};

// Bound: binary64 arithmetic (exp2, sincos).  131072 positions of 128 channels 65 us, by parts 82 (67 MB, 1.0 TB/s); 4096 positions 3.8 and 4.3 us.
__global__ void __launch_bounds__(kThreads) table_kernel(const TableArgs a)
{
    const int64_t n = a.rows * a.half;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / a.half;
        const int pair    = (int)(i - row * a.half);
        double f = exp2(-a.log2_base * pair / a.half);
        if (a.kind == SYMAR_ROPE_LINEAR) {
            f *= a.inv_factor;
        } else if (a.kind == SYMAR_ROPE_BY_PARTS) {
            const double turns = a.original * f / 6.283185307179586476925287;
            const double g = fmin(fmax((turns - a.low) / (a.high - a.low), 0.0), 1.0);
            f = (1.0 - g) * f * a.inv_factor + g * f;
        }
        double s, c;
        sincos((double)row * f, &s, &c);
        a.table[i] = make_float2((float)(c * a.magnitude), (float)(s * a.magnitude));
    }
}

bool make_rows(Rows *r, const void *p, int64_t ld, int64_t head, int dtype)
{
    const int64_t vec = dtype == SYMAR_F32 ? 4 : 8;
    if ((uintptr_t)p % (dtype == SYMAR_F32 ? 4 : 2) || ld < 0 || head < 0) return false;
    r->p    = (char *)const_cast<void *>(p);
    r->ld   = ld;
    r->head = head;
    r->vec  = (uintptr_t)p % 16 == 0 && ld % vec == 0 && head % vec == 0;
    return true;
}

// 2^32 / d rounded up (0 stands for 1): n * that / 2^32 is n / d while n d < 2^32
uint32_t reciprocal(int d) { return d <= 1 ? 0u : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d); }

// Blocks of append and read.  Finding a block's tokens takes two or three trips to memory, so a block takes as many tokens as still leave
// every multiprocessor eight blocks (sixteen at most), and a thread about four units of them where there are many.
dim3 token_grid(int tokens, int heads, int lanes, int num_sms, int *tokens_per_block)
{
    int tpb = 1;
    while (tpb < kMaxTokens && tokens / (2 * tpb) >= 8 * num_sms) tpb *= 2;
    *tokens_per_block = tpb;
    const int per_pass = kThreads / lanes, passes = (tpb * heads + per_pass - 1) / per_pass, deep = tpb >= 4 ? 4 : 1;
    return dim3((unsigned)((tokens + tpb - 1) / tpb), (unsigned)((passes + deep - 1) / deep), 1);
}

}  // namespace

int kv_check(const symar_kv_t *kv, const symar_kv_cache_t *cache, const symar_kv_batch_t *batch, KvView *c, KvBatch *b)
{
    if (!kv || !cache || !batch) return SYMAR_ERR_INVAL;
    if (!symar_kv_page_bytes(cache->kv_heads, cache->head_dim, cache->page_size)) return SYMAR_ERR_UNSUPPORTED;
    if (!cache->pages || (uintptr_t)cache->pages % 16 || cache->num_pages < 1) return SYMAR_ERR_INVAL;
    if (batch->seqs < 0 || batch->tokens < 0 || batch->table_ld < 0 || batch->table_ld >= 1ll << 48) return SYMAR_ERR_INVAL;
    if (batch->seqs > SYMAR_KV_MAX_SEQS || batch->tokens > 0x7fffff00) return SYMAR_ERR_UNSUPPORTED;      // (a block's last token stays below 2^31)
    if (batch->tokens > 0) {
        if (!batch->lengths || !batch->page_table || batch->seqs == 0) return SYMAR_ERR_INVAL;
        if (((uintptr_t)batch->lengths | (uintptr_t)batch->page_table | (uintptr_t)batch->token_start) % 4) return SYMAR_ERR_INVAL;
        if (!batch->token_start && batch->tokens != batch->seqs) return SYMAR_ERR_INVAL;
    }
    c->pages      = (unsigned char *)cache->pages;
    c->num_pages  = cache->num_pages;
    c->kv_heads   = cache->kv_heads;
    c->dim        = cache->head_dim;
    c->groups     = cache->head_dim / 64;
    c->page_shift = 4;
    while ((1 << c->page_shift) < cache->page_size) ++c->page_shift;
    c->head_bytes = kv_head_bytes(cache->head_dim, cache->page_size);
    c->page_bytes = c->head_bytes * cache->kv_heads;
    *b = KvBatch{batch->lengths, batch->token_start, batch->page_table, batch->table_ld, batch->seqs, batch->tokens};
    return SYMAR_OK;
}

}  // namespace symar

using namespace symar;

extern "C" {

size_t symar_kv_page_bytes(int kv_heads, int head_dim, int page_size)
{
    if (kv_heads < 1 || kv_heads > 4096 || (head_dim != 64 && head_dim != 128 && head_dim != 256)) return 0;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1))) return 0;
    return (size_t)kv_heads * (size_t)kv_head_bytes(head_dim, page_size);
}

size_t symar_kv_required_bytes(void)
{
    return kKvPartOff + (size_t)2 * kAttnMaxBlocks * kAttnMaxRows * (kAttnMaxDim + 2) * sizeof(float);
}

int symar_kv_create_on(symar_kv_t **kv, void *device_mem, size_t device_bytes)
{
    if (!kv || !device_mem || (uintptr_t)device_mem % 256) return SYMAR_ERR_INVAL;
    if (device_bytes < symar_kv_required_bytes()) return SYMAR_ERR_NOMEM;
    symar_kv *h = new (std::nothrow) symar_kv;
    if (!h) return SYMAR_ERR_NOMEM;
    h->mem      = (char *)device_mem;
    h->status   = (int *)h->mem;
    h->counters = (unsigned *)(h->mem + kKvCtrOff);
    h->partials = (float *)(h->mem + kKvPartOff);
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device);
    if (e == cudaSuccess) e = cudaMemset(h->mem, 0, kKvPartOff);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        delete h;
        return cuda_fail(e, "symar_kv_create");
    }
    *kv = h;
    return SYMAR_OK;
}

int symar_kv_create(symar_kv_t **kv)
{
    if (!kv) return SYMAR_ERR_INVAL;
    void *p = nullptr;
    cudaError_t e = cudaMalloc(&p, symar_kv_required_bytes());
    if (e == cudaErrorMemoryAllocation) {
        (void)cudaGetLastError();
        return SYMAR_ERR_NOMEM;
    }
    if (e != cudaSuccess) return cuda_fail(e, "cudaMalloc");
    const int rc = symar_kv_create_on(kv, p, symar_kv_required_bytes());
    if (rc != SYMAR_OK) (void)cudaFree(p);
    else (*kv)->owns = true;
    return rc;
}

int symar_kv_destroy(symar_kv_t *kv)
{
    if (!kv) return SYMAR_ERR_INVAL;
    int rc = SYMAR_OK;
    if (kv->owns) {
        cudaError_t e = cudaFree(kv->mem);
        if (e != cudaSuccess) rc = cuda_fail(e, "cudaFree");
    }
    delete kv;
    return rc;
}

int symar_kv_reset(symar_kv_t *kv, void *cuda_stream)
{
    if (!kv) return SYMAR_ERR_INVAL;
    cudaError_t e = cudaMemsetAsync(kv->mem, 0, kKvPartOff, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "cudaMemsetAsync");
}

int symar_kv_status(symar_kv_t *kv, int *code, int *seq, int *position)
{
    if (!kv) return SYMAR_ERR_INVAL;
    int w[3] = {0, 0, 0};
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(w, kv->status, sizeof w, cudaMemcpyDeviceToHost);
    if (e != cudaSuccess) return cuda_fail(e, "symar_kv_status");
    if (code) *code = w[0];
    if (seq) *seq = w[1];
    if (position) *position = w[2];
    return SYMAR_OK;
}

int symar_rope_table(void *table, int64_t rows, const symar_rope_scaling_t *s, void *cuda_stream)
{
    if (!s || rows < 0 || rows >= 1ll << 48 || s->rot_dim < 2 || s->rot_dim % 2 || s->rot_dim > 256) return SYMAR_ERR_INVAL;
    if (!(s->base > 0.0) || s->kind < SYMAR_ROPE_PLAIN || s->kind > SYMAR_ROPE_BY_PARTS) return SYMAR_ERR_INVAL;
    if (s->kind != SYMAR_ROPE_PLAIN && (!(s->factor > 0.0) || !std::isfinite(s->factor))) return SYMAR_ERR_INVAL;
    if (s->kind == SYMAR_ROPE_BASE && s->rot_dim < 4) return SYMAR_ERR_INVAL;
    if (s->kind == SYMAR_ROPE_BY_PARTS && (!(s->original > 0.0) || !(s->high > s->low))) return SYMAR_ERR_INVAL;
    const double base = s->kind == SYMAR_ROPE_BASE ? s->base * std::pow(s->factor, (double)s->rot_dim / (s->rot_dim - 2)) : s->base;
    const double inv_factor = s->kind == SYMAR_ROPE_PLAIN ? 1.0 : 1.0 / s->factor;
    // (an infinite base has no f_0, and infinite ends have no place between them)
    if (!(base > 0.0) || !std::isfinite(base) || !std::isfinite(inv_factor) || !std::isfinite(s->magnitude)) return SYMAR_ERR_INVAL;
    if (s->kind == SYMAR_ROPE_BY_PARTS && (!std::isfinite(s->original) || !std::isfinite(s->high - s->low))) return SYMAR_ERR_INVAL;
    if (rows == 0) return SYMAR_OK;
    if (!table || (uintptr_t)table % 8) return SYMAR_ERR_INVAL;
    TableArgs a;
    a.table      = (float2 *)table;
    a.rows       = rows;
    a.half       = s->rot_dim / 2;
    a.kind       = s->kind;
    a.inv_factor = inv_factor;
    a.log2_base  = std::log2(base);
    a.original   = s->original;
    a.low        = s->low;
    a.high       = s->high;
    a.magnitude  = s->magnitude == 0.0 ? 1.0 : s->magnitude;
    const int64_t blocks = (rows * a.half + kThreads - 1) / kThreads;
    table_kernel<<<(unsigned)(blocks < 16384 ? blocks : 16384), kThreads, 0, (cudaStream_t)cuda_stream>>>(a);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_rope_table");
}

int symar_kv_append(symar_kv_t *kv, const symar_kv_cache_t *cache, const symar_kv_batch_t *batch,
                    const symar_kv_append_t *args, void *cuda_stream)
{
    AppendArgs a;
    const int rc = kv_check(kv, cache, batch, &a.c, &a.b);
    if (rc != SYMAR_OK) return rc;
    if (!args || (args->dtype != SYMAR_F32 && args->dtype != SYMAR_BF16)) return SYMAR_ERR_INVAL;
    if (args->q_heads > 4096) return SYMAR_ERR_UNSUPPORTED;
    if (args->q_heads < 0 || (args->interleaved != 0 && args->interleaved != 1)) return SYMAR_ERR_INVAL;
    if (args->rotations && (args->rot_dim < 2 || args->rot_dim % 2 || args->rot_dim > cache->head_dim || args->rotation_rows < 0 ||
                            (uintptr_t)args->rotations % 8))
        return SYMAR_ERR_INVAL;
    if (batch->tokens == 0) return SYMAR_OK;
    a.q_heads = args->q ? args->q_heads : 0;
    if (!args->k || !args->v || (a.q_heads > 0 && !args->q_out)) return SYMAR_ERR_INVAL;
    if (!make_rows(&a.q, args->q, args->q_ld, args->q_head, args->dtype) ||
        !make_rows(&a.qo, args->q_out, args->q_out_ld, args->q_out_head, args->dtype) ||
        !make_rows(&a.k, args->k, args->k_ld, args->k_head, args->dtype) ||
        !make_rows(&a.v, args->v, args->v_ld, args->v_head, args->dtype) ||
        (a.q_heads > 0 && rows_meet(batch->tokens, args->q_out_ld, a.q_heads, args->q_out_head, a.c.dim)))
        return SYMAR_ERR_INVAL;
    a.table       = (const float2 *)args->rotations;
    a.table_rows  = args->rotation_rows;
    a.rot         = args->rotations ? args->rot_dim : 0;
    a.interleaved = args->interleaved;
    a.status      = kv->status;
    // queries by pairs of eights where their rotated part and its halves come in eights and the table's rows on 16 bytes
    const bool paired = a.q_heads > 0 && a.rot % 16 == 0 && (uintptr_t)a.table % 16 == 0;
    const int kv_heads = (paired || a.q_heads == 0 ? 0 : a.q_heads) + 2 * a.c.kv_heads;
    dim3 grid = token_grid(batch->tokens, kv_heads, a.c.dim / 8, kv->num_sms, &a.tokens_per_block);
    a.by_heads  = reciprocal(kv_heads);
    a.kv_blocks = (int)grid.y;
    a.run = a.groups = 1;
    a.by_groups = 0;
    if (paired) {
        // a run of heads per thread once there are more than a few waves of threads without it
        const int64_t threads = (int64_t)batch->tokens * a.q_heads * (a.c.dim / 16);
        a.run = 1;
        while (a.run < 8 && a.run < a.q_heads && threads / (2 * a.run) >= 4096ll * kv->num_sms) a.run *= 2;
        a.groups    = (a.q_heads + a.run - 1) / a.run;
        a.by_groups = reciprocal(a.groups);
        const int64_t per_block = (int64_t)a.tokens_per_block * a.groups * (a.c.dim / 16);
        grid.y += (unsigned)((per_block + kThreads - 1) / kThreads);
    }
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (args->dtype == SYMAR_F32) {
        if (paired) e = launch_early(append_kernel<float, true>, grid, kThreads, 0, s, a);
        else e = launch_early(append_kernel<float, false>, grid, kThreads, 0, s, a);
    } else {
        if (paired) e = launch_early(append_kernel<__nv_bfloat16, true>, grid, kThreads, 0, s, a);
        else e = launch_early(append_kernel<__nv_bfloat16, false>, grid, kThreads, 0, s, a);
    }
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_kv_append");
}

int symar_kv_read(symar_kv_t *kv, const symar_kv_cache_t *cache, const symar_kv_batch_t *batch, const symar_kv_read_t *args,
                  void *cuda_stream)
{
    ReadArgs a;
    const int rc = kv_check(kv, cache, batch, &a.c, &a.b);
    if (rc != SYMAR_OK) return rc;
    if (!args || (args->dtype != SYMAR_F32 && args->dtype != SYMAR_BF16)) return SYMAR_ERR_INVAL;
    if (batch->tokens == 0 || (!args->k && !args->v)) return SYMAR_OK;
    if (!make_rows(&a.k, args->k, args->k_ld, args->k_head, args->dtype) ||
        !make_rows(&a.v, args->v, args->v_ld, args->v_head, args->dtype) ||
        (args->k && rows_meet(batch->tokens, args->k_ld, a.c.kv_heads, args->k_head, a.c.dim)) ||
        (args->v && rows_meet(batch->tokens, args->v_ld, a.c.kv_heads, args->v_head, a.c.dim)))
        return SYMAR_ERR_INVAL;
    a.status = kv->status;
    a.by_heads = reciprocal(2 * a.c.kv_heads);
    const dim3 grid = token_grid(batch->tokens, 2 * a.c.kv_heads, a.c.dim / 8, kv->num_sms, &a.tokens_per_block);
    cudaError_t e;
    if (args->dtype == SYMAR_F32) e = launch_early(read_kernel<float>, grid, kThreads, 0, (cudaStream_t)cuda_stream, a);
    else e = launch_early(read_kernel<__nv_bfloat16>, grid, kThreads, 0, (cudaStream_t)cuda_stream, a);
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_kv_read");
}

}  // extern "C"
