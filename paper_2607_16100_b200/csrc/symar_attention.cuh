// Attention over the paged 4-bit cache: what its two kernels share.
#pragma once
#include "symar_ops.h"
#include "symar_tc.cuh"

namespace symar {

struct AttnArgs {
    KvView  c;
    KvBatch b;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    int64_t q_ld, q_head, out_ld, out_head;
    float   scale_log2;         // scale * log2(e): softmax in powers of two
    float   scale_code;         // the same times 2^69: what a product with codes lacks
    int     q_heads, share, window, q_vec, out_vec;
    uint32_t share_mul, share_shift;
    int    *status;
    unsigned *counters;
    float  *partials;
};

// ---- instructions -----------------------------------------------------------------------
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool on)
{
    const int n = on ? 16 : 0;         // 0: the 16 bytes become zeros and nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void matrices(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void matrices_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&h);
}
// A code n in bits 0-3 or 4-7 of a bf16 whose other bits are 0 is the number n 2^-133 or n 2^-129: the smallest numbers are evenly
// spaced.  So one AND makes two of them of a word (channels i and i + 4 of eight, 4 bits apart in i), and both the matrix instruction and
// fused multiply-add take them exactly (tested for every n and z).  The keys go into the product like that, against queries times
// 2^64 (2^60 for the second kind); the values are brought to (n - z) / 64 and (n - z) / 4 first, whose factors the result loses at the end.
__device__ __forceinline__ uint32_t codes(uint32_t w, int i) { return (i & 2 ? w >> 8 : w) & (i & 1 ? 0x00f000f0u : 0x000f000fu); }
__device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
constexpr uint32_t kTwo127 = 0x7f007f00u, kMinusTwo127 = 0xff00ff00u, kTwo64 = 0x5f805f80u, kTwo60 = 0x5d805d80u, kSixteen = 0x41804180u;
// a token's words
template <int N> __device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint32_t *p)
{
    if (N == 1) {
        w[0] = p[0];
    } else if (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        w[0] = v.x; w[N - 1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p + i);
            w[i] = v.x; w[(i + 1) % N] = v.y; w[(i + 2) % N] = v.z; w[(i + 3) % N] = v.w;
        }
    }
}
// -z / 64 of two words' zero points
__device__ __forceinline__ uint32_t zeros_of(uint32_t w0, uint32_t w1) { return mul2(__byte_perm(w0, w1, 0x5410) & 0x000f000fu, kMinusTwo127); }

static __device__ __noinline__ int64_t quotient(int64_t a, int64_t b)         // of what is hardly ever above 32 bits
{
    return ((uint64_t)a | (uint64_t)b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// n / share for 0 <= n < 2^31, by the reciprocal that the host rounded up
__device__ __forceinline__ int by_share(const AttnArgs &a, int n) { return (int)((uint64_t)(uint32_t)n * a.share_mul >> a.share_shift); }

// ---- the sequences as work ----------------------------------------------------------------
// An item is `rows` query rows (a token and a head of the key/value head's share, tokens first) of one sequence and one
// key/value head; its work is the chunks of 16 cached tokens that any of its rows sees, one at least.
struct Seq {
    int start, fresh, len;       // first row of q, new tokens, all tokens up to the last of them
};
__device__ __forceinline__ Seq sequence(const AttnArgs &a, int b)
{
    Seq s;
    s.len = a.b.lengths[b];
    if (a.b.token_start) {
        const int end = a.b.token_start[b + 1], last = min(end, a.b.tokens);
        s.start = max(a.b.token_start[b], 0);
        s.fresh = max(last - s.start, 0);
        s.len -= end - last;               // rows that the call does not have are tokens that none of its rows sees
    } else {
        s.start = b;
        s.fresh = 1;
    }
    return s;
}
struct Item {
    int lo, chunks;              // first token (a multiple of 16), chunks of 16 tokens
};
template <int R>
__device__ __forceinline__ Item item_of(const AttnArgs &a, const Seq &s, int block)
{
    const int first = by_share(a, block * R), last = min(by_share(a, block * R + R - 1), s.fresh - 1);
    const int64_t most = a.b.table_ld << a.c.page_shift;           // tokens that the table has room for
    int hi = s.len - s.fresh + last + 1;
    if (hi > most) hi = (int)most;
    int lo = a.window > 0 ? max(s.len - s.fresh + first + 1 - a.window, 0) : 0;
    lo &= ~15;
    return Item{lo, max((hi - lo + 15) >> 4, 1)};
}
// Four channels of a row's output, divided by the row's sum (0 where nothing was seen).
__device__ __forceinline__ void store4(const AttnArgs &a, const Seq &s, int rows, int r, int head, int d, float4 v, float sum)
{
    if (r >= rows) return;
    const int tok = by_share(a, r), hh = r - tok * a.share;
    const float f = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);
    __nv_bfloat16 *p = a.out + (int64_t)(s.start + tok) * a.out_ld + (int64_t)(head * a.share + hh) * a.out_head + d;
    const uint32_t x = pack_bf16(v.x * f, v.y * f), y = pack_bf16(v.z * f, v.w * f);
    if (a.out_vec) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(x, y);
    } else {
        uint16_t *h = reinterpret_cast<uint16_t *>(p);
        h[0] = (uint16_t)x; h[1] = (uint16_t)(x >> 16); h[2] = (uint16_t)y; h[3] = (uint16_t)(y >> 16);
    }
}

// Rows before token_start[0] and from token_start[seqs] on are no sequence's: zeros, by the first `threads` threads of `blocks` blocks, of
// which this one is `at`.  Blocks do this after their own work, or have no other (before it, it cost every call 1 to 2%, one without such rows too).
__device__ __forceinline__ void zero_other_rows(const AttnArgs &a, int at, int blocks, int threads)
{
    if (!a.b.token_start) return;
    const int first = min(max(a.b.token_start[0], 0), a.b.tokens), end = max(min(a.b.token_start[a.b.seqs], a.b.tokens), first);
    const int shift = 29 - __clz(a.c.dim);                     // 2^shift pieces of four channels
#pragma unroll 1
    for (int i = at; i < first + (a.b.tokens - end); i += blocks) {
        __nv_bfloat16 *row = a.out + (int64_t)(i < first ? i : i - first + end) * a.out_ld;
#pragma unroll 1
        for (int e = threadIdx.x; e < a.q_heads << shift; e += threads) {
            __nv_bfloat16 *p = row + (int64_t)(e >> shift) * a.out_head + ((e & ((1 << shift) - 1)) << 2);
            if (a.out_vec) {
                *reinterpret_cast<uint2 *>(p) = make_uint2(0, 0);
            } else {
                uint16_t *h = reinterpret_cast<uint16_t *>(p);
                h[0] = h[1] = h[2] = h[3] = 0;
            }
        }
    }
}

// One softmax over all work of an item, wherever it was done: unnormalised output relative to 2^m, and its sum.
constexpr float kNothing = -3.402823466e38f;

// Prompts: many query rows of a sequence (symar_prompt.cu).  False: not for this kernel.
bool prompt_attention_takes(const AttnArgs &a, int num_sms, int device);
cudaError_t launch_prompt_attention(const AttnArgs &a, int device, cudaStream_t stream);

}  // namespace symar
