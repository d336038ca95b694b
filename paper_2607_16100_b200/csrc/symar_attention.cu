// Attention of new tokens over the paged 4-bit cache (formulas in include/symar.h).
#include <cmath>

#include "symar_ops.h"

namespace symar {
namespace {

constexpr int kThreads = 256;

struct AttnArgs {
    KvView  c;
    KvBatch b;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    int64_t q_ld, q_head, out_ld, out_head;
    float   scale_log2;         // scale * log2(e): softmax in powers of two
    int     q_heads, window;
    int    *status;
};

// One warp per (token, query head): the running maximum, sum and output of a softmax, one key at a time.
template <int D>
__global__ void __launch_bounds__(kThreads) attention_kernel(const AttnArgs a)
{
    constexpr int E = D / 32;                       // channels of a lane: c = lane * E ..
    const int lane = (int)threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * (kThreads / 32) + (int)threadIdx.x / 32;
    if (item >= (int64_t)a.b.tokens * a.q_heads) return;
    const int token = (int)(item / a.q_heads), head = (int)(item - (int64_t)token * a.q_heads);
    const int kvh = head / (a.q_heads / a.c.kv_heads);
    int seq = token, pos;
    if (a.b.token_start) {
        int lo = 0, hi = a.b.seqs;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (a.b.token_start[mid + 1] > token) hi = mid;
            else lo = mid + 1;
        }
        seq = lo;
        if (seq >= a.b.seqs) return;
        pos = a.b.lengths[seq] - (a.b.token_start[seq + 1] - token);
    } else {
        pos = a.b.lengths[seq] - 1;
    }
    float q[E], o[E] = {};
    for (int i = 0; i < E; ++i)
        q[i] = __bfloat162float(a.q[(int64_t)token * a.q_ld + (int64_t)head * a.q_head + lane * E + i]);
    float m = -INFINITY, l = 0.0f;
    const int ps = 1 << a.c.page_shift, grp = lane * E / 64;
    for (int j = a.window > 0 ? max(0, pos - a.window + 1) : 0; j <= pos; ++j) {
        const int page = kv_page_of(a.c, a.b, a.status, seq, j);
        if (page < 0) continue;
        const unsigned char *base = a.c.pages + page * a.c.page_bytes + kvh * a.c.head_bytes;
        const int row = j & (ps - 1);
        const uint32_t *words = reinterpret_cast<const uint32_t *>(base + ps * D);
        const uint32_t kw = words[row * (D / 64) + grp], vw = words[(ps + row) * (D / 64) + grp];
        float s = 0.0f, v[E];
        for (int i = 0; i < E; ++i) {
            const int c = lane * E + i;
            const int kn = base[row * (D / 2) + c / 2] >> (4 * (c & 1)) & 15, vn = base[(ps + row) * (D / 2) + c / 2] >> (4 * (c & 1)) & 15;
            s    = fmaf(q[i], kv_scale(kw) * (float)(kn - kv_zero(kw)), s);
            v[i] = kv_scale(vw) * (float)(vn - kv_zero(vw));
        }
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= a.scale_log2;
        const float top = fmaxf(m, s), keep = m == -INFINITY ? 0.0f : exp2f(m - top), p = exp2f(s - top);
        l = fmaf(l, keep, p);
        for (int i = 0; i < E; ++i) o[i] = fmaf(o[i], keep, p * v[i]);
        m = top;
    }
    const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
    for (int i = 0; i < E; ++i)
        a.out[(int64_t)token * a.out_ld + (int64_t)head * a.out_head + lane * E + i] = __float2bfloat16_rn(o[i] * inv);
}

}  // namespace
}  // namespace symar

using namespace symar;

extern "C" int symar_kv_attention(symar_kv_t *kv, const symar_kv_cache_t *cache, const symar_kv_batch_t *batch,
                                  const symar_kv_attention_t *args, void *cuda_stream)
{
    AttnArgs a;
    const int rc = kv_check(kv, cache, batch, &a.c, &a.b);
    if (rc != SYMAR_OK) return rc;
    if (!args || (args->dtype != SYMAR_F32 && args->dtype != SYMAR_BF16)) return SYMAR_ERR_INVAL;
    if (args->dtype != SYMAR_BF16) return SYMAR_ERR_UNSUPPORTED;
    if (args->q_heads < 1 || args->q_heads % cache->kv_heads || args->q_heads > 65536 || args->window < 0) return SYMAR_ERR_INVAL;
    if (!(args->scale >= 0.0f) || std::isinf(args->scale)) return SYMAR_ERR_INVAL;
    if (batch->tokens == 0) return SYMAR_OK;
    if (!args->q || !args->out || ((uintptr_t)args->q | (uintptr_t)args->out) % 2) return SYMAR_ERR_INVAL;
    a.q          = (const __nv_bfloat16 *)args->q;
    a.out        = (__nv_bfloat16 *)args->out;
    a.q_ld       = args->q_ld;
    a.q_head     = args->q_head;
    a.out_ld     = args->out_ld;
    a.out_head   = args->out_head;
    const double scale = args->scale == 0.0f ? 1.0 / std::sqrt((double)cache->head_dim) : (double)args->scale;
    a.scale_log2 = (float)(scale * 1.4426950408889634);
    a.q_heads    = args->q_heads;
    a.window     = args->window;
    a.status     = kv->status;
    const int64_t items = (int64_t)a.b.tokens * a.q_heads, blocks = (items + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffff) return SYMAR_ERR_UNSUPPORTED;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (a.c.dim == 64) attention_kernel<64><<<(unsigned)blocks, kThreads, 0, s>>>(a);
    else if (a.c.dim == 128) attention_kernel<128><<<(unsigned)blocks, kThreads, 0, s>>>(a);
    else attention_kernel<256><<<(unsigned)blocks, kThreads, 0, s>>>(a);
    cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SYMAR_OK : cuda_fail(e, "symar_kv_attention");
}
