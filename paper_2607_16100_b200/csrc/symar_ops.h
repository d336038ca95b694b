// Shared by the operators around the AllReduces (symar_linear.cu, symar_kv.cu, symar_attention.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "symar.h"
#include "symar_internal.h"
#include "symar_rows.h"

// The context of the cache operators (owned by symar_kv.cu).
struct symar_kv {
    char *mem      = nullptr;     // [status block][counters][partial results]
    bool  owns     = false;
    int   device   = 0;
    int   num_sms  = 0;
    int  *status   = nullptr;     // device: {code, seq, position}
    unsigned *counters = nullptr; // device: one per block of the attention grid
    float *partials = nullptr;    // device
};

namespace symar {

// ---- sizes of the attention grid that the context has room for ----
constexpr int kAttnMaxBlocks = 256;      // blocks of the largest attention grid
constexpr int kAttnMaxRows   = 16;        // query rows of a block
constexpr int kAttnMaxDim    = 256;

constexpr size_t kKvCtrOff  = 256;
constexpr size_t kKvPartOff = kKvCtrOff + (size_t)kAttnMaxBlocks * sizeof(unsigned);

// ---- the paged 4-bit cache as kernels see it ----
struct KvView {
    unsigned char *pages;
    int64_t        num_pages;
    int            kv_heads, dim, page_shift, groups;      // groups of 64 channels per token
    int64_t        head_bytes, page_bytes;
};
struct KvBatch {
    const int32_t *lengths, *token_start, *page_table;
    int64_t        table_ld;
    int            seqs, tokens;
};

__host__ __device__ __forceinline__ int64_t kv_head_bytes(int dim, int page) { return (int64_t)page * dim + 8ll * page * (dim / 64); }

#ifdef __CUDACC__
// The four lowest bits of a word are the zero point, the rest is the scale.
__device__ __forceinline__ float kv_scale(uint32_t w) { return __uint_as_float(w & ~15u); }
__device__ __forceinline__ int kv_zero(uint32_t w) { return (int)(w & 15u); }

// First offence of a call is kept: code last, so that a reader that sees it sees where.
static __device__ __noinline__ void kv_record(int *status, int seq, int position)
{
    if (atomicCAS(status + 3, 0, 1) == 0) {
        status[1] = seq;
        status[2] = position;
        __threadfence();
        atomicExch(status, SYMAR_ERR_INVAL);
    }
}

// Page of position `pos` of sequence `seq`, or -1 (recorded) where the table or the pool has none.
__device__ __forceinline__ int kv_page_of(const KvView &c, const KvBatch &b, int *status, int seq, int pos)
{
    const int col  = pos >> c.page_shift;
    const int page = col < b.table_ld ? b.page_table[(int64_t)seq * b.table_ld + col] : -1;
    if (page >= 0 && page < c.num_pages) return page;
    kv_record(status, seq, pos);
    return -1;
}
#endif

// The operators are launched before the kernel ahead of them on the stream has drained, and wait for its results here, before they read
// or write anything; from then on the next kernel may be launched in the same way.
#ifdef __CUDACC__
__device__ __forceinline__ void wait_for_stream()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
template <typename... P, typename... A>
cudaError_t launch_early(void (*fn)(P...), dim3 grid, unsigned threads, size_t shared, cudaStream_t stream, A... args)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fn, args...);
}
#endif

// Dynamic shared memory of a kernel, allowed once per device (`done`: a bit per device, one word per kernel).
inline cudaError_t allow_shared(const void *fn, int bytes, int device, std::atomic<uint64_t> &done)
{
    const uint64_t bit = device >= 0 && device < 64 ? 1ull << device : 0;
    if (bit && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Argument checks shared by the calls on a cache; fills the views.
int kv_check(const symar_kv_t *kv, const symar_kv_cache_t *cache, const symar_kv_batch_t *batch, KvView *c, KvBatch *b);

}  // namespace symar
