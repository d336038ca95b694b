// Barriers in shared memory, the copy engine and the fifth generation's tensor cores, as the operators' kernels use them.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace symar {

constexpr uint64_t kWaitNs = 4000000000ull;       // longest wait of a kernel for its own copies and products

// ---- instructions -----------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_if(uint32_t bar, bool on)      // (no branch)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"((int)on) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// A thread's wait; false once it has lasted four seconds or another role has given up.
__device__ __forceinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int *failed)
{
    const uint64_t t0 = now_ns();
    for (;;) {
        for (int i = 0; i < 256; ++i)
            if (bar_try(bar, parity)) return true;
        if (*failed || now_ns() - t0 > kWaitNs) {
            *failed = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *failed)
{
    bool ok = false;
#pragma unroll 1
    for (int i = 0; i < 64 && !ok; ++i) ok = bar_try(bar, parity);
    if (!ok) ok = bar_wait_long(bar, parity, failed);
    return ok;
}
// The same for a whole warp: all its lanes go on, or none.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *failed)
{
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
        if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
    const uint64_t t0 = now_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 256; ++i)
            if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
        if (__any_sync(0xffffffffu, *failed || now_ns() - t0 > kWaitNs)) {
            *failed = 1;
            return false;
        }
    }
}
// one lane of a converged warp
__device__ __forceinline__ bool elected()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// shared-memory operand: rows of 128 bytes, swizzled in blocks of eight
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void product(uint32_t acc, uint64_t a, uint64_t b, uint32_t how, uint32_t add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(acc),
                 "l"(a), "l"(b), "r"(how), "r"(add) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// sixteen columns of this warp's 32 lanes; the wait is the caller's
__device__ __forceinline__ void acc_load16(uint32_t addr, float *v)
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

}  // namespace symar
