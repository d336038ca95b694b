// What the host asks once: the driver's encoder of tensor maps, and how many multiprocessors a device has.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "symar.h"
#include "symar_internal.h"

namespace symar {

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                              CUtensorMapFloatOOBfill);
inline EncodeFn encoder()
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

struct Device {
    int sms = 0, id = -1;
};
inline int device_info(Device *d)
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

}  // namespace symar
