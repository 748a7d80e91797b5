// The driver's encoder of tensor maps, looked up at run time (the library does not link the driver).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

namespace eg {

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeFn encoder() {
    static std::atomic<EncodeFn> known{nullptr};          // several threads may look it up at once: they find the same
    EncodeFn fn = known.load(std::memory_order_relaxed);
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            return nullptr;
        fn = reinterpret_cast<EncodeFn>(p);
        known.store(fn, std::memory_order_relaxed);
    }
    return fn;
}

}  // namespace eg
