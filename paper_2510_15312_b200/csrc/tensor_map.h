// The driver's tensor-map encoder, looked up once per process.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

namespace sdv {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_tiled_fn() {
    static std::atomic<EncodeTiledFn> fn{nullptr};   // the same for every thread and device
    EncodeTiledFn known = fn.load(std::memory_order_acquire);
    if (!known) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess) {
            known = (EncodeTiledFn)p;
            fn.store(known, std::memory_order_release);
        }
    }
    return known;
}

}  // namespace sdv
