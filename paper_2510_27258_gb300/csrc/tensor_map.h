// The driver's cuTensorMapEncodeTiled, without linking against the driver's library.
#pragma once

#include <atomic>

#include <cuda.h>
#include <cuda_runtime.h>

namespace hla {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Null where there is no driver.  Threads whose first calls come at once each look it up, and find the same.
inline EncodeTiledFn encode_fn() {
    static std::atomic<EncodeTiledFn> known{nullptr};
    EncodeTiledFn fn = known.load(std::memory_order_acquire);
    if (!fn) {
        cudaDriverEntryPointQueryResult qr;
        void *f = nullptr;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &qr) ==
                cudaSuccess &&
            qr == cudaDriverEntryPointSuccess) {
            fn = reinterpret_cast<EncodeTiledFn>(f);
            known.store(fn, std::memory_order_release);
        }
    }
    return fn;
}

}  // namespace hla
