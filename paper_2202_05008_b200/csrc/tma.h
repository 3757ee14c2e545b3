// The driver's encoder of tensor maps, looked up once.
#pragma once
#include <atomic>

#include <cuda.h>
#include <cuda_runtime.h>

namespace evo {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled tensor_map_encoder()
{
    static std::atomic<void*> known{ nullptr };
    void* f = known.load(std::memory_order_relaxed);
    if (!f) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
        known.store(f, std::memory_order_relaxed);
    }
    return reinterpret_cast<EncodeTiled>(f);
}

}  // namespace evo
