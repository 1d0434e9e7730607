// Shared by the temporal head's operators.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

typedef CUresult (*SrEncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
SrEncodeTiled sr_encode_tiled();                      // the driver's cuTensorMapEncodeTiled; null: there is none
int sr_device_sms();                                  // SMs of the current device; 0: no device
int* sr_operator_error_word();                        // set to 1 by a kernel of the current device whose bounded wait expired; null: no device

// A kernel's limit of dynamic shared memory, raised once per device.
struct SrSharedLimit {
    std::atomic<uint64_t> done{0};
    template <typename K>
    cudaError_t raise(K* kernel, int bytes)
    {
        int dev = 0;
        const cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
        if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
        const cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (r == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
        return r;
    }
};
