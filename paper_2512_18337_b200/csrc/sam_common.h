// Shared by the translation units of the C ABI: the calling thread's last CUDA error, the launch count, device facts.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "sam.h"

namespace samb200 {

inline thread_local int g_last_cuda = 0;
inline std::atomic<long long> g_launches{0};   // kernels this library has enqueued (diagnostic)

inline int cuda_fail(cudaError_t e) {
    g_last_cuda = static_cast<int>(e);
    return SAM_ERR_CUDA;
}

#define SAM_CUDA(call)                                   \
    do {                                                 \
        cudaError_t e__ = (call);                        \
        if (e__ != cudaSuccess) return cuda_fail(e__);   \
    } while (0)

struct DeviceInfo {
    int sms = 0;
};

inline int device_info(DeviceInfo* out) {
    static thread_local int cached_dev = -1;
    static thread_local DeviceInfo cached;
    int dev = 0;
    SAM_CUDA(cudaGetDevice(&dev));
    if (dev != cached_dev) {
        int sms = 0;
        SAM_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        cached.sms = sms;
        cached_dev = dev;
    }
    *out = cached;
    return SAM_OK;
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace samb200
