// Waits that end: what the attention kernels poll, and how often.  No CUDA in here, so that the host can run it too.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define SAM_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define SAM_HOST_DEVICE inline
#endif

namespace samb200 {

constexpr uint32_t kCachePolls = 1u << 20;

// False when ready() did not come true in time.
template <typename Ready>
SAM_HOST_DEVICE bool poll(Ready ready) {
    for (uint32_t i = 0; i < kCachePolls; ++i)
        if (ready()) return true;
    return false;
}

// The waits of a warp for the units of its ring, one after the other.  After one that ran out, the copies that are still under
// way are waited for once more each, so that nothing arrives behind the kernel's back, and the warp loads no other unit and asks
// once for each that follows: it polls at most 1 + stages times kCachePolls in vain.  The flag lies in memory, where it costs the
// waits that succeed nothing.
struct RingWaits {
    volatile bool* gave_up;
    template <typename Ready>
    SAM_HOST_DEVICE bool unit(Ready ready) const { return ready() || *gave_up || poll(ready); }
    // A wait for the first of `pending` loaded units ran out; ready(i) asks for the i-th of them.
    template <typename Ready>
    SAM_HOST_DEVICE void give_up(int pending, Ready ready) const {
        for (int i = 0; i < pending; ++i) poll([&] { return ready(i); });
        *gave_up = true;
    }
};

}  // namespace samb200
