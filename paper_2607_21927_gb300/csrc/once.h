// What has to be done once per device before a kernel's first launch there.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

namespace ris {

// Function attributes hold for the device that was current when they were set. Tried again where it failed;
// on devices past the table every time.
struct Once {
    static constexpr int kDevices = 64;
    std::atomic<bool> done[kDevices] = {};
    template <typename F>
    cudaError_t operator()(F f)
    {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const bool known = dev >= 0 && dev < kDevices;
        if (known && done[dev].load(std::memory_order_acquire)) return cudaSuccess;
        e = f();
        if (e == cudaSuccess && known) done[dev].store(true, std::memory_order_release);
        return e;
    }
};

}  // namespace ris
