// um_device.cuh -- what the host code keeps for each GPU that a process uses:
// found at the first call on a device, and kept only when that worked, so that
// a call after a failed one starts anew.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

namespace um {

// V: a number or a pointer.  Two threads may find the same value at once.
template <typename V> class PerDevice {
    static constexpr int kKept = 64;         // devices; others find theirs every time
    std::atomic<V> value_[kKept] = {};
    std::atomic<bool> have_[kKept] = {};

public:
    // *out: the current device's value, at the first call from find(device, out)
    template <typename F> cudaError_t get(V *out, F &&find) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const bool kept = dev >= 0 && dev < kKept;
        if (kept && have_[dev].load(std::memory_order_acquire)) {
            *out = value_[dev].load(std::memory_order_relaxed);
            return cudaSuccess;
        }
        e = find(dev, out);
        if (e == cudaSuccess && kept) {
            value_[dev].store(*out, std::memory_order_relaxed);
            have_[dev].store(true, std::memory_order_release);
        }
        return e;
    }
};

// Lets kernel K take `bytes` of dynamic shared memory, the same at every call.
template <auto K> cudaError_t allow_dynamic_smem(size_t bytes) {
    static PerDevice<int> allowed;
    int have = 0;
    return allowed.get(&have, [&](int, int *v) {
        *v = (int)bytes;
        return cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, *v);
    });
}

}  // namespace um
