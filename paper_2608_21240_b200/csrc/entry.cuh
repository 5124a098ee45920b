// What the C entry points share on the host: profiler ranges, alignment checks, facts about the current device.
#pragma once

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>
#include <stdint.h>

#include <atomic>

namespace spice {

// NVTX range around the host side of an entry point (named after it): a profiler's timeline shows which call enqueued
// which kernels; without a profiler attached the calls return at once.
struct Range {
    explicit Range(const char *name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
    Range(const Range &) = delete;
    Range &operator=(const Range &) = delete;
};

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Number of SMs of the calling thread's current device, asked once per device; 0 when there is no such device.
inline int current_device_sms(int *device_out = nullptr) {
    constexpr int MAX_DEVICES = 64;
    static std::atomic<int> sms[MAX_DEVICES];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 0;
    if (device_out) *device_out = dev;
    int n = sms[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        sms[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

}  // namespace spice
