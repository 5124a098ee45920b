// What the C entry points share on the host: profiler ranges, alignment checks, facts about the current device.
#pragma once

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>
#include <stdint.h>

#include <atomic>
#include <utility>

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

// Launches a kernel that may be set up while the kernel before it in the stream still drains: such a kernel calls
// grid_dependency() before its first access to global memory, which returns when everything before it is complete and
// visible, and lets its own successor be set up as soon as all its blocks run.  Stream order, as the caller sees it, is
// that of any launch; back to back, a call starts about a microsecond sooner.  (What such a kernel reads may still be
// written while it already runs, so it does not read it as constant for its lifetime: no __ldg, no __restrict__ on inputs.)
template <typename... P, typename... A>
inline bool launch_early(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, A &&...args) {
    cudaLaunchConfig_t lc{};
    lc.gridDim = grid;
    lc.blockDim = dim3((unsigned)threads, 1, 1);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&lc, kernel, std::forward<A>(args)...) == cudaSuccess;
}
__device__ __forceinline__ void grid_dependency() {
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

}  // namespace spice
