// Host helpers shared by the sources of the operators around the attention (backward pass, block operators).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

namespace lf {

inline size_t align_up_256(size_t x) { return (x + 255) / 256 * 256; }
inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// [a, a + na) and [b, b + nb) share a byte.
inline bool overlaps(const void* a, size_t na, const void* b, size_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

constexpr int kMaxDevices = 64;

// SM count of a compute capability 10.x device, looked up once per device; -1: no such device (or no CUDA), -2: another
// architecture.  Concurrent first calls store the same value.
inline int device_sm_count(int device)
{
    static std::atomic<int> known[kMaxDevices];
    if (device < 0 || device >= kMaxDevices) return -1;
    int n = known[device].load(std::memory_order_relaxed);
    if (n != 0) return n;
    int major = 0;
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        cudaGetLastError();
        return -1;
    }
    if (major != 10) n = -2;
    known[device].store(n, std::memory_order_relaxed);
    return n;
}

// The current device for the length of a call, put back afterwards.
struct CurrentDevice {
    int prev = -1;
    bool ok = false;
    explicit CurrentDevice(int device)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) {
            cudaGetLastError();
            return;
        }
        ok = prev == device || cudaSetDevice(device) == cudaSuccess;
        if (!ok) cudaGetLastError();
        changed = ok && prev != device;
    }
    ~CurrentDevice()
    {
        if (changed) cudaSetDevice(prev);
    }
    bool changed = false;
};

// Raises a kernel's dynamic shared-memory limit, once per device.  `done`: one bit per device, one word per kernel.
template <typename K>
inline cudaError_t allow_smem(K* kernel, size_t bytes, int device, std::atomic<uint64_t>* done)
{
    const uint64_t bit = uint64_t(1) << device;
    if (done->load(std::memory_order_acquire) & bit) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (e == cudaSuccess) done->fetch_or(bit, std::memory_order_release);
    return e;
}

// Launch that may be scheduled while the kernel before it in the stream drains (see pdl_wait()).
template <typename... KArgs, typename... Args>
inline cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

}  // namespace lf
