// Host-side helpers shared by the files that implement the C ABI: launch accounting, the calling
// thread's error text and index-check record, argument checks, per-device caches.
#pragma once
#include "../../include/civic.h"

#include <atomic>
#include <cstdint>
#include <cstdio>
#include <cuda_runtime.h>

namespace civic_host {

constexpr size_t kMaxDynamicSmem = 227 * 1024;

inline std::atomic<uint64_t> g_launches{0};
inline std::atomic<int> g_programmatic{1};

inline bool programmatic() { return g_programmatic.load(std::memory_order_relaxed) != 0; }
inline thread_local char g_cuda_error[512] = "";

// Fault record the calling thread's compaction calls validate their index arrays into (device
// int32[4]); NULL = the unchecked kernels.
inline thread_local int32_t* g_index_check = nullptr;

inline civic_status_t cuda_fail(cudaError_t e, const char* what)
{
    snprintf(g_cuda_error, sizeof g_cuda_error, "%s: %s", what, cudaGetErrorString(e));
    (void)cudaGetLastError();  // the runtime's own "last error" is not left behind for the caller's next call
    return CIVIC_ERR_CUDA;
}

#define CIVIC_CUDA_TRY(expr)                                        \
    do {                                                            \
        cudaError_t e_ = (expr);                                    \
        if (e_ != cudaSuccess) return cuda_fail(e_, #expr);         \
    } while (0)

inline bool overlaps(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    if (!a || !b || a_bytes == 0 || b_bytes == 0) return false;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + b_bytes && b0 < a0 + a_bytes;
}

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline int sm_count()
{
    static std::atomic<int> cached[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    int v = cached[dev].load(std::memory_order_relaxed);
    if (v == 0) {
        if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0)
            v = 148;
        cached[dev].store(v, std::memory_order_relaxed);
    }
    return v;
}

// Index of the current device in the per-device caches below, or -1 (then nothing is cached).
inline int device_slot()
{
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -1;
    return dev;
}

// The largest dynamic shared memory a kernel may ask for is a per-device function attribute.
// It is raised ONCE per device to the most the kernel can ever need, not per call to that
// call's size: two host threads launching different shapes would otherwise undo each other's
// setting between cudaFuncSetAttribute and the launch.
template <class Kernel>
civic_status_t allow_dynamic_smem(Kernel kernel, size_t max_bytes, std::atomic<int>* done /*[64]*/)
{
    const int dev = device_slot();
    if (dev >= 0 && done[dev].load(std::memory_order_acquire)) return CIVIC_OK;
    CIVIC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)max_bytes));
    if (dev >= 0) done[dev].store(1, std::memory_order_release);
    return CIVIC_OK;
}

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace civic_host
