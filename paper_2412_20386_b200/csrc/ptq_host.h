// What all host files of the library share: the error text, the launch counter and the checks that turn failures into codes.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <exception>

#include "../../include/ptq_linear.h"

namespace ptq_host {

inline thread_local char g_err[512] = "";
inline std::atomic<unsigned long long> g_launches{0};

inline ptq_status_t fail(ptq_status_t st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return st;
}

#define PTQ_CUDA(...)                                                                          \
    do {                                                                                       \
        cudaError_t e_ = (__VA_ARGS__);                                                        \
        if (e_ != cudaSuccess)                                                                 \
            return fail(e_ == cudaErrorMemoryAllocation ? PTQ_ERR_NOMEM : PTQ_ERR_CUDA,        \
                        "%s failed: %s", #__VA_ARGS__, cudaGetErrorString(e_));                \
    } while (0)

// The body of an entry point that allocates host memory: no exception may leave a C function.
template <class Fn>
ptq_status_t no_throw(Fn fn)
{
    try {
        return fn();
    } catch (const std::exception &) {      // std::bad_alloc is all that these bodies raise
        return fail(PTQ_ERR_NOMEM, "host allocation failed");
    }
}

// Opt a kernel in to `bytes` of dynamic shared memory, once per kernel and device (the attribute belongs
// to the function on the CURRENT device, which is `device`).  The kernel is
// a template argument so that every kernel has its own flags.
template <auto kKern>
ptq_status_t ensure_smem(int device, int bytes)
{
    constexpr int kMaxDevices = 64;
    static std::atomic<bool> done[kMaxDevices] = {};
    if (device < 0 || device >= kMaxDevices) return fail(PTQ_ERR_CUDA, "device index %d out of range", device);
    // lock-free once the attribute is set; two threads racing on the first call both set the same value
    if (!done[device].load(std::memory_order_acquire)) {
        PTQ_CUDA(cudaFuncSetAttribute(kKern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        done[device].store(true, std::memory_order_release);
    }
    return PTQ_OK;
}
template <auto kKern>
ptq_status_t ensure_smem(int bytes)
{
    int device = -1;
    PTQ_CUDA(cudaGetDevice(&device));
    return ensure_smem<kKern>(device, bytes);
}

}  // namespace ptq_host
