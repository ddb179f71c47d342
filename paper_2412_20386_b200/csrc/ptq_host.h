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

}  // namespace ptq_host
