// What the host files of the operators of include/ptq_block.h share.
#pragma once

#include <initializer_list>
#include <type_traits>

#include "../../include/ptq_block.h"
#include "ptq_host.h"

namespace ptq_host {

constexpr int kSms = 148;             // of the one GPU that the library is for; only cuts of the work go by it
constexpr long long kMaxGrid = 0x7fffffffll;

#define PTQ_TRY(...)                                  \
    do {                                              \
        const ptq_status_t st_ = (__VA_ARGS__);       \
        if (st_ != PTQ_OK) return st_;                \
    } while (0)

inline ptq_status_t launched()
{
    g_launches.fetch_add(1, std::memory_order_relaxed);
    PTQ_CUDA(cudaGetLastError());
    return PTQ_OK;
}

// Launch of a call's second or third kernel: it may begin while the one before it drains, and waits for its end (griddep_wait) before it
// touches memory.  The first kernel of a call is launched the ordinary way.
template <typename... KArgs, typename... Args>
ptq_status_t launch_next(void (*kern)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    PTQ_CUDA(cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...));
    return launched();
}

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Calls fn with the flag as a constant.
template <class Fn>
ptq_status_t with_flag(bool flag, Fn fn)
{
    return flag ? fn(std::true_type()) : fn(std::false_type());
}

}  // namespace ptq_host
