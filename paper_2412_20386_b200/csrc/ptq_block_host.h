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

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Calls fn with the flag as a constant.
template <class Fn>
ptq_status_t with_flag(bool flag, Fn fn)
{
    return flag ? fn(std::true_type()) : fn(std::false_type());
}

}  // namespace ptq_host
