// Launches of the scan's kernels for one type of activations; each type is compiled as a file of its own.
#pragma once

#include <algorithm>

#include "ptq_block_host.h"
#include "ptq_scan.cuh"

namespace ptq_host {

// Lanes per channel and states per lane.
struct ScanSplit {
    int lanes, states;
};
inline ScanSplit scan_split(int states)
{
    if (states <= 2) return {1, states};
    if (states <= 4) return {2, 2};   // one lane of four would hold 64 products of the backward pass and 32 sums
    return {states <= 8 ? 2 : states <= 16 ? 4 : 8, 4};
}
template <class Fn>
ptq_status_t with_split(int states, Fn fn)
{
    using std::integral_constant;
    const ScanSplit sp = scan_split(states);
    if (sp.lanes == 1 && sp.states == 1) return fn(integral_constant<int, 1>(), integral_constant<int, 1>());
    if (sp.lanes == 1) return fn(integral_constant<int, 2>(), integral_constant<int, 1>());
    if (sp.states == 2) return fn(integral_constant<int, 2>(), integral_constant<int, 2>());
    if (sp.lanes == 2) return fn(integral_constant<int, 4>(), integral_constant<int, 2>());
    if (sp.lanes == 4) return fn(integral_constant<int, 4>(), integral_constant<int, 4>());
    return fn(integral_constant<int, 4>(), integral_constant<int, 8>());
}

// How a call is cut: threads of a CTA, CTAs, and whether rows are moved 16 bytes at a time.
struct ScanCut {
    int threads;
    long long ctas;
    bool whole;
};

template <typename T>
struct ScanLaunch {
    static ptq_status_t forward(int mode, const ptq::ScanParams &p, const ScanCut &cut, cudaStream_t stream);
    static ptq_status_t backward(const ptq::ScanParams &p, const ScanCut &cut, cudaStream_t stream);
    static ptq_status_t finish(const ptq::ScanParams &p, float *dA, float *dD, float *dbias, cudaStream_t stream);
    static ptq_status_t step(const ptq::ScanParams &p, bool whole, cudaStream_t stream);
};

#ifdef PTQ_SCAN_TYPE
template <typename T>
ptq_status_t ScanLaunch<T>::forward(int mode, const ptq::ScanParams &p, const ScanCut &cut, cudaStream_t stream)
{
    return with_split(p.states, [&](auto ns, auto lanes) {
        return with_flag(cut.whole, [&](auto whole) {
            constexpr int kNS = decltype(ns)::value, kS = decltype(lanes)::value;
            constexpr bool kWhole = decltype(whole)::value;
            const size_t smem = static_cast<size_t>(64) * cut.threads + 64 * kS * kS * kNS;
            const unsigned grid = static_cast<unsigned>(cut.ctas);
            if (mode == ptq::kScanForward)
                ptq::ptq_scan_kernel<T, kNS, kS, ptq::kScanForward, kWhole><<<grid, cut.threads, smem, stream>>>(p);
            else if (mode == ptq::kScanSum)
                ptq::ptq_scan_kernel<T, kNS, kS, ptq::kScanSum, kWhole><<<grid, cut.threads, smem, stream>>>(p);
            else
                ptq::ptq_scan_kernel<T, kNS, kS, ptq::kScanGradSum, kWhole><<<grid, cut.threads, smem, stream>>>(p);
            return launched();
        });
    });
}
template <typename T>
ptq_status_t ScanLaunch<T>::backward(const ptq::ScanParams &p, const ScanCut &cut, cudaStream_t stream)
{
    return with_split(p.states, [&](auto ns, auto lanes) {
        return with_flag(cut.whole, [&](auto whole) {
            constexpr int kNS = decltype(ns)::value, kS = decltype(lanes)::value;
            const size_t rows = ptq::kScanHistory, np = kNS * kS;
            const size_t smem = rows * (cut.threads / kS) * 16 + rows * np * 8 + (cut.threads / 32) * rows * np * 8;
            ptq::ptq_scan_backward_kernel<T, kNS, kS, decltype(whole)::value><<<static_cast<unsigned>(cut.ctas), cut.threads, smem, stream>>>(p);
            return launched();
        });
    });
}
template <typename T>
ptq_status_t ScanLaunch<T>::finish(const ptq::ScanParams &p, float *dA, float *dD, float *dbias, cudaStream_t stream)
{
    const int blocks_A = static_cast<int>(ceil_div(static_cast<long long>(p.channels) * p.states, 32));
    const int blocks_D = static_cast<int>(ceil_div(p.channels, 32));
    const long long outputs = p.part_BC ? static_cast<long long>(p.batch) * p.length * 2 * p.states * p.groups : 0;
    const int blocks_BC = static_cast<int>(std::min<long long>(ceil_div(outputs, 256), 16 * kSms));
    ptq::ptq_scan_finish_kernel<T><<<blocks_A + 2 * blocks_D + blocks_BC, 256, 0, stream>>>(p, dA, dD, dbias, blocks_A, blocks_D);
    return launched();
}
template <typename T>
ptq_status_t ScanLaunch<T>::step(const ptq::ScanParams &p, bool whole_rows, cudaStream_t stream)
{
    return with_split(p.states, [&](auto ns, auto lanes) {
        return with_flag(whole_rows, [&](auto whole) {
            constexpr int kNS = decltype(ns)::value, kS = decltype(lanes)::value;
            const long long blocks = ceil_div(p.channels, 256 / kS);
            const long long rows = std::min<long long>(p.batch, std::max(1ll, ceil_div(16 * kSms, blocks)));
            ptq::ptq_scan_step_kernel<T, kNS, kS, decltype(whole)::value><<<static_cast<unsigned>(blocks * rows), 256, 0, stream>>>(p);
            return launched();
        });
    });
}
template struct ScanLaunch<PTQ_SCAN_TYPE>;
#endif

}  // namespace ptq_host
