// Launches of the scan's kernels for one type of activations; each type is compiled as a file of its own.
#pragma once

#include <algorithm>

#include "ptq_block_host.h"
#include "ptq_scan.cuh"

namespace ptq_host {

// Lanes per channel, channels of a lane and states of each.  Forward, a lane has two channels: the values of B and C that it reads from
// shared memory serve both (128 x 197 x 768, N = 16: 135 us; one channel of eight states 145, of four 183; four channels 148, too few warps).
// Where two lanes a channel leave few warps, a channel has four, with two channels a lane or with one (64 x 197 x 384: 46 and 60 us;
// 1 x 197 x 384 in one pass: 18 with one channel a lane).
struct ScanSplit {
    int lanes, channels, states;
    int width() const { return 32 / lanes * channels; }
};
inline ScanSplit scan_split_forward(int states, int level)      // 0: many warps, 1, 2: few
{
    if (states <= 4) return {1, 1, states == 3 ? 4 : states};
    if (states <= 8) return level == 2 ? ScanSplit{2, 1, 4} : ScanSplit{2, 2, 4};
    if (states <= 16) return level == 2 ? ScanSplit{4, 1, 4} : level == 1 ? ScanSplit{4, 2, 4} : ScanSplit{2, 2, 8};
    return {4, 2, 8};
}
inline ScanSplit scan_split_backward(int states)
{
    if (states <= 4) return {1, 1, states == 3 ? 4 : states};
    return {states <= 8 ? 2 : states <= 16 ? 4 : 8, 2, 4};        // a lane holds 64 products of the stretch
}
template <int kC, int kNS, int kS>
struct ScanForm {
    static constexpr int channels = kC, states = kNS, lanes = kS;
};
template <class Fn>
ptq_status_t with_forward_split(ScanSplit sp, Fn fn)
{
    if (sp.lanes == 1 && sp.states == 1) return fn(ScanForm<1, 1, 1>());
    if (sp.lanes == 1 && sp.states == 2) return fn(ScanForm<1, 2, 1>());
    if (sp.lanes == 1) return fn(ScanForm<1, 4, 1>());
    if (sp.lanes == 2 && sp.channels == 1) return fn(ScanForm<1, 4, 2>());
    if (sp.lanes == 2 && sp.states == 4) return fn(ScanForm<2, 4, 2>());
    if (sp.lanes == 2) return fn(ScanForm<2, 8, 2>());
    if (sp.channels == 1) return fn(ScanForm<1, 4, 4>());
    if (sp.states == 4) return fn(ScanForm<2, 4, 4>());
    return fn(ScanForm<2, 8, 4>());
}
template <class Fn>
ptq_status_t with_backward_split(int states, Fn fn)
{
    const ScanSplit sp = scan_split_backward(states);
    if (sp.lanes == 1 && sp.states == 1) return fn(ScanForm<1, 1, 1>());
    if (sp.lanes == 1 && sp.states == 2) return fn(ScanForm<1, 2, 1>());
    if (sp.lanes == 1) return fn(ScanForm<1, 4, 1>());
    if (sp.lanes == 2) return fn(ScanForm<2, 4, 2>());
    if (sp.lanes == 4) return fn(ScanForm<2, 4, 4>());
    return fn(ScanForm<2, 4, 8>());
}
// One token per sequence: lanes of a channel, states of a lane.
template <class Fn>
ptq_status_t with_step_split(int states, Fn fn)
{
    if (states == 1) return fn(ScanForm<1, 1, 1>());
    if (states == 2) return fn(ScanForm<1, 2, 1>());
    if (states <= 4) return fn(ScanForm<1, 4, 1>());
    if (states <= 8) return fn(ScanForm<1, 4, 2>());
    if (states <= 16) return fn(ScanForm<1, 4, 4>());
    return fn(ScanForm<1, 4, 8>());
}

// How a launch is cut: the forward pass's split and its warps, CTAs of the backward pass, and whether rows are moved 16 bytes at a time.
struct ScanCut {
    ScanSplit split;
    long long warps, ctas;
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
    return with_forward_split(cut.split, [&](auto form) {
        return with_flag(cut.whole, [&](auto whole) {
            using F = decltype(form);
            constexpr int kThreads = ptq::kScanWarps * 32;
            constexpr bool kWhole = decltype(whole)::value;
            const unsigned grid = static_cast<unsigned>(ceil_div(cut.warps, ptq::kScanWarps));
            if (mode == ptq::kScanForward && p.chunks > 1)
                return launch_next(ptq::ptq_scan_kernel<T, F::channels, F::states, F::lanes, ptq::kScanForward, kWhole>, grid, kThreads, 0, stream, p);
            if (mode == ptq::kScanForward)
                ptq::ptq_scan_kernel<T, F::channels, F::states, F::lanes, ptq::kScanForward, kWhole><<<grid, kThreads, 0, stream>>>(p);
            else if (mode == ptq::kScanSum)
                ptq::ptq_scan_kernel<T, F::channels, F::states, F::lanes, ptq::kScanSum, kWhole><<<grid, kThreads, 0, stream>>>(p);
            else
                ptq::ptq_scan_kernel<T, F::channels, F::states, F::lanes, ptq::kScanGradSum, kWhole><<<grid, kThreads, 0, stream>>>(p);
            return launched();
        });
    });
}
template <typename T>
ptq_status_t ScanLaunch<T>::backward(const ptq::ScanParams &p, const ScanCut &cut, cudaStream_t stream)
{
    return with_backward_split(p.states, [&](auto form) {
        return with_flag(cut.whole, [&](auto whole) {
            using F = decltype(form);
            constexpr auto kKern = ptq::ptq_scan_backward_kernel<T, F::channels, F::states, F::lanes, decltype(whole)::value>;
            constexpr size_t kBytes = ptq::scan_backward_smem(F::channels, F::states, F::lanes, sizeof(T));
            PTQ_TRY(ensure_smem<kKern>(static_cast<int>(kBytes)));
            if (p.chunks > 1) return launch_next(kKern, static_cast<unsigned>(cut.ctas), ptq::kScanWarps * 32, kBytes, stream, p);
            kKern<<<static_cast<unsigned>(cut.ctas), ptq::kScanWarps * 32, kBytes, stream>>>(p);
            return launched();
        });
    });
}
template <typename T>
ptq_status_t ScanLaunch<T>::finish(const ptq::ScanParams &p, float *dA, float *dD, float *dbias, cudaStream_t stream)
{
    const int blocks_A = static_cast<int>(ceil_div(static_cast<long long>(p.channels) * p.states, 32));
    const int blocks_D = static_cast<int>(ceil_div(p.channels, 32));
    const long long sets = p.part_BC ? ceil_div(static_cast<long long>(p.batch) * p.length, ptq::kScanFinishThreads / (2 * p.states)) * p.groups : 0;
    const int blocks_BC = static_cast<int>(std::min<long long>(sets, 8 * kSms));
    return launch_next(ptq::ptq_scan_finish_kernel<T>, static_cast<unsigned>(blocks_A + 2 * blocks_D + blocks_BC), ptq::kScanFinishThreads, 0, stream, p,
                       dA, dD, dbias, blocks_A, blocks_D);
}
template <typename T>
ptq_status_t ScanLaunch<T>::step(const ptq::ScanParams &p, bool whole_rows, cudaStream_t stream)
{
    return with_step_split(p.states, [&](auto form) {
        return with_flag(whole_rows, [&](auto whole) {
            using F = decltype(form);
            const long long blocks = ceil_div(p.channels, 256 / F::lanes);
            const long long rows = std::max(1ll, std::min<long long>(ceil_div(p.batch, F::lanes), 4 * kSms / blocks));
            ptq::ptq_scan_step_kernel<T, F::states, F::lanes, decltype(whole)::value><<<static_cast<unsigned>(blocks * rows), 256, 0, stream>>>(p);
            return launched();
        });
    });
}
template struct ScanLaunch<PTQ_SCAN_TYPE>;
#endif

}  // namespace ptq_host
