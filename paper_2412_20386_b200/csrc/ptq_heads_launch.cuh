// Launches of the kernels of linear attention with decays per head for one type of activations; ptq_heads_{f16,bf16,f32}.cu each
// instantiate one.
#pragma once

#include "ptq_block_host.h"
#include "ptq_heads_backward.cuh"

namespace ptq_host {

template <class Fn>
ptq_status_t with_states(int states, Fn fn)
{
    if (states <= 32) return fn(std::integral_constant<int, 32>());
    if (states <= 64) return fn(std::integral_constant<int, 64>());
    return fn(std::integral_constant<int, 128>());
}

template <typename T>
struct HeadsLaunch {
    static ptq_status_t chunks(int mode, const ptq::HeadParams &p, bool whole, bool next, cudaStream_t stream);
    static ptq_status_t step(const ptq::HeadParams &p, bool whole, cudaStream_t stream);
    static ptq_status_t backward(const ptq::HeadParams &p, bool whole, bool next, cudaStream_t stream);
};

#ifdef PTQ_HEADS_DEFINE
template <typename T>
ptq_status_t HeadsLaunch<T>::chunks(int mode, const ptq::HeadParams &p, bool whole, bool next, cudaStream_t stream)
{
    return with_states(p.states, [&](auto n) {
        constexpr int NP = decltype(n)::value;
        const auto go = [&](auto m) {
            return with_flag(whole, [&](auto w) {
                constexpr int kMode = decltype(m)::value;
                constexpr auto kKern = ptq::ptq_heads_kernel<T, NP, kMode, decltype(w)::value>;
                constexpr int kBytes = ptq::HeadSmem<T, NP, kMode>::kBytes;
                static_assert(kBytes <= 232448, "shared memory of one CTA");
                PTQ_TRY(ensure_smem<kKern>(kBytes));
                const long long ctas = static_cast<long long>(p.batch) * p.heads * p.col_tiles * (kMode == ptq::kHeadForward ? p.segments : p.segments - 1);
                const dim3 grid(static_cast<unsigned>(ctas));
                if (next) return launch_next(kKern, grid, 256, kBytes, stream, p);
                kKern<<<grid, 256, kBytes, stream>>>(p);
                return launched();
            });
        };
        if (mode == ptq::kHeadForward) return go(std::integral_constant<int, ptq::kHeadForward>());
        if (mode == ptq::kHeadSum) return go(std::integral_constant<int, ptq::kHeadSum>());
        return go(std::integral_constant<int, ptq::kHeadGradSum>());
    });
}

template <typename T>
ptq_status_t HeadsLaunch<T>::step(const ptq::HeadParams &p, bool whole, cudaStream_t stream)
{
    return with_states(p.states, [&](auto n) {
        return with_flag(whole, [&](auto w) {
            constexpr int kLanes = decltype(n)::value / 4;
            constexpr int kRows = 32;                // rows of a CTA
            const long long ctas = static_cast<long long>(p.batch) * p.heads * ceil_div(p.cols, kRows);
            if (ctas > kMaxGrid) return fail(PTQ_ERR_SHAPE, "the batch is too large for one launch");
            ptq::ptq_heads_step_kernel<T, kLanes, decltype(w)::value><<<static_cast<unsigned>(ctas), 128, 0, stream>>>(p);
            return launched();
        });
    });
}

template <typename T>
ptq_status_t HeadsLaunch<T>::backward(const ptq::HeadParams &p, bool whole, bool next, cudaStream_t stream)
{
    return with_states(p.states, [&](auto n) {
        constexpr int NP = decltype(n)::value;
        return with_flag(whole, [&](auto w) {
            constexpr auto kKern = ptq::ptq_heads_backward_kernel<T, NP, decltype(w)::value>;
            constexpr int kBytes = ptq::HeadBackSmem<T, NP>::kBytes;
            static_assert(kBytes <= 232448, "shared memory of one CTA");
            PTQ_TRY(ensure_smem<kKern>(kBytes));
            const dim3 grid(static_cast<unsigned>(static_cast<long long>(p.batch) * p.heads * p.col_tiles * p.segments));
            if (next) return launch_next(kKern, grid, 256, kBytes, stream, p);
            kKern<<<grid, 256, kBytes, stream>>>(p);
            return launched();
        });
    });
}
#endif

}  // namespace ptq_host
