// Small kernels of linear attention with decays per head: the joint of segments, the ends of the backward pass.
#pragma once

#include "ptq_heads.cuh"

namespace ptq {

// 2^l v + w for any l: growth over a segment may leave binary32's range where what it multiplies (nothing, or a small state) does not.
__device__ __forceinline__ float fold_add(float l, float v, float w)
{
    if (l < 126.0f) return fmaf(exp2f(l), v, w);
    const float whole = rintf(l);
    return scalbnf(v * exp2f(l - whole), static_cast<int>(whole)) + w;
}

// Joins the segments, one element of a state per thread: slot s becomes the state behind segment s (gradients: that in front of
// it); forward, the last slot a copy of the start.
__global__ void __launch_bounds__(256) ptq_heads_fold_kernel(float *slots, const float *logs, const float *start, int64_t heads, int segments, int64_t size, int grad)
{
    griddep_wait();
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < heads * size) {
        const int64_t head = i / size, e = i - head * size;
        float v = start ? start[i] : 0.0f;
        if (!grad && start) slots[(head * segments + segments - 1) * size + e] = v;
        for (int k = 0; k < segments - 1; ++k) {
            const int s = grad ? segments - 1 - k : k;
            float *slot = slots + (head * segments + s) * size + e;
            v = k == 0 && !start ? *slot : fold_add(logs[head * segments + s], v, *slot);
            *slot = v;
        }
    }
    griddep_launch_dependents();
}

// ddelta of one head of one sequence, and that sequence's shares of dA and ddelta_bias.
template <typename T>
__device__ __forceinline__ void finish_delta(const HeadParams &p, int b, int h, T *ddelta, float2 *shares)
{
    const int n = p.lengths ? max(0, min(p.length, __ldg(p.lengths + b))) : p.length;
    const float A = __ldg(p.A + h), bias = p.delta_bias ? __ldg(p.delta_bias + h) : 0.0f;
    const int64_t rows = static_cast<int64_t>(p.batch) * p.length;
    const T *delta = static_cast<const T *>(p.delta);
    double sum_A = 0.0, sum_bias = 0.0;
    for (int t = threadIdx.x; t < p.length; t += 256) {
        const int64_t row = static_cast<int64_t>(b) * p.length + t;
        float de = 0.0f;
        if (t < n) {
            float2 v = make_float2(0.0f, 0.0f);
            for (int tile = 0; tile < p.col_tiles; ++tile) {
                const float2 x = p.part_dt[(static_cast<int64_t>(tile) * p.heads + h) * rows + row];
                v.x += x.x;
                v.y += x.y;
            }
            const float raw = delta ? head_f32(delta[b * p.delta_b + t * p.delta_l + h * p.delta_h]) : 0.0f, dt = head_dt(p, raw, bias);
            if (dt != 0.0f) sum_A += static_cast<double>(dt) * v.x;          // a step with dt = 0 keeps the state with any A
            const float slope = p.flags & kHeadsSoftplus ? 1.0f / (1.0f + expf(-(raw + bias))) : 1.0f;
            // an infinite rate does nothing where no step passes, and where softplus gives the step no length with any delta nearby
            const bool rate = v.x != 0.0f && !(slope == 0.0f && isinf(A));
            de = ((rate ? A * v.x : 0.0f) + (p.flags & kHeadsUnscaled ? 0.0f : v.y)) * slope;
            sum_bias += de;
        }
        if (ddelta) ddelta[row * p.heads + h] = head_round<T>(de);
    }
    __shared__ double warps[2][8];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        sum_A += __shfl_xor_sync(0xffffffffu, sum_A, d);
        sum_bias += __shfl_xor_sync(0xffffffffu, sum_bias, d);
    }
    if ((threadIdx.x & 31) == 0) {
        warps[0][threadIdx.x >> 5] = sum_A;
        warps[1][threadIdx.x >> 5] = sum_bias;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        double v[2] = {};
        for (int k = 0; k < 8; ++k) {
            v[0] += warps[0][k];
            v[1] += warps[1][k];
        }
        shares[static_cast<int64_t>(b) * p.heads + h] = make_float2(static_cast<float>(v[0]), static_cast<float>(v[1]));
    }
}

// blockIdx.y 0: ddelta; dB (1) and dC (2): the heads of a group and their column tiles summed in their order, rounded; kN neighbouring
// states a thread (four where `states` and the outputs' alignment allow it).  Bound by reading the binary32 parts once: 77 MB of a
// training batch of 64 x 197 x 12 heads, 64 states, in 20 us, 23 with ddelta beside it (9 us as a launch of its own).
template <typename T, int kN>
__global__ void __launch_bounds__(256) ptq_heads_finish_kernel(const HeadParams p, T *dB, T *dC, T *ddelta, float2 *shares)
{
    griddep_wait();
    if (blockIdx.y == 0) {
        if (blockIdx.x < static_cast<unsigned>(p.batch * p.heads)) finish_delta(p, static_cast<int>(blockIdx.x) / p.heads, static_cast<int>(blockIdx.x) % p.heads, ddelta, shares);
        return;
    }
    const float *part = blockIdx.y == 2 ? p.part_C : p.part_B;
    T *to = blockIdx.y == 2 ? dC : dB;
    const int sets = p.states / kN;
    const int64_t rows = static_cast<int64_t>(p.batch) * p.length, i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= rows * p.groups * sets) return;
    const int64_t row = i / (p.groups * sets);
    const int in = static_cast<int>(i - row * p.groups * sets), g = in / sets, n = (in - g * sets) * kN;
    const int b = static_cast<int>(row / p.length), t = static_cast<int>(row - static_cast<int64_t>(b) * p.length);
    struct alignas(kN * 4) Parts { float v[kN]; };
    struct alignas(kN * sizeof(T)) Out { T v[kN]; };
    Parts sum = {};
    if (!p.lengths || t < __ldg(p.lengths + b)) {
        for (int tile = 0; tile < p.col_tiles; ++tile) {
            const float *at = part + ((static_cast<int64_t>(tile) * p.heads + g * p.group_heads) * rows + row) * p.states + n;
#pragma unroll 8
            for (int h = 0; h < p.group_heads; ++h) {
                const Parts x = *reinterpret_cast<const Parts *>(at + h * rows * p.states);
#pragma unroll
                for (int k = 0; k < kN; ++k) sum.v[k] += x.v[k];
            }
        }
    }
    Out out;
#pragma unroll
    for (int k = 0; k < kN; ++k) out.v[k] = head_round<T>(sum.v[k]);
    *reinterpret_cast<Out *>(to + kN * i) = out;
}

// dA, ddelta_bias and dD of one head: the sequences' shares in their order.
__global__ void __launch_bounds__(128) ptq_heads_finish_sums_kernel(const HeadParams p, const float2 *shares, float *dA, float *ddelta_bias, float *dD)
{
    griddep_wait();
    const int h = static_cast<int>(blockIdx.x);
    double v[3] = {};
    for (int b = threadIdx.x; b < p.batch; b += 128) {
        const float2 x = shares[static_cast<int64_t>(b) * p.heads + h];
        v[0] += x.x;
        v[1] += x.y;
        if (dD)
            for (int k = 0; k < p.col_tiles * p.segments; ++k) v[2] += p.part_D[(static_cast<int64_t>(k) * p.batch + b) * p.heads + h];
    }
    __shared__ double warps[3][4];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], d);
        if ((threadIdx.x & 31) == 0) warps[k][threadIdx.x >> 5] = v[k];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        dA[h] = static_cast<float>(warps[0][0] + warps[0][1] + warps[0][2] + warps[0][3]);
        if (ddelta_bias) ddelta_bias[h] = static_cast<float>(warps[1][0] + warps[1][1] + warps[1][2] + warps[1][3]);
        if (dD) dD[h] = static_cast<float>(warps[2][0] + warps[2][1] + warps[2][2] + warps[2][3]);
    }
}

}  // namespace ptq
