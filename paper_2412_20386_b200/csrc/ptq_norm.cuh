// Norm before or behind a block, with what stands around it in one pass:
//
//   v = x silu(gate)  (gate in front)  or x;   r = residual + scale v;   n = (r - mean) / sqrt(var + eps), or r / rms
//   y = (n weight + bias) silu(gate)  (gate behind)  or n weight + bias;   r and y are written
//
// and the gradients of all of it.  Bound: the bytes of the rows, each read and written once.  A thread owns 8 columns, whose
// parameters (and, backward, whose sums of dweight, dbias and dscale) stay in its registers, a CTA of ceil(D / 256) warps the
// whole row; it goes over the rows kRB at a time, so that one barrier serves the sums of kRB rows.  Mean and variance are
// two passes over the registers.  The norm is taken of the unrounded r, in both directions, so y does not depend on the type of r.
#pragma once

#include "ptq_block.cuh"

namespace ptq {

constexpr int kNormMaxWarps = 32;     // 8192 columns
enum { kGateNone = 0, kGateIn = 1, kGateOut = 2 };

struct NormParams {
    const void *x, *residual, *gate;            // residual and gate may be null
    long long x_l, residual_l, gate_l;          // pitches in elements
    const float *weight, *bias, *scale;         // each may be null
    long long rows;
    int cols, gate_at;
    float eps, inv_cols;
    bool layer;
    int stages;                                 // sets of rows in shared memory
    void *y, *residual_out;                     // dense
    // backward
    const void *dy, *dresidual_out;             // dense; dresidual_out may be null
    void *dx, *dresidual, *dgate;               // dense; the last two may be null
    float *part;                                // [gridDim.x][3][cols]: dweight, dbias, dscale
};

// Sums over the CTA of kV values per thread, the same in every thread.  `buf` [kV][warps]; a barrier lies between the writes and
// the reads, and the caller gives another buffer the next time.
template <int kV>
__device__ __forceinline__ void row_sums(float (&v)[kV], float *buf, int warp, int warps, int lane)
{
#pragma unroll
    for (int i = 0; i < kV; ++i) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    if (warps == 1) return;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < kV; ++i) buf[i * kNormMaxWarps + warp] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        v[i] = 0.0f;
        for (int w = 0; w < warps; ++w) v[i] += buf[i * kNormMaxWarps + w];
    }
}

// Where a thread's pieces of the rows lie in shared memory, in units of 16 bytes: kRB rows of each tensor that the call has.
struct NormStage {
    int x, residual, gate, dy, dresidual, size;
    __host__ __device__ NormStage(bool has_residual, bool has_gate, bool has_dy, bool has_dresidual, int parts, int residual_parts, int rows, int threads)
    {
        const int unit = rows * threads;
        x = 0;
        residual = x + unit * parts;
        gate = residual + (has_residual ? unit * residual_parts : 0);
        dy = gate + (has_gate ? unit * parts : 0);
        dresidual = dy + (has_dy ? unit * parts : 0);
        size = dresidual + (has_dresidual ? unit * residual_parts : 0);
    }
};

// kWide: rows of more than 2048 columns, up to 32 warps of 64 registers: the parameters are taken from the cache for every row.
// The rows come through shared memory, one set of kRB under way while the other is worked on (p.stages = 2; 1 where a row is too wide
// for that): held in registers, the loads of two sets would leave too few warps to keep the memory busy.
template <typename T, typename R, int kRB, bool kWide, bool kBackward, bool kWhole>
__global__ void __launch_bounds__(kWide ? 1024 : 256) ptq_norm_kernel(const NormParams p)
{
    constexpr int kStages = 3;
    constexpr int kParts = sizeof(T) / 2, kResidualParts = sizeof(R) / 2;
    __shared__ float s_sum[2][kStages][2 * kRB * kNormMaxWarps];
    extern __shared__ __align__(16) uint4 norm_rows[];
    const int threads = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = threads >> 5;
    const int c = threadIdx.x * 8, cn = max(min(8, p.cols - c), 0);
    const bool has_dr = kBackward && p.dresidual_out;
    const NormStage at(p.residual, p.gate, kBackward, has_dr, kParts, kResidualParts, kRB, threads);
    Piece<float, 8> weight, bias, scale;
    const auto parameters = [&] {
        weight = load_piece<kWhole, float, 8>(p.weight + c, p.weight ? cn : 0);
        bias = load_piece<kWhole, float, 8>(p.bias + c, p.bias ? cn : 0);
        scale = load_piece<kWhole, float, 8>(p.scale + c, p.scale ? cn : 0);
        if (!p.weight) {
#pragma unroll
            for (int e = 0; e < 8; ++e) weight.w[e] = __float_as_uint(1.0f);
        }
        if (!p.scale) {
#pragma unroll
            for (int e = 0; e < 8; ++e) scale.w[e] = __float_as_uint(1.0f);
        }
    };
    if (!kWide) parameters();
    float sum_w[8], sum_b[8], sum_s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (kBackward) sum_w[e] = sum_b[e] = sum_s[e] = 0.0f;
    const auto fetch = [&](long long m0, int stage) {
        uint4 *to = norm_rows + stage * at.size + threadIdx.x;
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            const long long m = m0 + i;
            const int n = m < p.rows ? cn : 0;
            stage_piece<kWhole, T, 8>(to + at.x + i * kParts * threads, static_cast<const T *>(p.x) + m * p.x_l + c, n, threads);
            if (p.residual)
                stage_piece<kWhole, R, 8>(to + at.residual + i * kResidualParts * threads, static_cast<const R *>(p.residual) + m * p.residual_l + c, n, threads);
            if (p.gate) stage_piece<kWhole, T, 8>(to + at.gate + i * kParts * threads, static_cast<const T *>(p.gate) + m * p.gate_l + c, n, threads);
            if (kBackward) stage_piece<kWhole, T, 8>(to + at.dy + i * kParts * threads, static_cast<const T *>(p.dy) + m * p.cols + c, n, threads);
            if (has_dr)
                stage_piece<kWhole, R, 8>(to + at.dresidual + i * kResidualParts * threads, static_cast<const R *>(p.dresidual_out) + m * p.cols + c, n, threads);
        }
        stage_group();
    };
    const long long step = static_cast<long long>(gridDim.x) * kRB;
    long long m0 = static_cast<long long>(blockIdx.x) * kRB;
    if (p.stages == 2 && m0 < p.rows) fetch(m0, 0);
    for (int parity = 0; m0 < p.rows; m0 += step, parity ^= 1) {
        if (p.stages == 2) {
            if (m0 + step < p.rows)
                fetch(m0 + step, parity ^ 1);
            else
                stage_group();
            staged_but<1>();
        } else {
            fetch(m0, 0);
            staged();
        }
        const uint4 *from = norm_rows + (p.stages == 2 ? parity * at.size : 0) + threadIdx.x;
        const auto x_of = [&](int i) { return staged_piece<T, 8>(from + at.x + i * kParts * threads, threads); };
        const auto gate_of = [&](int i) { return staged_piece<T, 8>(from + at.gate + i * kParts * threads, threads); };
        if (kWide) parameters();
        float r[kRB][8], mean[kRB], rstd[kRB];
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            mean[i] = 0.0f;
            const Piece<T, 8> x = x_of(i);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[i][e] = x[e];
            if (p.gate_at == kGateIn) {
                const Piece<T, 8> g = gate_of(i);
#pragma unroll
                for (int e = 0; e < 8; ++e) r[i][e] *= g[e] * sigmoid_f32(g[e]);
            }
            if (p.scale) {
#pragma unroll
                for (int e = 0; e < 8; ++e) r[i][e] *= scale[e];
            }
            if (p.residual) {
                const Piece<R, 8> res = staged_piece<R, 8>(from + at.residual + i * kResidualParts * threads, threads);
#pragma unroll
                for (int e = 0; e < 8; ++e) r[i][e] += res[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) mean[i] += r[i][e];
        }
        if (p.layer) {
            row_sums<kRB>(mean, s_sum[parity][0], warp, warps, lane);
#pragma unroll
            for (int i = 0; i < kRB; ++i) mean[i] *= p.inv_cols;
        }
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            if (!kBackward && p.residual_out && m0 + i < p.rows)
                store_piece<kWhole, R, 8>(static_cast<R *>(p.residual_out) + (m0 + i) * p.cols + c, r[i], cn);
            rstd[i] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (p.layer) r[i][e] = e < cn ? r[i][e] - mean[i] : 0.0f;
                rstd[i] = fmaf(r[i][e], r[i][e], rstd[i]);
            }
        }
        row_sums<kRB>(rstd, s_sum[parity][1], warp, warps, lane);
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            rstd[i] = rsqrtf(fmaf(rstd[i], p.inv_cols, p.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) r[i][e] *= rstd[i];                          // n from here on
        }
        if constexpr (!kBackward) {
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                if (m0 + i >= p.rows) break;
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(r[i][e], weight[e], bias[e]);
                if (p.gate_at == kGateOut) {
                    const Piece<T, 8> g = gate_of(i);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= g[e] * sigmoid_f32(g[e]);
                }
                store_piece<kWhole, T, 8>(static_cast<T *>(p.y) + (m0 + i) * p.cols + c, y, cn);
            }
        } else {
            float sums[2 * kRB], dn[kRB][8];
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                const Piece<T, 8> dy = staged_piece<T, 8>(from + at.dy + i * kParts * threads, threads);
                sums[2 * i] = sums[2 * i + 1] = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) dn[i][e] = dy[e];
                if (p.gate_at == kGateOut) {
                    const Piece<T, 8> g = gate_of(i);
                    float dg[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float z = g[e], s = sigmoid_f32(z);
                        dg[e] = dn[i][e] * fmaf(r[i][e], weight[e], bias[e]) * s * fmaf(z, 1.0f - s, 1.0f);
                        dn[i][e] *= z * s;
                    }
                    if (m0 + i < p.rows) store_piece<kWhole, T, 8>(static_cast<T *>(p.dgate) + (m0 + i) * p.cols + c, dg, cn);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum_w[e] = fmaf(dn[i][e], r[i][e], sum_w[e]);
                    sum_b[e] += dn[i][e];
                    dn[i][e] *= weight[e];
                    sums[2 * i] = fmaf(dn[i][e], r[i][e], sums[2 * i]);
                    sums[2 * i + 1] += dn[i][e];
                }
            }
            row_sums<2 * kRB>(sums, s_sum[parity][2], warp, warps, lane);
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                if (m0 + i >= p.rows) break;
                const float along = sums[2 * i] * p.inv_cols, flat = p.layer ? sums[2 * i + 1] * p.inv_cols : 0.0f;
                const long long out = (m0 + i) * p.cols + c;
                float dx[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) dn[i][e] = (fmaf(-r[i][e], along, dn[i][e]) - flat) * rstd[i];       // dr from here on
                if (has_dr) {
                    const Piece<R, 8> dres = staged_piece<R, 8>(from + at.dresidual + i * kResidualParts * threads, threads);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dn[i][e] += dres[e];
                }
                if (p.dresidual) store_piece<kWhole, R, 8>(static_cast<R *>(p.dresidual) + out, dn[i], cn);
                const Piece<T, 8> x = x_of(i);
                if (p.gate_at == kGateIn) {
                    const Piece<T, 8> g = gate_of(i);
                    float dg[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float z = g[e], s = sigmoid_f32(z);
                        dx[e] = dn[i][e] * scale[e];
                        dg[e] = dx[e] * x[e] * s * fmaf(z, 1.0f - s, 1.0f);
                        dx[e] *= z * s;
                        sum_s[e] = fmaf(dn[i][e], x[e] * z * s, sum_s[e]);
                    }
                    store_piece<kWhole, T, 8>(static_cast<T *>(p.dgate) + out, dg, cn);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        dx[e] = dn[i][e] * scale[e];
                        sum_s[e] = fmaf(dn[i][e], x[e], sum_s[e]);
                    }
                }
                store_piece<kWhole, T, 8>(static_cast<T *>(p.dx) + out, dx, cn);
            }
        }
    }
    if constexpr (kBackward) {
        float *part = p.part + static_cast<long long>(blockIdx.x) * 3 * p.cols + c;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < cn) {
                part[e] = sum_w[e];
                part[p.cols + e] = sum_b[e];
                part[2 * p.cols + e] = sum_s[e];
            }
    }
}

// Column sums of the CTAs' shares: part[rows][3][cols].
__global__ void __launch_bounds__(1024) ptq_norm_finish_kernel(const float *part, int rows, int cols, float *dweight, float *dbias, float *dscale)
{
    __shared__ float s[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31);
    float *out = blockIdx.y == 0 ? dweight : blockIdx.y == 1 ? dbias : dscale;
    if (!out) return;
    const float v = sum_rows(part + static_cast<long long>(blockIdx.y) * cols + col, rows, 3ll * cols, col < cols, s);
    if (threadIdx.x < 32 && col < cols) out[col] = v;
}

}  // namespace ptq
