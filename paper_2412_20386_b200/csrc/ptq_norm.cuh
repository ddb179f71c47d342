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

template <typename T, typename R, int kRB, bool kBackward, bool kWhole>
__global__ void __launch_bounds__(kRB > 1 ? 256 : 1024) ptq_norm_kernel(const NormParams p)
{
    constexpr int kStages = 3;
    __shared__ float s_sum[2][kStages][2 * kRB * kNormMaxWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int c = threadIdx.x * 8, cn = max(min(8, p.cols - c), 0);
    float weight[8], bias[8], scale[8];
    float sum_w[8], sum_b[8], sum_s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        weight[e] = e < cn ? (p.weight ? p.weight[c + e] : 1.0f) : 0.0f;
        bias[e] = e < cn && p.bias ? p.bias[c + e] : 0.0f;
        scale[e] = e < cn && p.scale ? p.scale[c + e] : 1.0f;
        if (kBackward) sum_w[e] = sum_b[e] = sum_s[e] = 0.0f;
    }
    int parity = 0;
    for (long long m0 = static_cast<long long>(blockIdx.x) * kRB; m0 < p.rows; m0 += static_cast<long long>(gridDim.x) * kRB, parity ^= 1) {
        Piece<T, 8> x[kRB], g[kRB], dy[kRB];
        Piece<R, 8> res[kRB], dres[kRB];
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            const long long m = m0 + i;
            const int n = m < p.rows ? cn : 0;
            x[i] = load_piece<kWhole, T, 8>(static_cast<const T *>(p.x) + m * p.x_l + c, n);
            if (p.residual) res[i] = load_piece<kWhole, R, 8>(static_cast<const R *>(p.residual) + m * p.residual_l + c, n);
            if (p.gate) g[i] = load_piece<kWhole, T, 8>(static_cast<const T *>(p.gate) + m * p.gate_l + c, n);
            if (kBackward) {
                dy[i] = load_piece<kWhole, T, 8>(static_cast<const T *>(p.dy) + m * p.cols + c, n);
                if (p.dresidual_out) dres[i] = load_piece<kWhole, R, 8>(static_cast<const R *>(p.dresidual_out) + m * p.cols + c, n);
            }
        }
        float r[kRB][8], mean[kRB], rstd[kRB];
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            mean[i] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v = x[i][e];
                if (p.gate_at == kGateIn) v *= g[i][e] * sigmoid_f32(g[i][e]);
                if (p.scale) v *= scale[e];
                r[i][e] = p.residual ? v + res[i][e] : v;
                mean[i] += r[i][e];
            }
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
                for (int e = 0; e < 8; ++e) {
                    y[e] = fmaf(r[i][e], weight[e], bias[e]);
                    if (p.gate_at == kGateOut) y[e] *= g[i][e] * sigmoid_f32(g[i][e]);
                }
                store_piece<kWhole, T, 8>(static_cast<T *>(p.y) + (m0 + i) * p.cols + c, y, cn);
            }
        } else {
            float sums[2 * kRB], dn[kRB][8];
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                sums[2 * i] = sums[2 * i + 1] = 0.0f;
                float dg[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float d = dy[i][e];
                    if (p.gate_at == kGateOut) {
                        const float z = g[i][e], s = sigmoid_f32(z);
                        dg[e] = d * fmaf(r[i][e], weight[e], bias[e]) * s * fmaf(z, 1.0f - s, 1.0f);
                        d *= z * s;
                    }
                    sum_w[e] = fmaf(d, r[i][e], sum_w[e]);
                    sum_b[e] += d;
                    dn[i][e] = d * weight[e];
                    sums[2 * i] = fmaf(dn[i][e], r[i][e], sums[2 * i]);
                    sums[2 * i + 1] += dn[i][e];
                }
                if (p.gate_at == kGateOut && m0 + i < p.rows) store_piece<kWhole, T, 8>(static_cast<T *>(p.dgate) + (m0 + i) * p.cols + c, dg, cn);
            }
            row_sums<2 * kRB>(sums, s_sum[parity][2], warp, warps, lane);
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                if (m0 + i >= p.rows) break;
                const float along = sums[2 * i] * p.inv_cols, flat = p.layer ? sums[2 * i + 1] * p.inv_cols : 0.0f;
                float dr[8], dx[8], dg[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dr[e] = (fmaf(-r[i][e], along, dn[i][e]) - flat) * rstd[i];
                    if (p.dresidual_out) dr[e] += dres[i][e];
                    dx[e] = dr[e] * scale[e];
                    float v = x[i][e];
                    if (p.gate_at == kGateIn) {
                        const float z = g[i][e], s = sigmoid_f32(z);
                        dg[e] = dx[e] * v * s * fmaf(z, 1.0f - s, 1.0f);
                        dx[e] *= z * s;
                        v *= z * s;
                    }
                    sum_s[e] = fmaf(dr[e], v, sum_s[e]);
                }
                const long long at = (m0 + i) * p.cols + c;
                store_piece<kWhole, T, 8>(static_cast<T *>(p.dx) + at, dx, cn);
                if (p.dresidual) store_piece<kWhole, R, 8>(static_cast<R *>(p.dresidual) + at, dr, cn);
                if (p.gate_at == kGateIn) store_piece<kWhole, T, 8>(static_cast<T *>(p.dgate) + at, dg, cn);
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

// Column sums of the CTAs' shares, in the order of the CTAs: part[rows][3][cols].
__global__ void __launch_bounds__(256) ptq_norm_finish_kernel(const float *part, int rows, int cols, float *dweight, float *dbias, float *dscale)
{
    __shared__ float s[8][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, col = blockIdx.x * 32 + x;
    float *out = blockIdx.y == 0 ? dweight : blockIdx.y == 1 ? dbias : dscale;
    if (!out) return;
    float v = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int r = y; r < rows; r += 8) v += part[(static_cast<long long>(r) * 3 + blockIdx.y) * cols + col];
    }
    s[y][x] = v;
    __syncthreads();
    if (y == 0 && col < cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += s[i][x];
        out[col] = v;
    }
}

}  // namespace ptq
