// Short causal depthwise convolution between in_proj and x_proj.  For step i of a sequence (token i, or len-1-i reversed):
//
//   pre[i,d] = bias[d] + sum_j weight[d,j] x[i - (W-1) + j, d],   y = silu(pre)  (or pre)
//
// where the W-1 steps in front of the first one are the caller's state (zeros without one).  Bound: the bytes.  A thread
// holds a few channels and walks over a segment of steps with the last W - 1 rows in registers, its loads kAhead rows ahead.
#pragma once

#include "ptq_block.cuh"

namespace ptq {

constexpr unsigned kConvSilu = 1u, kConvReverse = 2u;

struct ConvParams {
    const void *x, *state;            // state [batch][W-1][channels], may be null
    long long x_b, x_l;               // pitches in elements
    const float *weight, *bias;       // [channels][W]; bias may be null
    const int *lengths;               // may be null
    int batch, length, channels;
    int segment, segments;            // steps of a segment (at least W-1), segments of a sequence
    int pieces;                       // pieces of a row
    unsigned flags;
    void *y, *final_state;            // dense; final_state may be null or the state itself
    // backward
    const void *dy, *dfinal;
    void *dx, *dstate;
    float *part;                      // [gridDim.y][W + 1][channels]
};

template <typename T, int kE, int kW, bool kWhole>
struct ConvRow {
    const ConvParams &p;
    int b, c, cn, len;
    __device__ __forceinline__ ConvRow(const ConvParams &q, int b_, int piece) : p(q), b(b_), c(piece * kE)
    {
        cn = max(min(kE, p.channels - c), 0);
        len = p.lengths ? min(max(p.lengths[b], 0), p.length) : p.length;
    }
    __device__ __forceinline__ long long token(int i) const { return (p.flags & kConvReverse) && i < len ? len - 1 - i : i; }
    // row i of the sequence with its state in front: i from -(W-1) on; zeros behind the end
    __device__ __forceinline__ Piece<T, kE> input(int i) const
    {
        if (i < 0)
            return load_piece<kWhole, T, kE>(static_cast<const T *>(p.state) + (static_cast<long long>(b) * (kW - 1) + (i + kW - 1)) * p.channels + c,
                                     p.state ? cn : 0);
        return load_piece<kWhole, T, kE>(static_cast<const T *>(p.x) + b * p.x_b + token(min(i, p.length - 1)) * p.x_l + c, i < len ? cn : 0);
    }
    __device__ __forceinline__ long long dense(int i) const { return (static_cast<long long>(b) * p.length + token(i)) * p.channels + c; }
};

template <typename T, int kE, int kW>
__device__ __forceinline__ void conv_weights(const ConvParams &p, int c, int cn, float (&w)[kW][kE], float (&bias)[kE])
{
#pragma unroll
    for (int e = 0; e < kE; ++e) {
#pragma unroll
        for (int j = 0; j < kW; ++j) w[j][e] = e < cn ? __ldg(p.weight + static_cast<long long>(c + e) * kW + j) : 0.0f;
        bias[e] = p.bias && e < cn ? __ldg(p.bias + c + e) : 0.0f;
    }
}

template <typename T, int kE, int kW, bool kWhole>
__global__ void __launch_bounds__(256) ptq_conv_kernel(const ConvParams p)
{
    constexpr int kAhead = 4;
    const long long idx = blockIdx.x * 256ll + threadIdx.x;
    const long long row = idx / p.pieces;
    if (row >= static_cast<long long>(p.batch) * p.segments) return;
    const int seg = static_cast<int>(row % p.segments);
    const ConvRow<T, kE, kW, kWhole> in(p, static_cast<int>(row / p.segments), static_cast<int>(idx - row * p.pieces));
    float w[kW][kE], bias[kE], x[kW][kE];
    conv_weights<T, kE, kW>(p, in.c, in.cn, w, bias);
    const int i0 = seg * p.segment, i1 = min(i0 + p.segment, in.len);
#pragma unroll
    for (int j = 0; j < kW - 1; ++j) {
        const Piece<T, kE> v = in.input(i0 - (kW - 1) + j);
#pragma unroll
        for (int e = 0; e < kE; ++e) x[j][e] = v[e];
    }
    // the thread that reads the state replaces it: the two may be one buffer
    if (seg == 0 && p.final_state) {
        T *out = static_cast<T *>(p.final_state) + static_cast<long long>(in.b) * (kW - 1) * p.channels + in.c;
        Piece<T, kE> last[kW - 1];
#pragma unroll
        for (int j = 0; j < kW - 1; ++j) last[j] = in.input(in.len - (kW - 1) + j);
#pragma unroll
        for (int j = 0; j < kW - 1; ++j) {
            float f[kE];
#pragma unroll
            for (int e = 0; e < kE; ++e) f[e] = last[j][e];
            store_piece<kWhole, T, kE>(out + static_cast<long long>(j) * p.channels, f, in.cn);
        }
    }
    for (int i = i0; i < i1; i += kAhead) {
        Piece<T, kE> next[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) next[a] = in.input(min(i + a, i1 - 1));
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            float y[kE];
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                x[kW - 1][e] = next[a][e];
                float v = bias[e];
#pragma unroll
                for (int j = 0; j < kW; ++j) v = fmaf(w[j][e], x[j][e], v);
                y[e] = p.flags & kConvSilu ? v * sigmoid_f32(v) : v;
#pragma unroll
                for (int j = 0; j < kW - 1; ++j) x[j][e] = x[j + 1][e];
            }
            if (i + a < i1) store_piece<kWhole, T, kE>(static_cast<T *>(p.y) + in.dense(i + a), y, in.cn);
        }
    }
}

// Gradients: dpre = dy silu'(pre) of the segment's outputs and of the W - 1 behind it gives dx of the segment,
// dx[i] = sum_j weight[j] dpre[i + (W-1) - j], and x times dpre of the segment's own outputs dweight.  A warp takes 32 pieces of a
// segment, goes on to others and keeps the sums of dweight and dbias in registers.
template <typename T, int kE, int kW, bool kWhole>
__global__ void __launch_bounds__(256) ptq_conv_backward_kernel(const ConvParams p)
{
    __shared__ float s_sum[8][32 * kE];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int piece = blockIdx.x * 32 + lane;
    const int c = piece * kE, cn = max(min(kE, p.channels - c), 0);
    float w[kW][kE], bias[kE], dw[kW][kE], db[kE];
    conv_weights<T, kE, kW>(p, c, cn, w, bias);
#pragma unroll
    for (int e = 0; e < kE; ++e) {
        db[e] = 0.0f;
#pragma unroll
        for (int j = 0; j < kW; ++j) dw[j][e] = 0.0f;
    }
    const long long total = static_cast<long long>(p.batch) * p.segments;
    for (long long row = blockIdx.y * 8ll + warp; row < total && cn > 0; row += gridDim.y * 8ll) {
        const int seg = static_cast<int>(row % p.segments);
        const ConvRow<T, kE, kW, kWhole> in(p, static_cast<int>(row / p.segments), piece);
        const int i0 = seg * p.segment, end = min(i0 + p.segment, p.length), i1 = min(end, in.len);
        const int first = seg == 0 ? -(kW - 1) : i0;      // the first segment makes the state's gradient too
        float x[kW][kE], d[kW][kE];                        // rows o-(W-1) .. o; dpre of the same rows
#pragma unroll
        for (int j = 0; j < kW - 1; ++j) {
            const Piece<T, kE> v = in.input(i0 - (kW - 1) + j);
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                x[j][e] = v[e];
                d[j][e] = 0.0f;
            }
        }
        // outputs o = i0 .. ; d of outputs in front of the segment is of no use to it, in front of the sequence it is zero
        const int tail = in.len - (kW - 1);               // step of the final state's first row
        Piece<T, kE> nx = in.input(i0), nd;
        const auto dy_of = [&](int o) {
            return load_piece<kWhole, T, kE>(static_cast<const T *>(p.dy) + in.dense(min(o, p.length - 1)), o < in.len ? cn : 0);
        };
        nd = dy_of(i0);
        for (int o = i0; o < end + kW - 1; ++o) {
            const Piece<T, kE> vx = nx, vd = nd;
            if (o + 1 < end + kW - 1) {
                nx = in.input(o + 1);
                nd = dy_of(o + 1);
            }
            const bool on = o < in.len, own = o < i1;
            float out[kE];
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                x[kW - 1][e] = vx[e];
                float v = bias[e];
#pragma unroll
                for (int j = 0; j < kW; ++j) v = fmaf(w[j][e], x[j][e], v);
                float g = vd[e];
                if (p.flags & kConvSilu) {
                    const float s = sigmoid_f32(v);
                    g *= s * fmaf(v, 1.0f - s, 1.0f);
                }
                d[kW - 1][e] = on ? g : 0.0f;
                if (own) {
                    db[e] += g;
#pragma unroll
                    for (int j = 0; j < kW; ++j) dw[j][e] = fmaf(g, x[j][e], dw[j][e]);
                }
                out[e] = 0.0f;
#pragma unroll
                for (int j = 0; j < kW; ++j) out[e] = fmaf(w[j][e], d[kW - 1 - j][e], out[e]);
#pragma unroll
                for (int j = 0; j < kW - 1; ++j) {
                    x[j][e] = x[j + 1][e];
                    d[j][e] = d[j + 1][e];
                }
            }
            const int i = o - (kW - 1);                    // the step whose gradient is complete now
            if (i >= first && i < end) {
                if (p.dfinal && i >= tail && i < in.len) {
                    const Piece<T, kE> f = load_piece<kWhole, T, kE>(
                        static_cast<const T *>(p.dfinal) + (static_cast<long long>(in.b) * (kW - 1) + (i - tail)) * p.channels + c, cn);
#pragma unroll
                    for (int e = 0; e < kE; ++e) out[e] += f[e];
                }
                if (i >= 0)
                    store_piece<kWhole, T, kE>(static_cast<T *>(p.dx) + in.dense(i), out, cn);
                else if (p.dstate)
                    store_piece<kWhole, T, kE>(static_cast<T *>(p.dstate) + (static_cast<long long>(in.b) * (kW - 1) + (i + kW - 1)) * p.channels + c, out,
                                       cn);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kW + 1; ++j) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kE; ++e) s_sum[warp][lane * kE + e] = j < kW ? dw[j < kW ? j : 0][e] : db[e];
        __syncthreads();
        for (int i = threadIdx.x; i < 32 * kE; i += 256) {
            const int col = blockIdx.x * 32 * kE + i;
            if (col >= p.channels) continue;
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) v += s_sum[k][i];
            p.part[(static_cast<long long>(blockIdx.y) * (kW + 1) + j) * p.channels + col] = v;
        }
    }
}

// Sums of the CTAs' shares: part[rows][W + 1][cols] -> dweight [cols][W], dbias [cols].
__global__ void __launch_bounds__(1024) ptq_conv_finish_kernel(const float *part, int rows, int cols, int taps, float *dweight, float *dbias)
{
    __shared__ float s[32][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), j = blockIdx.y;
    if (j == taps && !dbias) return;
    const float v = sum_rows(part + static_cast<long long>(j) * cols + col, rows, static_cast<long long>(taps + 1) * cols, col < cols, s);
    if (threadIdx.x >= 32 || col >= cols) return;
    if (j < taps)
        dweight[static_cast<long long>(col) * taps + j] = v;
    else
        dbias[col] = v;
}

}  // namespace ptq
