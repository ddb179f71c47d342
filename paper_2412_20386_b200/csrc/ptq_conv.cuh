// Short causal depthwise convolution between in_proj and x_proj.  For step i of a sequence (token i, or len-1-i reversed):
//
//   pre[i,d] = bias[d] + sum_j weight[d,j] x[i - (W-1) + j, d],   y = silu(pre)  (or pre)
//
// where the W-1 steps in front of the first one are the caller's state (zeros without one).  Bound: the bytes.  A thread
// holds four channels and walks over a segment of steps with the last W - 1 rows in registers, its loads kConvAhead rows ahead.
// Measured, 64 x 197 x 768 binary16, W = 4: forward 16 us (2.4 TB/s), backward 30 us (2 TB/s): both wait for loads, of which a thread has
// few in flight; eight channels a thread took 40 and 56, the bytes alone 6 and 9.
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
    long long way;                    // tokens between two steps of the sequence
    const T *first;                   // the token of step 0
    __device__ __forceinline__ ConvRow(const ConvParams &q, int b_, int piece) : p(q), b(b_), c(piece * kE)
    {
        cn = max(min(kE, p.channels - c), 0);
        len = p.lengths ? min(max(p.lengths[b], 0), p.length) : p.length;
        const bool reverse = p.flags & kConvReverse;
        way = reverse ? -1 : 1;
        first = static_cast<const T *>(p.x) + b * p.x_b + (reverse ? len - 1ll : 0ll) * p.x_l + c;
    }
    __device__ __forceinline__ long long token(int i) const { return (p.flags & kConvReverse) && i < len ? len - 1 - i : i; }
    // step i of the sequence with its state in front: i from -(W-1) on; zeros behind the end
    __device__ __forceinline__ Piece<T, kE> input(int i) const
    {
        if (i < 0)
            return load_piece<kWhole, T, kE>(static_cast<const T *>(p.state) + (static_cast<long long>(b) * (kW - 1) + (i + kW - 1)) * p.channels + c,
                                             p.state ? cn : 0);
        return step(i);
    }
    __device__ __forceinline__ Piece<T, kE> step(int i) const { return load_piece<kWhole, T, kE>(first + way * i * p.x_l, i < len ? cn : 0); }
    __device__ __forceinline__ long long dense(int i) const { return (static_cast<long long>(b) * p.length + token(i)) * p.channels + c; }
};

// Weights and bias of a thread's channels.
template <int kE, int kW, bool kWhole>
__device__ __forceinline__ void conv_weights(const ConvParams &p, int c, int cn, float (&w)[kW][kE], float (&bias)[kE])
{
    float f[kE * kW];                 // the channels' weights lie one behind the other
    const Piece<float, kE> b = load_piece<kWhole, float, kE>(p.bias + c, p.bias ? cn : 0);
    const Piece<float, kE * kW> all = load_piece<kWhole, float, kE * kW>(p.weight + static_cast<long long>(c) * kW, cn * kW);
#pragma unroll
    for (int i = 0; i < kE * kW; ++i) f[i] = all[i];
#pragma unroll
    for (int e = 0; e < kE; ++e) {
#pragma unroll
        for (int j = 0; j < kW; ++j) w[j][e] = f[e * kW + j];
        bias[e] = b[e];
    }
}

// pre of the newest row of the window
template <int kE, int kW>
__device__ __forceinline__ void conv_row(float (&v)[kE], const float (&w)[kW][kE], const float (&x)[kW][kE], const float (&bias)[kE])
{
#pragma unroll
    for (int e = 0; e < kE; ++e) v[e] = bias[e];
#pragma unroll
    for (int j = 0; j < kW; ++j) fma_each<kE>(v, w[j], x[j], v);
}
template <int kE, int kW>
__device__ __forceinline__ void conv_shift(float (&x)[kW][kE])
{
#pragma unroll
    for (int j = 0; j < kW - 1; ++j)
#pragma unroll
        for (int e = 0; e < kE; ++e) x[j][e] = x[j + 1][e];
}

constexpr int kConvE = 4;             // channels of a thread: with eight, weights and window leave too few warps
// Rows that are loaded together, one set under way while the other is worked on.  With four the call above takes 56 us, with eight 66, of
// which two take 50: the warps that the registers cost weigh more.
constexpr int kConvAhead = 2;

template <typename T, int kW, bool kWhole>
__global__ void __launch_bounds__(256) ptq_conv_kernel(const ConvParams p)
{
    constexpr int kE = kConvE;
    const long long idx = blockIdx.x * 256ll + threadIdx.x;
    const long long row = idx / p.pieces;
    if (row >= static_cast<long long>(p.batch) * p.segments) return;
    const int seg = static_cast<int>(row % p.segments);
    const ConvRow<T, kE, kW, kWhole> in(p, static_cast<int>(row / p.segments), static_cast<int>(idx - row * p.pieces));
    const int i0 = seg * p.segment, i1 = min(i0 + p.segment, in.len);
    Piece<T, kE> before[kW - 1], next[kConvAhead];
#pragma unroll
    for (int j = 0; j < kW - 1; ++j) before[j] = in.input(i0 - (kW - 1) + j);
#pragma unroll
    for (int a = 0; a < kConvAhead; ++a) next[a] = in.step(i0 + a);
    float w[kW][kE], bias[kE], x[kW][kE];
    conv_weights<kE, kW, kWhole>(p, in.c, in.cn, w, bias);
#pragma unroll
    for (int j = 0; j < kW - 1; ++j)
#pragma unroll
        for (int e = 0; e < kE; ++e) x[j][e] = before[j][e];
    // the thread that reads the state replaces it: the two may be one buffer
    if (seg == 0 && p.final_state) {
        T *out = static_cast<T *>(p.final_state) + static_cast<long long>(in.b) * (kW - 1) * p.channels + in.c;
        Piece<T, kE> last[kW - 1];
#pragma unroll
        for (int j = 0; j < kW - 1; ++j) last[j] = in.input(in.len - (kW - 1) + j);
#pragma unroll
        for (int j = 0; j < kW - 1; ++j) store_piece<kWhole, T, kE>(out + static_cast<long long>(j) * p.channels, last[j], in.cn);
    }
    T *y = static_cast<T *>(p.y) + in.dense(i0);
    const long long y_step = in.way * p.channels;
    for (int i = i0; i < i1; i += kConvAhead) {
        Piece<T, kE> now[kConvAhead];
#pragma unroll
        for (int a = 0; a < kConvAhead; ++a) {
            now[a] = next[a];
            next[a] = in.step(i + kConvAhead + a);
        }
#pragma unroll
        for (int a = 0; a < kConvAhead; ++a) {
            float v[kE];
#pragma unroll
            for (int e = 0; e < kE; ++e) x[kW - 1][e] = now[a][e];
            conv_row<kE, kW>(v, w, x, bias);
            if (p.flags & kConvSilu) {
#pragma unroll
                for (int e = 0; e < kE; ++e) v[e] *= sigmoid_f32(v[e]);
            }
            conv_shift<kE, kW>(x);
            if (i + a < i1) store_piece<kWhole, T, kE>(y, v, in.cn);
            y += y_step;
        }
    }
}

// Gradients: dpre = dy silu'(pre) of the segment's outputs and of the W - 1 behind it gives dx of the segment,
// dx[i] = sum_j weight[j] dpre[i + (W-1) - j], and x times dpre of the segment's own outputs dweight.  A warp takes 32 pieces of a
// segment, goes on to others and keeps the sums of dweight and dbias in registers.
template <typename T, int kW, bool kWhole>
__global__ void __launch_bounds__(256, 2) ptq_conv_backward_kernel(const ConvParams p)
{
    constexpr int kE = kConvE;
    __shared__ float s_sum[8][32 * kE];
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int piece = blockIdx.x * 32 + lane;
    const int c = piece * kE, cn = max(min(kE, p.channels - c), 0);
    float w[kW][kE], bias[kE], dw[kW][kE], db[kE];
    conv_weights<kE, kW, kWhole>(p, c, cn, w, bias);
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
        const int tail = in.len - (kW - 1);               // step of the final state's first row
        const int last = end + kW - 1;                    // behind the last output whose dpre is needed
        const T *dy0 = static_cast<const T *>(p.dy) + (static_cast<long long>(in.b) * p.length + (in.way < 0 ? in.len - 1 : 0)) * p.channels + c;
        const auto dy_of = [&](int o) { return load_piece<kWhole, T, kE>(dy0 + in.way * o * p.channels, o < in.len && o < last ? cn : 0); };
        Piece<T, kE> before[kW - 1], next_x[kConvAhead], next_dy[kConvAhead];
#pragma unroll
        for (int j = 0; j < kW - 1; ++j) before[j] = in.input(i0 - (kW - 1) + j);
#pragma unroll
        for (int a = 0; a < kConvAhead; ++a) {
            next_x[a] = in.step(i0 + a);
            next_dy[a] = dy_of(i0 + a);
        }
        float x[kW][kE], d[kW][kE];                        // rows o-(W-1) .. o; dpre of the same rows
#pragma unroll
        for (int j = 0; j < kW - 1; ++j)
#pragma unroll
            for (int e = 0; e < kE; ++e) {
                x[j][e] = before[j][e];
                d[j][e] = 0.0f;                            // outputs in front of the segment: no dx of it needs them
            }
        for (int o0 = i0; o0 < last; o0 += kConvAhead) {
            Piece<T, kE> now_x[kConvAhead], now_dy[kConvAhead];
#pragma unroll
            for (int a = 0; a < kConvAhead; ++a) {
                now_x[a] = next_x[a];
                now_dy[a] = next_dy[a];
                if (o0 + kConvAhead < last) {
                    next_x[a] = in.step(o0 + kConvAhead + a);
                    next_dy[a] = dy_of(o0 + kConvAhead + a);
                }
            }
#pragma unroll
            for (int a = 0; a < kConvAhead; ++a) {
                const int o = o0 + a;
                float v[kE], g[kE], out[kE];
#pragma unroll
                for (int e = 0; e < kE; ++e) {
                    x[kW - 1][e] = now_x[a][e];
                    g[e] = now_dy[a][e];
                }
                if (p.flags & kConvSilu) {
                    conv_row<kE, kW>(v, w, x, bias);
#pragma unroll
                    for (int e = 0; e < kE; ++e) {
                        const float s = sigmoid_f32(v[e]);
                        g[e] *= s * fmaf(v[e], 1.0f - s, 1.0f);
                    }
                }
#pragma unroll
                for (int e = 0; e < kE; ++e) {
                    if (o >= in.len || o >= last) g[e] = 0.0f;
                    d[kW - 1][e] = g[e];
                    if (o >= i1) g[e] = 0.0f;              // the next segment's own
                    db[e] += g[e];
                    out[e] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < kW; ++j) {
                    fma_each<kE>(dw[j], g, x[j], dw[j]);
                    fma_each<kE>(out, w[j], d[kW - 1 - j], out);
                }
                conv_shift<kE, kW>(x);
                conv_shift<kE, kW>(d);
                const int i = o - (kW - 1);                // the step whose gradient is complete now
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
                        store_piece<kWhole, T, kE>(static_cast<T *>(p.dstate) + (static_cast<long long>(in.b) * (kW - 1) + (i + kW - 1)) * p.channels + c,
                                                   out, cn);
                }
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
    griddep_wait();
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), j = blockIdx.y;
    if (j == taps && !dbias) return;
    const float v = sum_rows<32>(part + static_cast<long long>(j) * cols + col, rows, static_cast<long long>(taps + 1) * cols, col < cols, s);
    if (threadIdx.x >= 32 || col >= cols) return;
    if (j < taps)
        dweight[static_cast<long long>(col) * taps + j] = v;
    else
        dbias[col] = v;
}

}  // namespace ptq
