// Gated linear recurrence between dt_proj and out_proj.  For step i of a sequence (token p = i, or len-1-i reversed),
// channel d with its group g of B and C, and state n:
//
//   dt = softplus(delta[p,d] + delta_bias[d])           (or without softplus)
//   h[n] <- exp(dt A[d,n]) h[n] + dt u[p,d] B[p,g,n]
//   o = sum_n C[p,g,n] h[n] + D[d] u[p,d],   y[p,d] = o silu(z[p,d])
//
// Bound: the port on which exponentials and shared-memory reads return to the registers (16 powers of two of a warp 71 cycles with three warps
// per scheduler, with four 16-byte reads beside them 135), from N = 4 or so on; below that issue slots and bytes.  A warp works alone on 32 kC / kS channels: kS neighbouring lanes hold the states of a channel, kNS each, and kC channels
// (N = 16 and many rows: two lanes, two channels, eight states), in registers.  A tile is 256 elements: its lanes load eight channels of one
// row each (the next tile's are under way meanwhile), put dt and dt u into shared memory, run the recurrence, and finish the rows that they
// loaded; no barrier but the warp's.  Few rows: the steps are cut into chunks.  A first launch computes what each
// chunk adds to the state and by how much it decays (exp(A sum dt)), the second folds these into the state it starts a chunk from.
// Measured, N = 16: 128 x 197 x 768 binary16 135 us (the N + 3 exponentials per element
// alone: 45), of which 100 us is the recurrence by itself; CTAs of four
// warps that shared a tile took 180, one channel per lane 137 to 190 (every value of B and C read from shared memory for 8 decays
// instead of 16), loads whose 16-bit values were taken apart on arrival 220.  A quarter
// of the decays by polynomial on the multiply-add pipe: 137 -> 154.  2 x 20011 x 1024 bfloat16 466 us in two launches (exponentials
// of one pass 95).  1 x 197 x 384: 10.2 us in two launches of chunks of 32 steps, 18.4 in one.
#pragma once

#include "ptq_block.cuh"

namespace ptq {

constexpr int kScanHistory = 8;       // steps between two states that are kept for the backward pass
constexpr int kScanWarps = 4;         // of a CTA; the forward pass's work alone

constexpr unsigned kScanSoftplus = 1u, kScanReverse = 2u;

struct ScanParams {
    const void *u, *delta, *z, *B, *C;          // z may be null
    long long u_b, u_l, delta_b, delta_l, z_b, z_l, B_b, B_l, B_g, C_b, C_l, C_g;      // pitches in elements
    const float *A, *D, *delta_bias, *state;    // all but A may be null
    const int *lengths;                         // may be null
    int batch, length, channels, states, groups;
    int group_channels;                         // channels / groups
    int group_warps, group_blocks;              // warps (CTAs of the backward pass) that share the channels of a group
    int chunk_len, chunks;
    unsigned flags;
    int unit;                                   // channels that an access of general rows may take: 4, 2 or 1
    int bc_unit;                                // the same of the states of B and C
    float *slots;                               // [chunks][batch][channels][states]
    float *sums;                                // [chunks][batch][channels]: sum of dt of a chunk
    // forward
    void *y;                                    // dense
    float *final_state, *history;
    // backward
    const void *dy;                             // dense
    const float *dfinal, *kept;                 // dfinal may be null; kept: the forward pass's history
    void *du, *ddelta, *dz, *dB, *dC;           // dense
    float *dstate;
    float *part_A, *part_D, *part_bias;         // [batch * chunks][channels (states)]
    float *part_BC;                             // [groups * group_blocks][batch][length][2 states], null: straight to dB, dC
};

// Of two values: t = e^-|x| and log(1 + e^x) = max(x, 0) + log(1 + t).  The argument of the power of two is carried to about 2^-46
// (its rounding alone would cost four units in the last place at |x| = 7); |x| is cut at 126, where t is zero.  log(1 + t) / t is a
// polynomial fitted on [0, 1]; with the coefficients as written, log(1 + t) is high by up to 2.3e-8, 3.4e-8 relative (half a unit in the last place),
// small results too, with half the instructions of expf and log1pf.
__device__ __forceinline__ void exp_minus_abs_pair(float &t0, float &t1, float x0, float x1)
{
    const float m0 = -fminf(fabsf(x0), 126.0f), m1 = -fminf(fabsf(x1), 126.0f);
    float y0, y1, r0, r1;
    mul_pair(y0, y1, m0, m1, kLog2e, kLog2e);
    fma_pair(r0, r1, m0, m1, kLog2e, kLog2e, -y0, -y1);
    fma_pair(r0, r1, m0, m1, 1.925963033e-8f, 1.925963033e-8f, r0, r1);
    y0 = exp2_approx(y0);
    y1 = exp2_approx(y1);
    mul_pair(r0, r1, r0, r1, kLn2, kLn2);
    fma_pair(t0, t1, y0, y1, r0, r1, y0, y1);
}
__device__ __forceinline__ void softplus_pair(float &s0, float &s1, float x0, float x1, float t0, float t1)
{
    constexpr float kCoeff[] = {0.01985144429f, -0.05695949867f, 0.106036514f, -0.1530559063f, 0.1967593879f,
                                -0.2495413423f, 0.3332996368f,   -0.4999990165f, 1.0f};
    float p0 = -0.0032440212f, p1 = p0;
#pragma unroll
    for (float k : kCoeff) fma_pair(p0, p1, p0, p1, t0, t1, k, k);
    fma_pair(s0, s1, p0, p1, t0, t1, x0 <= 0.0f ? 0.0f : x0, x1 <= 0.0f ? 0.0f : x1);      // NaN passes through
}
__device__ __forceinline__ float softplus_f32(float x)
{
    float t, s, unused;
    exp_minus_abs_pair(t, unused, x, 0.0f);
    softplus_pair(s, unused, x, 0.0f, t, 1.0f);
    return s;
}

// exp(dt A) as 2^(dt rate).  The hardware's power of two is low by 0.1 to 0.35 units of 2^-24 on average for the arguments of slow
// decays (-0.1 .. 0), where a state multiplies hundreds of them: the argument is raised by a quarter of a unit, which the fused
// multiply-add does at no cost and which rounds away where the memory is short.  2^kDecayShift is 1: a step with dt = 0 keeps the state.
constexpr float kDecayShift = 2.15e-8f;
template <int kNS>
__device__ __forceinline__ void scan_decays(float (&a)[kNS], float dt, const float (&rate)[kNS])
{
    float shift[kNS];
#pragma unroll
    for (int k = 0; k < kNS; ++k) shift[k] = kDecayShift;
    fma_each<kNS>(a, dt, rate, shift);
#pragma unroll
    for (int k = 0; k < kNS; ++k) a[k] = exp2_approx(a[k]);
}

// Decay rates times log2(e); no infinities, so that a step without a token (dt = 0) leaves the state as it is.
__device__ __forceinline__ float scan_rate(float a) { return a != a ? a : fminf(fmaxf(a * kLog2e, -3.0e38f), 3.0e38f); }

struct ScanBlock {
    int b, chunk, g, c0, c_end, len, i0, i1;
    // block: which of the shares of `width` channels (group_blocks to a group) of which chunk of which sequence
    __device__ __forceinline__ ScanBlock(const ScanParams &p, int block, int group_blocks, int chunks, int first_chunk, int width)
    {
        const int per = p.groups * group_blocks;
        const int rest = block / per, blk = block - rest * per;
        b = rest / chunks;
        chunk = first_chunk + rest - b * chunks;
        g = blk / group_blocks;
        c0 = g * p.group_channels + (blk - g * group_blocks) * width;
        c_end = min(c0 + width, (g + 1) * p.group_channels);
        len = p.lengths ? min(max(p.lengths[b], 0), p.length) : p.length;
        i0 = chunk * p.chunk_len;
        i1 = min(i0 + min(p.chunk_len, p.length - i0), len);
    }
};

// The square root of a chunk's decay 2^(rate s).  Multiplied in twice it takes a state over a chunk whose decay itself leaves binary32: states that
// grow (rates above zero, negative dt) by 2^138 in 32 steps of e^3, from nothing or from little.  It is kept finite and above zero, so that nothing
// times any growth is nothing and an infinite state stays one, as step by step.
__device__ __forceinline__ float chunk_decay_root(float rate, float s) { return exp2_approx(fminf(fmaxf(0.5f * (rate * s), -126.0f), 127.0f)); }

// The state that enters a chunk, from what the chunks between it and `first` add: slot j holds the sum of chunk j alone (that of the
// one next to the sequence's end holds the true state), sums[j] its dt.
template <bool kWhole, int kNS>
__device__ __forceinline__ void scan_fold(float (&h)[kNS], const float (&rate)[kNS], const ScanParams &p, int b, int d, int n0, int nn, int from,
                                          int to, int by)
{
    const long long row = static_cast<long long>(b) * p.channels + d, step = static_cast<long long>(p.batch) * p.channels;
    load_floats<kWhole, kNS>(h, p.slots + (from * step + row) * p.states + n0, nn);
#pragma unroll 4
    for (int j = from + by; j != to; j += by) {
        float v[kNS];
        load_floats<kWhole, kNS>(v, p.slots + (j * step + row) * p.states + n0, nn);
        const float s = p.sums[j * step + row];
#pragma unroll
        for (int k = 0; k < kNS; ++k) {
            const float half = chunk_decay_root(rate[k], s);
            h[k] = fmaf(half, half * h[k], v[k]);
        }
    }
}

// kMode 0: y and the final state.  1: the state that each chunk but the last one adds.  2: the same for the gradient of the
// state, from the last step to the first: e <- exp(dt A) (C dy silu(z) + e), for each chunk but the first one.
enum { kScanForward = 0, kScanSum = 1, kScanGradSum = 2 };

template <typename T, int kC, int kNS, int kS, int kMode, bool kWhole>
__global__ void __launch_bounds__(kScanWarps * 32, kC * kNS <= 2 ? 4 : 3) ptq_scan_kernel(const ScanParams p)
{
    constexpr int kWidth = 32 / kS * kC, kPitch = kWidth + 2;      // channels of the warp; the pad keeps the rows' lanes off each other's banks
    constexpr int kRows = 256 / kWidth, kNP = kNS * kS;            // steps of a tile, states padded
    constexpr int kGroup = kS < 4 ? 4 : kS;               // steps of an unrolled group
    constexpr bool kBackward = kMode == kScanGradSum;
    constexpr int kKinds = kMode == kScanForward ? 2 : 1; // B and C, or one of them
    constexpr int kPer = kNP >= 2 ? 2 : 1;                // their values in an access
    constexpr int kBC = (kRows * kNP + 32 * kPer - 1) / (32 * kPer);       // accesses of a lane to each
    __shared__ __align__(16) float2 s_pairs[kScanWarps][kRows * kPitch];                   // (dt, dt u), later (o, -)
    __shared__ __align__(16) float s_states[kScanWarps][kKinds * kRows * kNP];           // [B, C][step][state]
    griddep_wait();
    if (kMode != kScanForward) griddep_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long unit = blockIdx.x * static_cast<long long>(kScanWarps) + warp;
    const int chunks = kMode == kScanForward ? p.chunks : p.chunks - 1;
    if (unit >= static_cast<long long>(p.batch) * p.groups * p.group_warps * chunks) return;
    const ScanBlock blk(p, static_cast<int>(unit), p.group_warps, chunks, kBackward ? 1 : 0, kWidth);
    float2 *const s_pair = s_pairs[warp];
    float *const s_BC = s_states[warp];
    const bool softplus = p.flags & kScanSoftplus, reverse = p.flags & kScanReverse;
    const int n_steps = max(blk.i1 - blk.i0, 0);
    // step k of the chunk's loop is step i of the sequence, token first + k * way
    const int first_step = kBackward ? blk.i1 - 1 : blk.i0;
    const long long first = reverse ? blk.len - 1 - first_step : first_step;
    const int way = reverse != kBackward ? -1 : 1;

    // the lane's part of a row
    const int row = lane / (kWidth / 8), c = blk.c0 + lane % (kWidth / 8) * 8;
    const int cn = max(min(8, blk.c_end - c), 0);
    const long long tok = first + way * row;
    const T *at_u = kBackward ? static_cast<const T *>(p.dy) + (static_cast<long long>(blk.b) * p.length + tok) * p.channels + c
                              : static_cast<const T *>(p.u) + blk.b * p.u_b + tok * p.u_l + c;
    const T *at_delta = static_cast<const T *>(p.delta) + blk.b * p.delta_b + tok * p.delta_l + c;
    const T *at_z = static_cast<const T *>(p.z) + blk.b * p.z_b + tok * p.z_l + c;
    const long long next_u = way * kRows * (kBackward ? static_cast<long long>(p.channels) : p.u_l), next_delta = way * kRows * p.delta_l,
                    next_z = way * kRows * p.z_l;
    const bool gated = kMode != kScanSum && p.z;
    Piece<T, 8> r_u, r_delta, r_z;
    Piece<T, kPer> r_BC[kKinds][kBC];
    // the lane's first value of B and C in the tile: step t0, state n1; the others are kApart steps apart
    constexpr int kApart = kBC > 1 ? 32 * kPer / kNP : kRows;
    static_assert(kApart * kBC == kRows, "a fetch goes one tile on");
    const int t0 = kPer * lane / kNP, n1 = kPer * lane % kNP;
    const bool has = kPer * lane < kRows * kNP;
    const T *at_BC[kKinds];
    long long apart[kKinds];
#pragma unroll
    for (int j = 0; j < kKinds; ++j) {
        const bool is_C = kMode == kScanForward ? j == 1 : kBackward;
        const long long pitch = is_C ? p.C_l : p.B_l;
        at_BC[j] = is_C ? static_cast<const T *>(p.C) + blk.b * p.C_b + blk.g * p.C_g : static_cast<const T *>(p.B) + blk.b * p.B_b + blk.g * p.B_g;
        at_BC[j] += (first + way * t0) * pitch + n1;
        apart[j] = way * kApart * pitch;
    }
    const auto fetch = [&](int k0) {
        const int n = k0 + row < n_steps ? cn : 0;
        r_u = load_piece<kWhole, T, 8>(at_u, n, p.unit);
        r_delta = load_piece<kWhole, T, 8>(at_delta, n, p.unit);
        if (gated) r_z = load_piece<kWhole, T, 8>(at_z, n, p.unit);
        at_u += next_u;
        at_delta += next_delta;
        at_z += next_z;
#pragma unroll
        for (int j = 0; j < kKinds; ++j) {
#pragma unroll
            for (int i = 0; i < kBC; ++i) {
                const int states = has && k0 + t0 + i * kApart < n_steps ? p.states - n1 : 0;
                r_BC[j][i] = p.bc_unit >= 2 ? load_piece<true, T, kPer>(at_BC[j], states) : load_piece<false, T, kPer>(at_BC[j], states);
                at_BC[j] += apart[j];
            }
        }
    };
    if (n_steps > 0) fetch(0);
    const Piece<float, 8> bias = load_piece<kWhole, float, 8>(p.delta_bias + c, p.delta_bias ? cn : 0);

    // the lane's channels and states
    const int ch = lane / kS * kC, n0 = (lane % kS) * kNS, d = blk.c0 + ch;
    int nn[kC];
    float rate[kC][kNS], h[kC][kNS];
    const long long state_at = (static_cast<long long>(blk.b) * p.channels + d) * p.states + n0;
    const long long slot_step = static_cast<long long>(p.batch) * p.channels * p.states;
    float sum_dt[kC];
#pragma unroll
    for (int j = 0; j < kC; ++j) {
        nn[j] = d + j < blk.c_end ? max(min(kNS, p.states - n0), 0) : 0;
        load_floats<kWhole, kNS>(rate[j], p.A + static_cast<long long>(d + j) * p.states + n0, nn[j]);
#pragma unroll
        for (int n = 0; n < kNS; ++n) {
            rate[j][n] = scan_rate(rate[j][n]);
            h[j][n] = 0.0f;
        }
        sum_dt[j] = 0.0f;
        const long long at = state_at + j * p.states;
        if constexpr (kMode == kScanForward) {
            if (blk.chunk > 0) {
                if (nn[j] > 0) scan_fold<kWhole, kNS>(h[j], rate[j], p, blk.b, d + j, n0, nn[j], 1, blk.chunk + 1, 1);
            } else if (p.state) {
                load_floats<kWhole, kNS>(h[j], (p.chunks > 1 ? p.slots : p.state) + at, nn[j]);
            }
        } else if constexpr (kMode == kScanSum) {
            // chunk 0 starts from the true state; the second launch takes it from a copy, since the final state may replace it
            if (blk.chunk == 0 && p.state) {
                load_floats<kWhole, kNS>(h[j], p.state + at, nn[j]);
                store_floats<kWhole, kNS>(p.slots + at, h[j], nn[j]);
            }
        } else if (blk.chunk == p.chunks - 1 && p.dfinal) {
            load_floats<kWhole, kNS>(h[j], p.dfinal + at, nn[j]);
        }
    }
    T *at_y = static_cast<T *>(p.y) + (static_cast<long long>(blk.b) * p.length + tok) * p.channels + c;
    float *at_kept = nullptr;
    if (kMode == kScanForward && p.history)
        at_kept = p.history +
                  ((blk.b * static_cast<long long>((p.length + kScanHistory - 1) / kScanHistory) + blk.i0 / kScanHistory) * p.channels + d) * p.states + n0;

    float4 *const own = reinterpret_cast<float4 *>(s_pair + row * kPitch + lane % (kWidth / 8) * 8);      // what the lane fills and finishes
    for (int k0 = 0; k0 < n_steps; k0 += kRows) {
        const bool row_on = k0 + row < n_steps;
        const Piece<T, 8> u = r_u, z = r_z;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float4 f;
            f.x = r_delta[e] + bias[e];
            f.z = r_delta[e + 1] + bias[e + 1];
            if (softplus) {
                float t0, t1;
                exp_minus_abs_pair(t0, t1, f.x, f.z);
                softplus_pair(f.x, f.z, f.x, f.z, t0, t1);
            }
            f.y = r_u[e];
            f.w = r_u[e + 1];
            if constexpr (kBackward) {
                if (gated) {
                    f.y *= r_z[e] * sigmoid_f32(r_z[e]);
                    f.w *= r_z[e + 1] * sigmoid_f32(r_z[e + 1]);
                }
            } else {
                mul_pair(f.y, f.w, f.y, f.w, f.x, f.z);
            }
            if (!row_on) f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            own[e / 2] = f;
        }
#pragma unroll
        for (int j = 0; j < kKinds; ++j) {
#pragma unroll
            for (int i = 0; i < kBC; ++i) {
                float *at = s_BC + j * kRows * kNP + kPer * (lane + 32 * i);
                if (!has) continue;
                if constexpr (kPer == 2)
                    *reinterpret_cast<float2 *>(at) = make_float2(r_BC[j][i][0], r_BC[j][i][1]);
                else
                    *at = r_BC[j][i][0];
            }
        }
        __syncwarp();
        if (k0 + kRows < n_steps) fetch(k0 + kRows);
        const int rows = min(kRows, n_steps - k0);
        for (int t = 0; t < rows; t += kGroup) {          // rows without a token have dt = 0: the state stays as it is
            if (kMode == kScanForward && at_kept && ((k0 + t) & (kScanHistory - 1)) == 0) {
#pragma unroll
                for (int j = 0; j < kC; ++j) store_floats<kWhole, kNS>(at_kept + j * p.states, h[j], nn[j]);
                at_kept += static_cast<long long>(p.channels) * p.states;
            }
            float o[kGroup * kC];
#pragma unroll
            for (int s = 0; s < kGroup; ++s) {
                float x[2 * kC], in[kNS], out[kNS];
                load_floats<true, 2 * kC>(x, reinterpret_cast<const float *>(s_pair + (t + s) * kPitch + ch), 2 * kC);
                load_floats<true, kNS>(in, s_BC + (t + s) * kNP + n0, kNS);
                if (kMode == kScanForward) load_floats<true, kNS>(out, s_BC + kRows * kNP + (t + s) * kNP + n0, kNS);
#pragma unroll
                for (int j = 0; j < kC; ++j) {
                    float a[kNS], v[kNS];
                    scan_decays<kNS>(a, x[2 * j], rate[j]);
                    if constexpr (kBackward) {
                        fma_each<kNS>(v, x[2 * j + 1], in, h[j]);
                        mul_each<kNS>(h[j], a, v);
                    } else {
                        mul_each<kNS>(v, x[2 * j + 1], in);
                        fma_each<kNS>(h[j], a, h[j], v);
                    }
                    if constexpr (kMode == kScanForward)
                        o[s * kC + j] = dot_each<kNS>(h[j], out);
                    else
                        sum_dt[j] += x[2 * j];
                }
            }
            if constexpr (kMode == kScanForward) {
                // every lane of the channels ends up with the sum of one of kS values
#pragma unroll
                for (int s = 0; s < kGroup * kC; s += kS) {
                    float v[kS];
#pragma unroll
                    for (int i = 0; i < kS; ++i) v[i] = o[s + i];
                    lane_sums<kS, 1, kS / 2>(v, lane);
                    const int i = s + first_sum<kS, 1, kS / 2>(lane);
                    __syncwarp();                         // all lanes of the channels have read the steps' pairs
                    s_pair[(t + i / kC) * kPitch + ch + i % kC].x = v[0];
                }
            }
        }
        __syncwarp();
        if constexpr (kMode == kScanForward) {
            if (row_on) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float4 f = own[e / 2];
                    y[e] = f.x;
                    y[e + 1] = f.z;
                }
                if (p.D) {
                    const Piece<float, 8> skip = load_piece<kWhole, float, 8>(p.D + c, cn);
#pragma unroll
                    for (int e = 0; e < 8; e += 2) fma_pair(y[e], y[e + 1], skip[e], skip[e + 1], u[e], u[e + 1], y[e], y[e + 1]);
                }
                if (gated) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= z[e] * sigmoid_f32(z[e]);
                }
                store_piece<kWhole, T, 8>(at_y, y, cn, p.unit);
            }
            at_y += static_cast<long long>(way * kRows) * p.channels;
        }
    }
#pragma unroll
    for (int j = 0; j < kC; ++j) {
        const long long at = state_at + j * p.states;
        if constexpr (kMode == kScanForward) {
            if (p.final_state && blk.chunk == p.chunks - 1) store_floats<kWhole, kNS>(p.final_state + at, h[j], nn[j]);
        } else {
            // forward: slot j + 1 is the state behind chunk j; backward: slot j the gradient in front of chunk j
            const long long slot = blk.chunk + (kBackward ? 0 : 1);
            store_floats<kWhole, kNS>(p.slots + slot * slot_step + at, h[j], nn[j]);
            if (n0 == 0 && nn[j] > 0) p.sums[(slot * p.batch + blk.b) * p.channels + d + j] = sum_dt[j];
        }
    }
}

// Shared memory of a CTA of the backward pass.
__host__ __device__ constexpr size_t scan_backward_smem(int channels, int states, int lanes, int bytes)
{
    const size_t width = 32 / lanes * channels, rows = 256 / width, np = static_cast<size_t>(states) * lanes;
    const size_t warp = 2 * 4 * 32 * 8 * bytes + rows * (width + 2) * 20 + 2 * rows * np * 4 + 2 * width * 4 + 2 * 32 * 8 * 4;
    return kScanWarps * (warp + 2 * rows * 2 * np * 4);
}

// Backward pass of a chunk, tile by tile from the last one to the first, each in stretches of kScanHistory steps.  From the state that the
// forward pass kept in front of the stretch the lanes run the recurrence forward once more and hold a h of its steps in registers;
// then they run
//   G = C dyo + e,   q = G a h,   s = sum_n G B,   r = sum_n rate q,   dA += dt q,   e <- a G         (dyo = dy silu(z))
// backward, a taken again from dt.  Over the channels sum dC = h dyo and dB = G dt u: the two of a lane first, then eight values at a time
// over the lanes of a warp, the four warps' sums through shared memory, the CTAs' through global memory, each in a fixed order.  Over the
// states of a channel sum o, s and r.  The rows' lanes then make du = dt s + D dyo, ddelta = (u s + r ln 2) sigmoid and dz.
// Bound: latency at the 10 to 12 warps that an SM holds (45 % of the issue slots are used), not one unit: 64 x 197 x 384,
// N = 16, binary16: 140 to 147 us, of it 60 for all but the recurrence, 20 for the sums over lanes, 18 for the last step; with eight warps per SM 177.
// Three CTAs are as many as 168 registers allow, and as many as 72,704 bytes of shared memory do; with more states or binary32 rows the
// shared memory allows fewer: two CTAs at N = 9 .. 16 in binary32, one from N = 17 on.
// The rows wait in shared memory for their second use (registers: spills; read again: 10 us more).  The whole backward pass
// 155 us, exponentials alone 22.
template <typename T, int kC, int kNS, int kS, bool kWhole>
__global__ void __launch_bounds__(kScanWarps * 32, kC * kNS <= 2 && sizeof(T) == 2 ? 4 : 3) ptq_scan_backward_kernel(const ScanParams p)
{
    constexpr int kWidth = 32 / kS * kC, kPitch = kWidth + 2;      // channels of a warp
    constexpr int kRows = 256 / kWidth, kNP = kNS * kS;            // steps of a tile, states padded
    constexpr int kStretch = kScanHistory;
    constexpr int kSteps = 8 / kNS;                       // steps whose dB (dC) values are summed together: eight values
    constexpr int kLeft = kS >= 4 ? kS / 4 : 1;           // of them left in a lane
    constexpr int kSR = 2 * kC > kS ? 2 * kC : kS;        // values s and r that are summed together
    constexpr int kO = kC > kS ? kC : kS;                 // values o that are summed together
    constexpr int kPer = kNP >= 2 ? 2 : 1;
    constexpr int kBC = (kRows * kNP + 32 * kPer - 1) / (32 * kPer);
    constexpr int kApart = kBC > 1 ? 32 * kPer / kNP : kRows;
    static_assert(kApart * kBC == kRows && kRows % kStretch == 0, "a fetch goes one tile on, in whole stretches");
    constexpr int kThreads = kScanWarps * 32;
    enum { kU, kDelta, kDy, kZ, kTensors };               // what a lane reads of a row
    constexpr int kParts = sizeof(T) / 2;
    struct Warp {
        uint4 rows[2][kTensors][kParts][32];              // of this tile and, on their way, of the next one
        float2 pair[kRows * kPitch];                      // (dt, dt u), later (s, r)
        float g[kRows * kPitch], o[kRows * kPitch];       // dyo; o without D u
        float dt[kRows * kPitch];
        float BC[2][kRows * kNP];
        float bias[kWidth], skip[kWidth];                 // delta_bias and D of the warp's channels, zeros for none
        float2 sum_D[4][32], sum_bias[4][32];             // of the lane's channels, over its rows
    };
    extern __shared__ __align__(16) unsigned char scan_smem[];
    griddep_wait();
    griddep_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    Warp &w = reinterpret_cast<Warp *>(scan_smem)[warp];
    float *const s_sum = reinterpret_cast<float *>(scan_smem + kScanWarps * sizeof(Warp));      // [2][kScanWarps][kRows][2][kNP]: dB, dC
    constexpr int kSums = kRows * 2 * kNP;
    static_assert(kScanWarps * (sizeof(Warp) + 2 * kSums * sizeof(float)) == scan_backward_smem(kC, kNS, kS, sizeof(T)), "as the launch sizes it");
    const ScanBlock blk(p, blockIdx.x, p.group_blocks, p.chunks, 0, kWidth * kScanWarps);
    const bool softplus = p.flags & kScanSoftplus, reverse = p.flags & kScanReverse;

    const int ch = lane / kS * kC, n0 = (lane % kS) * kNS, d = blk.c0 + warp * kWidth + ch;
    const long long state_at = (static_cast<long long>(blk.b) * p.channels + d) * p.states + n0;
    int nn[kC];
    float rate[kC][kNS], e[kC][kNS], dA[kC][kNS];
#pragma unroll
    for (int j = 0; j < kC; ++j) {
        nn[j] = d + j < blk.c_end ? max(min(kNS, p.states - n0), 0) : 0;
        load_floats<kWhole, kNS>(rate[j], p.A + static_cast<long long>(d + j) * p.states + n0, nn[j]);
#pragma unroll
        for (int k = 0; k < kNS; ++k) {
            rate[j][k] = scan_rate(rate[j][k]);
            e[j][k] = dA[j][k] = 0.0f;
        }
        if (blk.chunk < p.chunks - 1) {
            if (nn[j] > 0) scan_fold<kWhole, kNS>(e[j], rate[j], p, blk.b, d + j, n0, nn[j], p.chunks - 1, blk.chunk, -1);
        } else if (p.dfinal) {
            load_floats<kWhole, kNS>(e[j], p.dfinal + state_at + j * p.states, nn[j]);
        }
    }

    // the lane's part of a row
    const int row = lane / (kWidth / 8), part8 = lane % (kWidth / 8) * 8, c = blk.c0 + warp * kWidth + part8;
    const int cn = max(min(8, blk.c_end - c), 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) w.sum_D[i][lane] = w.sum_bias[i][lane] = make_float2(0.0f, 0.0f);
    const long long sequence = static_cast<long long>(blk.b) * p.length;
    const auto token_of = [&](int i) { return static_cast<long long>(reverse && i < blk.len ? blk.len - 1 - i : i); };
    const auto fetch_rows = [&](int i0, int to) {
        const bool on = i0 + row < blk.i1;
        const long long at = on ? token_of(i0 + row) : 0;
        const int n = on ? cn : 0;
        stage_piece<kWhole, T, 8>(&w.rows[to][kU][0][lane], static_cast<const T *>(p.u) + blk.b * p.u_b + at * p.u_l + c, n, 32, p.unit);
        stage_piece<kWhole, T, 8>(&w.rows[to][kDelta][0][lane], static_cast<const T *>(p.delta) + blk.b * p.delta_b + at * p.delta_l + c, n, 32, p.unit);
        stage_piece<kWhole, T, 8>(&w.rows[to][kDy][0][lane], static_cast<const T *>(p.dy) + (sequence + at) * p.channels + c, n, 32, p.unit);
        if (p.z) stage_piece<kWhole, T, 8>(&w.rows[to][kZ][0][lane], static_cast<const T *>(p.z) + blk.b * p.z_b + at * p.z_l + c, n, 32, p.unit);
    };
    Piece<T, kPer> r_BC[2][kBC];
    const int bc_t = kPer * lane / kNP, bc_n = kPer * lane % kNP;
    const bool has = kPer * lane < kRows * kNP;
    const long long way = reverse ? -1 : 1, first = reverse ? blk.len - 1ll : 0ll;         // step i is token first + way i
    const T *const B0 = static_cast<const T *>(p.B) + blk.b * p.B_b + blk.g * p.B_g + bc_n + first * p.B_l,
            *const C0 = static_cast<const T *>(p.C) + blk.b * p.C_b + blk.g * p.C_g + bc_n + first * p.C_l;
    const auto fetch = [&](int i0) {
        const T *at[2] = {B0 + way * (i0 + bc_t) * p.B_l, C0 + way * (i0 + bc_t) * p.C_l};
        const long long apart[2] = {way * kApart * p.B_l, way * kApart * p.C_l};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
#pragma unroll
            for (int i = 0; i < kBC; ++i) {
                const int states = has && i0 + bc_t + i * kApart < blk.i1 ? p.states - bc_n : 0;
                r_BC[k][i] = p.bc_unit >= 2 ? load_piece<true, T, kPer>(at[k], states) : load_piece<false, T, kPer>(at[k], states);
                at[k] += apart[k];
            }
        }
    };
    const long long kept_step = static_cast<long long>(p.channels) * p.states;
    const float *const kept = p.kept + static_cast<long long>(blk.b) * ((p.length + kScanHistory - 1) / kScanHistory) * kept_step + static_cast<long long>(d) * p.states + n0;
    float r_h[kC][kNS];
    const auto fetch_state = [&](int i) {
#pragma unroll
        for (int j = 0; j < kC; ++j) load_floats<kWhole, kNS>(r_h[j], kept + i / kScanHistory * kept_step + j * p.states, nn[j]);
    };

    const int end = min(blk.i0 + p.chunk_len, p.length);
    int i0 = blk.i0 + (end - 1 - blk.i0) / kRows * kRows;
    // tiles without a token: their gradients are zeros
    for (; i0 >= blk.i0 && i0 >= blk.i1; i0 -= kRows) {
        if (i0 + row < end) {
            float zero[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) zero[i] = 0.0f;
            const long long at = (sequence + i0 + row) * p.channels + c;
            store_piece<kWhole, T, 8>(static_cast<T *>(p.du) + at, zero, cn, p.unit);
            store_piece<kWhole, T, 8>(static_cast<T *>(p.ddelta) + at, zero, cn, p.unit);
            if (p.z) store_piece<kWhole, T, 8>(static_cast<T *>(p.dz) + at, zero, cn, p.unit);
        }
    }
    // the thread's sums of dB and dC: which of the two, which state, which step of the tile first
    const int out_which = tid / kNP & 1, out_n = tid % kNP, out_t = tid / (2 * kNP), share = blockIdx.x % (p.groups * p.group_blocks);
    const auto put_BC = [&](int i, float v) {
        const long long tok = sequence + token_of(i);
        if (p.part_BC)
            p.part_BC[((static_cast<long long>(share) * p.batch * p.length + tok) * 2 + out_which) * p.states + out_n] = v;
        else
            static_cast<T *>(out_which ? p.dC : p.dB)[(tok * p.groups + blk.g) * p.states + out_n] = from_f32<T>(v);
    };
    if (out_n < p.states)
        for (int i = max(i0 + kRows, blk.i0) + out_t; i < end; i += kThreads / (2 * kNP)) put_BC(i, 0.0f);

    if (i0 >= blk.i0) {
        fetch(i0);
        fetch_rows(i0, 0);
        fetch_state(i0 + (min(kRows, blk.i1 - i0) - 1) / kStretch * kStretch);
    }
    for (int i = lane; i < kWidth; i += 32) {
        const int channel = blk.c0 + warp * kWidth + i;
        w.bias[i] = p.delta_bias && channel < blk.c_end ? p.delta_bias[channel] : 0.0f;
        w.skip[i] = p.D && channel < blk.c_end ? p.D[channel] : 0.0f;
    }
    __syncwarp();
    float4 *const own = reinterpret_cast<float4 *>(w.pair + row * kPitch + part8);
    float *const own_g = w.g + row * kPitch + part8, *const own_dt = w.dt + row * kPitch + part8;
    for (int parity = 0; i0 >= blk.i0; i0 -= kRows, parity ^= 1) {
        const bool row_on = i0 + row < blk.i1;
        staged();
        {
            const Piece<T, 8> u = staged_piece<T, 8>(&w.rows[parity][kU][0][lane]), delta = staged_piece<T, 8>(&w.rows[parity][kDelta][0][lane]),
                              dy = staged_piece<T, 8>(&w.rows[parity][kDy][0][lane]);
            Piece<T, 8> z;
            if (p.z) z = staged_piece<T, 8>(&w.rows[parity][kZ][0][lane]);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float2 bias = *reinterpret_cast<const float2 *>(w.bias + part8 + i);
                float4 f;
                f.x = delta[i] + bias.x;
                f.z = delta[i + 1] + bias.y;
                if (softplus) {
                    float t0, t1;
                    exp_minus_abs_pair(t0, t1, f.x, f.z);
                    softplus_pair(f.x, f.z, f.x, f.z, t0, t1);
                }
                mul_pair(f.y, f.w, u[i], u[i + 1], f.x, f.z);
                float2 g = make_float2(dy[i], dy[i + 1]);
                if (p.z) {
                    g.x *= z[i] * sigmoid_f32(z[i]);
                    g.y *= z[i + 1] * sigmoid_f32(z[i + 1]);
                }
                if (!row_on) {
                    f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    g = make_float2(0.0f, 0.0f);
                }
                own[i / 2] = f;
                *reinterpret_cast<float2 *>(own_g + i) = g;
                *reinterpret_cast<float2 *>(own_dt + i) = make_float2(f.x, f.z);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
#pragma unroll
                for (int i = 0; i < kBC; ++i) {
                    float *at = w.BC[k] + kPer * (lane + 32 * i);
                    if (!has) continue;
                    if constexpr (kPer == 2)
                        *reinterpret_cast<float2 *>(at) = make_float2(r_BC[k][i][0], r_BC[k][i][1]);
                    else
                        *at = r_BC[k][i][0];
                }
            }
        }
        __syncwarp();
        if (i0 > blk.i0) {
            fetch(i0 - kRows);
            fetch_rows(i0 - kRows, parity ^ 1);
        }
        float *const sums = s_sum + (parity * kScanWarps + warp) * kSums;
        for (int t0 = (min(kRows, blk.i1 - i0) - 1) / kStretch * kStretch; t0 >= 0; t0 -= kStretch) {
            float h[kC][kNS], ah[kStretch][kC][kNS];
#pragma unroll
            for (int j = 0; j < kC; ++j)
#pragma unroll
                for (int k = 0; k < kNS; ++k) h[j][k] = r_h[j][k];
            if (i0 + t0 > blk.i0) fetch_state(i0 + t0 - kStretch);
            float o[kStretch * kC], v8[kStretch * kNS];
#pragma unroll
            for (int s = 0; s < kStretch; ++s) {
                float x[2 * kC], g[kC], in[kNS], out[kNS];
                load_floats<true, 2 * kC>(x, reinterpret_cast<const float *>(w.pair + (t0 + s) * kPitch + ch), 2 * kC);
                load_floats<true, kC>(g, w.g + (t0 + s) * kPitch + ch, kC);
                load_floats<true, kNS>(in, w.BC[0] + (t0 + s) * kNP + n0, kNS);
                load_floats<true, kNS>(out, w.BC[1] + (t0 + s) * kNP + n0, kNS);
                float dc[kNS];
#pragma unroll
                for (int j = 0; j < kC; ++j) {
                    float a[kNS];
                    scan_decays<kNS>(a, x[2 * j], rate[j]);
                    mul_each<kNS>(ah[s][j], a, h[j]);
                    fma_each<kNS>(h[j], x[2 * j + 1], in, ah[s][j]);
                    o[s * kC + j] = dot_each<kNS>(h[j], out);
                    if (j == 0)
                        mul_each<kNS>(dc, g[j], h[j]);
                    else
                        fma_each<kNS>(dc, g[j], h[j], dc);
                }
#pragma unroll
                for (int k = 0; k < kNS; ++k) v8[s * kNS + k] = dc[k];
                if ((s + 1) * kC % kO == 0 && p.z) {
                    constexpr int kOSteps = kO / kC;
                    float v[kO];
#pragma unroll
                    for (int i = 0; i < kO; ++i) v[i] = o[(s + 1 - kOSteps) * kC + i];
                    lane_sums<kO, 1, kS / 2>(v, lane);
#pragma unroll
                    for (int i = 0; i < kO / kS; ++i) {
                        const int idx = first_sum<kO, 1, kS / 2>(lane) + i;
                        w.o[(t0 + s + 1 - kOSteps + idx / kC) * kPitch + ch + idx % kC] = v[i];
                    }
                }
                if ((s + 1) % kSteps == 0) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = v8[(s + 1 - kSteps) * kNS + i];
                    lane_sums<8, kS, 16>(v, lane);
                    if (lane / kS < 8) {
#pragma unroll
                        for (int i = 0; i < kLeft; ++i) {
                            const int idx = first_sum<8, kS, 16>(lane) + i;
                            sums[((t0 + s + 1 - kSteps + idx / kNS) * 2 + 1) * kNP + n0 + idx % kNS] = v[i];
                        }
                    }
                }
            }
#pragma unroll
            for (int s = kStretch - 1; s >= 0; --s) {
                float x[2 * kC], g[kC], in[kNS], out[kNS];
                load_floats<true, 2 * kC>(x, reinterpret_cast<const float *>(w.pair + (t0 + s) * kPitch + ch), 2 * kC);
                load_floats<true, kC>(g, w.g + (t0 + s) * kPitch + ch, kC);
                load_floats<true, kNS>(in, w.BC[0] + (t0 + s) * kNP + n0, kNS);
                load_floats<true, kNS>(out, w.BC[1] + (t0 + s) * kNP + n0, kNS);
                float db[kNS];
#pragma unroll
                for (int j = 0; j < kC; ++j) {
                    float a[kNS], G[kNS], q[kNS];
                    scan_decays<kNS>(a, x[2 * j], rate[j]);
                    fma_each<kNS>(G, g[j], out, e[j]);
                    mul_each<kNS>(e[j], a, G);
                    if (j == 0)
                        mul_each<kNS>(db, x[2 * j + 1], G);
                    else
                        fma_each<kNS>(db, x[2 * j + 1], G, db);
                    o[s * kC + j] = dot_each<kNS>(G, in);                            // s
                    mul_each<kNS>(q, G, ah[s][j]);
                    ah[s][j][0] = dot_each<kNS>(q, rate[j]);                         // r
                    fma_each<kNS>(dA[j], x[2 * j], q, dA[j]);
                }
#pragma unroll
                for (int k = 0; k < kNS; ++k) v8[s * kNS + k] = db[k];
                if (s % kSteps == 0) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = v8[s * kNS + i];
                    lane_sums<8, kS, 16>(v, lane);
                    if (lane / kS < 8) {
#pragma unroll
                        for (int i = 0; i < kLeft; ++i) {
                            const int idx = first_sum<8, kS, 16>(lane) + i;
                            sums[(t0 + s + idx / kNS) * 2 * kNP + n0 + idx % kNS] = v[i];
                        }
                    }
                }
                if (s * 2 * kC % kSR == 0) {
                    float v[kSR];
#pragma unroll
                    for (int i = 0; i < kSR; ++i) {
                        const int at = s * kC + i / 2;
                        v[i] = i & 1 ? ah[at / kC][at % kC][0] : o[at];
                    }
                    lane_sums<kSR, 1, kS / 2>(v, lane);
                    __syncwarp();                         // all lanes of the channels have read the steps' pairs
#pragma unroll
                    for (int i = 0; i < kSR / kS; ++i) {
                        const int idx = first_sum<kSR, 1, kS / 2>(lane) + i, at = s * kC + idx / 2;
                        reinterpret_cast<float *>(w.pair + (t0 + at / kC) * kPitch + ch + at % kC)[idx & 1] = v[i];
                    }
                }
            }
        }
        __syncthreads();                                   // the warps' sums of dB and dC; the next tile's go to the other half
        if (i0 + row < end) {
            const Piece<T, 8> u = staged_piece<T, 8>(&w.rows[parity][kU][0][lane]), delta = staged_piece<T, 8>(&w.rows[parity][kDelta][0][lane]);
            Piece<T, 8> z, dy;
            if (p.z) {
                z = staged_piece<T, 8>(&w.rows[parity][kZ][0][lane]);
                dy = staged_piece<T, 8>(&w.rows[parity][kDy][0][lane]);
            }
            float du[8], dd[8], dz[8];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float2 dts = *reinterpret_cast<const float2 *>(own_dt + i);
                const float dt[2] = {dts.x, dts.y};
                float slope[2] = {1.0f, 1.0f};
                if (softplus) {
                    const float2 bias = *reinterpret_cast<const float2 *>(w.bias + part8 + i);
                    const float x0 = delta[i] + bias.x, x1 = delta[i + 1] + bias.y;
                    float t0, t1;
                    exp_minus_abs_pair(t0, t1, x0, x1);
                    slope[0] = __fdividef(x0 < 0.0f ? t0 : 1.0f, 1.0f + t0);
                    slope[1] = __fdividef(x1 < 0.0f ? t1 : 1.0f, 1.0f + t1);
                }
                const float4 f = own[i / 2];
                const float2 skip = *reinterpret_cast<const float2 *>(w.skip + part8 + i);
                const float2 gs = *reinterpret_cast<const float2 *>(own_g + i), os = *reinterpret_cast<const float2 *>(w.o + row * kPitch + part8 + i);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float s = k ? f.z : f.x, q = k ? f.w : f.y, uu = u[i + k], dyo = k ? gs.y : gs.x;
                    du[i + k] = dt[k] * s;
                    if (p.D) du[i + k] = fmaf(k ? skip.y : skip.x, dyo, du[i + k]);
                    dd[i + k] = fmaf(uu, s, q * kLn2) * slope[k];
                    dz[i + k] = 0.0f;
                    if (p.z) {
                        float o = k ? os.y : os.x;
                        if (p.D) o = fmaf(k ? skip.y : skip.x, uu, o);
                        const float zz = z[i + k], gate = sigmoid_f32(zz);
                        dz[i + k] = dy[i + k] * o * gate * fmaf(zz, 1.0f - gate, 1.0f);
                    }
                    if (!row_on) du[i + k] = dd[i + k] = dz[i + k] = 0.0f;
                }
                if (row_on) {
                    float2 sum = w.sum_D[i / 2][lane];
                    fma_pair(sum.x, sum.y, u[i], u[i + 1], gs.x, gs.y, sum.x, sum.y);
                    w.sum_D[i / 2][lane] = sum;
                    sum = w.sum_bias[i / 2][lane];
                    add_pair(sum.x, sum.y, sum.x, sum.y, dd[i], dd[i + 1]);
                    w.sum_bias[i / 2][lane] = sum;
                }
            }
            const long long at = (sequence + token_of(i0 + row)) * p.channels + c;
            store_piece<kWhole, T, 8>(static_cast<T *>(p.du) + at, du, cn, p.unit);
            store_piece<kWhole, T, 8>(static_cast<T *>(p.ddelta) + at, dd, cn, p.unit);
            if (p.z) store_piece<kWhole, T, 8>(static_cast<T *>(p.dz) + at, dz, cn, p.unit);
        }
        if (out_n < p.states) {
            constexpr int kApartOut = kThreads / (2 * kNP) < kRows ? kThreads / (2 * kNP) : kRows;
            const float *from = s_sum + parity * kScanWarps * kSums + (out_t * 2 + out_which) * kNP + out_n;
            const bool inside = i0 + kRows <= blk.i1;       // the whole tile has tokens: they follow one another
            const long long tok = sequence + first + way * (i0 + out_t), tok_step = way * kApartOut;
            float *share_at = p.part_BC + ((static_cast<long long>(share) * p.batch * p.length + tok) * 2 + out_which) * p.states + out_n;
#pragma unroll
            for (int j = 0; j < kRows / kApartOut; ++j) {
                const int i = i0 + out_t + j * kApartOut;
                if (out_t >= kRows) continue;
                float v = 0.0f;
#pragma unroll
                for (int k = 0; k < kScanWarps; ++k) v += from[k * kSums + j * kApartOut * 2 * kNP];
                if (inside && p.part_BC)
                    share_at[j * tok_step * 2 * p.states] = v;
                else if (i < end)
                    put_BC(i, i < blk.i1 ? v : 0.0f);
            }
        }
        __syncwarp();
    }
    const long long part = static_cast<long long>(blk.b) * p.chunks + blk.chunk;
#pragma unroll
    for (int j = 0; j < kC; ++j) {
        store_floats<kWhole, kNS>(p.part_A + (part * p.channels + d + j) * p.states + n0, dA[j], nn[j]);
        if (p.dstate && blk.chunk == 0) store_floats<kWhole, kNS>(p.dstate + state_at + j * p.states, e[j], nn[j]);
    }
    // the rows' sums of a channel, in the order of the rows
    __syncwarp();
    for (int i = lane; i < kWidth && blk.c0 + warp * kWidth + i < blk.c_end; i += 32) {
        float a = 0.0f, b = 0.0f;
#pragma unroll 8
        for (int r = 0; r < kRows; ++r) {
            const float2 D2 = w.sum_D[i % 8 / 2][r * (kWidth / 8) + i / 8], b2 = w.sum_bias[i % 8 / 2][r * (kWidth / 8) + i / 8];
            a += i & 1 ? D2.y : D2.x;
            b += i & 1 ? b2.y : b2.x;
        }
        p.part_D[part * p.channels + blk.c0 + warp * kWidth + i] = a;
        p.part_bias[part * p.channels + blk.c0 + warp * kWidth + i] = b;
    }
}

// The shares of the CTAs of the backward pass: dA, dD and ddelta_bias over the sequences and chunks, dB and dC over the CTAs of a group.
constexpr int kScanFinishThreads = 256;     // the threads behind the last whole token have nothing to do
template <typename T>
__global__ void __launch_bounds__(kScanFinishThreads) ptq_scan_finish_kernel(const ScanParams p, float *dA, float *dD, float *dbias, int blocks_A, int blocks_D)
{
    __shared__ float s[kScanFinishThreads / 32][33];
    griddep_wait();
    const long long rows = static_cast<long long>(p.batch) * p.chunks;
    int block = blockIdx.x;
    if (block < blocks_A + 2 * blocks_D) {
        const bool is_A = block < blocks_A, is_D = block < blocks_A + blocks_D;
        float *out = is_A ? dA : is_D ? dD : dbias;
        if (!out) return;
        const long long cols = is_A ? static_cast<long long>(p.channels) * p.states : p.channels;
        const long long col = (is_A ? block : (block - blocks_A) % blocks_D) * 32ll + (threadIdx.x & 31);
        const float v = sum_rows<kScanFinishThreads / 32>((is_A ? p.part_A : is_D ? p.part_D : p.part_bias) + col, rows, cols, col < cols, s);
        if (threadIdx.x < 32 && col < cols) out[col] = v;
        return;
    }
    // dB and dC: a CTA takes whole tokens; one 64-bit division per CTA, the threads' own are of 32 bits
    block -= blocks_A + 2 * blocks_D;
    const int pair = 2 * p.states, tokens = kScanFinishThreads / pair, t = threadIdx.x / pair, q = threadIdx.x - t * pair;
    const long long all = static_cast<long long>(p.batch) * p.length, per = all * pair;
    const long long sets = (all + tokens - 1) / tokens, stride = gridDim.x - blocks_A - 2 * blocks_D;
    if (t >= tokens) return;
    T *const out = static_cast<T *>(q >= p.states ? p.dC : p.dB) + (q >= p.states ? q - p.states : q);
    for (long long set = block; set < sets * p.groups; set += stride) {
        const long long g = set / sets, tok = (set - g * sets) * tokens + t;
        if (tok >= all) continue;
        const float *from = p.part_BC + g * p.group_blocks * per + tok * pair + q;
        float v = 0.0f;
#pragma unroll 8
        for (int j = 0; j < p.group_blocks; ++j, from += per) v += *from;
        out[(tok * p.groups + g) * p.states] = from_f32<T>(v);
    }
}

// One token per sequence.  Bound: the state's bytes, read and written once, and close behind it the issue slots: 1024 sequences of 1536
// channels, N = 16, bfloat16 50 us, 4.3 TB/s (the bytes alone 33; every lane with its own softplus 80, states copied
// asynchronously ahead 70).  The kS lanes of a channel
// hold kNS states each and take kS sequences at a time: every lane makes dt, dt u and in the end y of one of them and hands the former
// round; all loads of the set go out before its first store.  Eight sequences at a time (N > 16) take more registers than four CTAs leave: 1024 sequences
// of 1536 channels, N = 32, binary32 with two CTAs per SM 107 us, four 176 (spills); bfloat16 99 with either.
template <typename T, int kNS, int kS, bool kWhole>
__global__ void __launch_bounds__(256, kS > 4 ? 2 : 4) ptq_scan_step_kernel(const ScanParams p)
{
    const int lane = threadIdx.x & 31, own = lane % kS, base = lane - own;
    const int per_cta = 256 / kS;
    const int blocks = (p.channels + per_cta - 1) / per_cta, rows = gridDim.x / blocks;
    const int d = (blockIdx.x % blocks) * per_cta + threadIdx.x / kS, n0 = own * kNS;
    const bool on = d < p.channels;
    const int nn = on ? max(min(kNS, p.states - n0), 0) : 0;
    const int g = on ? d / p.group_channels : 0;
    float rate[kNS];
    load_floats<kWhole, kNS>(rate, p.A + static_cast<long long>(d) * p.states + n0, nn);
#pragma unroll
    for (int k = 0; k < kNS; ++k) rate[k] = scan_rate(rate[k]);
    const float bias = on && p.delta_bias ? p.delta_bias[d] : 0.0f, D = on && p.D ? p.D[d] : 0.0f;
    const long long state_step = static_cast<long long>(p.channels) * p.states, jump = static_cast<long long>(rows) * kS;
    long long b0 = static_cast<long long>(blockIdx.x / blocks) * kS;
    const T *at_u = static_cast<const T *>(p.u) + (b0 + own) * p.u_b + d, *at_delta = static_cast<const T *>(p.delta) + (b0 + own) * p.delta_b + d,
            *at_z = static_cast<const T *>(p.z) + (b0 + own) * p.z_b + d, *at_B = static_cast<const T *>(p.B) + b0 * p.B_b + g * p.B_g + n0,
            *at_C = static_cast<const T *>(p.C) + b0 * p.C_b + g * p.C_g + n0;
    long long at_state = b0 * state_step + static_cast<long long>(d) * p.states + n0;
    T *at_y = static_cast<T *>(p.y) + (b0 + own) * p.channels + d;
    for (; b0 < p.batch; b0 += jump) {
        const bool token = on && b0 + own < p.batch && (!p.lengths || p.lengths[b0 + own] > 0);
        const unsigned tokens = __ballot_sync(0xffffffffu, token) >> base;           // of the set's sequences: of one without, only the state is read
        float h[kS][kNS];
        Piece<T, kNS> B[kS], C[kS];
#pragma unroll
        for (int i = 0; i < kS; ++i) {
            load_floats<kWhole, kNS>(h[i], p.state + at_state + i * state_step, p.state && b0 + i < p.batch ? nn : 0);
            const int n = tokens >> i & 1 ? nn : 0;
            B[i] = load_piece<kWhole, T, kNS>(at_B + i * p.B_b, n);
            C[i] = load_piece<kWhole, T, kNS>(at_C + i * p.C_b, n);
        }
        const Piece<T, 1> ru = load_piece<false, T, 1>(at_u, token), rdelta = load_piece<false, T, 1>(at_delta, token),
                          rz = load_piece<false, T, 1>(at_z, token && p.z);
        const float x = rdelta[0] + bias, u = ru[0];
        const float dt = !token ? 0.0f : p.flags & kScanSoftplus ? softplus_f32(x) : x;
        float o[kS];
#pragma unroll
        for (int i = 0; i < kS; ++i) {
            const float dt_i = __shfl_sync(0xffffffffu, dt, base + i), in = __shfl_sync(0xffffffffu, dt * u, base + i);
            const bool token_i = tokens >> i & 1;
            float a[kNS], f[kNS];
            scan_decays<kNS>(a, dt_i, rate);
            floats_of(f, B[i]);
            mul_each<kNS>(f, in, f);
            fma_each<kNS>(a, a, h[i], f);
#pragma unroll
            for (int k = 0; k < kNS; ++k) h[i][k] = token_i ? a[k] : h[i][k];       // as it was, infinities too
            floats_of(f, C[i]);
            o[i] = dot_each<kNS>(h[i], f);
            if (p.final_state) store_floats<kWhole, kNS>(p.final_state + at_state + i * state_step, h[i], b0 + i < p.batch ? nn : 0);
        }
        lane_sums<kS, 1, kS / 2>(o, lane);
        // the lane holds the sum of sequence first_sum: its own bits in reverse
        float y = o[0];
        if (kS > 2) y = __shfl_sync(0xffffffffu, y, base + first_sum<kS, 1, kS / 2>(own));
        if (token) {
            if (p.D) y = fmaf(D, u, y);
            if (p.z) y *= rz[0] * sigmoid_f32(rz[0]);
            *at_y = from_f32<T>(y);
        }
        at_u += jump * p.u_b;
        at_delta += jump * p.delta_b;
        at_z += jump * p.z_b;
        at_B += jump * p.B_b;
        at_C += jump * p.C_b;
        at_state += jump * state_step;
        at_y += jump * p.channels;
    }
}

}  // namespace ptq
