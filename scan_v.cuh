// Gated linear recurrence between dt_proj and out_proj.  For step i of a sequence (token p = i, or len-1-i reversed),
// channel d with its group g of B and C, and state n:
//
//   dt = softplus(delta[p,d] + delta_bias[d])           (or without softplus)
//   h[n] <- exp(dt A[d,n]) h[n] + dt u[p,d] B[p,g,n]
//   o = sum_n C[p,g,n] h[n] + D[d] u[p,d],   y[p,d] = o silu(z[p,d])
//
// Bound: the exponentials, N per element at 16 per clock and SM, from N = 4 or so on; below that the bytes.  The states of
// a channel lie in the registers of kS neighbouring lanes, kNS each (N = 16: four lanes of four), so that a warp works
// on 32 / kS channels and every shared-memory word of dt, dt u, B and C that it reads serves several lanes.  A CTA takes a
// tile of 8 kS steps at a time: its threads load 8 channels of one row each (the next tile's rows are under way
// meanwhile), put dt and dt u into shared memory, the lanes run the recurrence, and the threads finish the rows
// that they loaded.  Few rows: the steps are cut into chunks.  A first launch computes what each chunk adds to the state and by
// how much it decays (exp(A sum dt)), the second folds these into the state it starts a chunk from.
#pragma once

#include "ptq_block.cuh"

namespace ptq {

constexpr int kScanHistory = 16;      // steps between two states that are kept for the backward pass
constexpr int kScanThreads = 256, kScanLeast = 128;       // of a CTA: most, and fewest where a channel has fewer than eight lanes

constexpr unsigned kScanSoftplus = 1u, kScanReverse = 2u;

struct ScanParams {
    const void *u, *delta, *z, *B, *C;          // z may be null
    long long u_b, u_l, delta_b, delta_l, z_b, z_l, B_b, B_l, B_g, C_b, C_l, C_g;      // pitches in elements
    const float *A, *D, *delta_bias, *state;    // all but A may be null
    const int *lengths;                         // may be null
    int batch, length, channels, states, groups;
    int group_channels;                         // channels / groups
    int group_blocks;                           // CTAs that share the channels of a group
    int chunk_len, chunks;
    unsigned flags;
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

// e^-|x|, the argument of the power of two to about 2^-46: its rounding alone would cost four units in the last place at |x| = 7.
// |x| is cut at 126, where the result is zero.
__device__ __forceinline__ float exp_minus_abs(float x)
{
    const float m = -fminf(fabsf(x), 126.0f), y = m * kLog2e;
    const float rest = fmaf(m, 1.925963033e-8f, fmaf(m, kLog2e, -y));
    const float t = exp2_approx(y);
    return fmaf(t, rest * kLn2, t);
}
// log(1 + e^x) = max(x, 0) + log(1 + t), t = e^-|x|; log(1 + t) / t is a polynomial fitted to 5e-9 on [0, 1]: accurate relative to the
// result, small ones too, with about 20 instructions (expf and log1pf take twice as many).
__device__ __forceinline__ float softplus_of(float x, float t)
{
    float p = -0.0032440212f;
    p = fmaf(p, t, 0.01985144429f);
    p = fmaf(p, t, -0.05695949867f);
    p = fmaf(p, t, 0.106036514f);
    p = fmaf(p, t, -0.1530559063f);
    p = fmaf(p, t, 0.1967593879f);
    p = fmaf(p, t, -0.2495413423f);
    p = fmaf(p, t, 0.3332996368f);
    p = fmaf(p, t, -0.4999990165f);
    p = fmaf(p, t, 1.0f);
    return fmaf(p, t, x <= 0.0f ? 0.0f : x);              // NaN passes through
}
__device__ __forceinline__ float softplus_f32(float x) { return softplus_of(x, exp_minus_abs(x)); }

// exp(dt A) as 2^(dt rate).  The hardware's power of two is low by 0.1 to 0.35 units of 2^-24 on average for the arguments of slow decays
// (-0.1 .. 0), where a state multiplies hundreds of them: the argument is raised by a quarter of a unit, which the fused multiply-add
// does at no cost and which rounds away where the memory is short.  2^kDecayShift is 1: a step with dt = 0 keeps the state.
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

// Decay rates times log2(e); finite, so that a step without a token (dt = 0) leaves the state as it is.
__device__ __forceinline__ float scan_rate(float a) { return fminf(fmaxf(a * kLog2e, -3.0e38f), 3.0e38f); }

// Where a channel's pair (dt, dt u) of a row lies: the four 16-byte pieces of eight channels are permuted by the number of
// the eight, so that the rows' threads, which write eight channels each, meet no bank twice.
__device__ __forceinline__ int scan_column(int ch) { return (ch & ~7) | (((((ch >> 1) & 3) ^ ((ch >> 4) & 3)) << 1) | (ch & 1)); }

struct ScanBlock {
    int b, chunk, g, c0, c_end, len, i0, i1;
    __device__ __forceinline__ ScanBlock(const ScanParams &p, int block, int chunks, int first_chunk, int width)
    {
        const int per = p.groups * p.group_blocks;
        const int rest = block / per, blk = block - rest * per;
        b = rest / chunks;
        chunk = first_chunk + rest - b * chunks;
        g = blk / p.group_blocks;
        c0 = g * p.group_channels + (blk - g * p.group_blocks) * width;
        c_end = min(c0 + width, (g + 1) * p.group_channels);
        len = p.lengths ? min(max(p.lengths[b], 0), p.length) : p.length;
        i0 = chunk * p.chunk_len;
        i1 = min(i0 + min(p.chunk_len, p.length - i0), len);
    }
};

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
        for (int k = 0; k < kNS; ++k) h[k] = fmaf(exp2_approx(rate[k] * s), h[k], v[k]);
    }
}

// kMode 0: y and the final state.  1: the state that each chunk but the last one adds.  2: the same for the gradient of the
// state, from the last step to the first: e <- exp(dt A) (C dy silu(z) + e), for each chunk but the first one.
enum { kScanForward = 0, kScanSum = 1, kScanGradSum = 2 };

template <typename T, int kNS, int kS, int kMode, bool kWhole>
__global__ void __launch_bounds__(kScanThreads, BOUNDS) ptq_scan_kernel(const ScanParams p)
{
    constexpr int kRows = 8 * kS, kNP = kNS * kS;         // steps of a tile, states padded
    constexpr int kGroup = kS < 4 ? 4 : kS;               // steps between two joint sums over the lanes of a channel
    constexpr bool kBackward = kMode == kScanGradSum;
    constexpr int kHalf = kRows * kS;                     // pieces of B (or of C) in a tile
    constexpr int kLeast = kS == 8 ? kScanThreads : kScanLeast;
    constexpr int kPieces = ((kMode == kScanForward ? 2 : 1) * kHalf + kLeast - 1) / kLeast;      // of a thread, at most
    extern __shared__ __align__(16) unsigned char scan_smem[];
    const int threads = blockDim.x, tid = threadIdx.x, lane = tid & 31;
    const int width = threads / kS;                       // channels of the CTA
    float2 *s_pair = reinterpret_cast<float2 *>(scan_smem);                       // [kRows][width]: (dt, dt u), later (o, -)
    float *s_B = reinterpret_cast<float *>(s_pair + kRows * width);               // [kRows][kNP], then C likewise
    const ScanBlock blk(p, blockIdx.x, kMode == kScanForward ? p.chunks : p.chunks - 1, kBackward ? 1 : 0, width);
    const bool softplus = p.flags & kScanSoftplus, reverse = p.flags & kScanReverse;
    const int n_steps = max(blk.i1 - blk.i0, 0);
    // step k of the chunk's loop is step i of the sequence, token first + k * way
    const bool down = reverse != kBackward;
    const int first_step = kBackward ? blk.i1 - 1 : blk.i0;
    const long long first = reverse ? blk.len - 1 - first_step : first_step;
    const int way = down ? -1 : 1;

    // the thread's part of a row
    const int row = tid / (width / 8), c = blk.c0 + (tid % (width / 8)) * 8;
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
    Piece<T, kNS> r_BC[kPieces];
    const auto fetch = [&](int k0) {
        const int n = k0 + row < n_steps ? cn : 0;
        r_u = load_piece<kWhole, T, 8>(at_u, n);
        r_delta = load_piece<kWhole, T, 8>(at_delta, n);
        if (gated) r_z = load_piece<kWhole, T, 8>(at_z, n);
        at_u += next_u;
        at_delta += next_delta;
        at_z += next_z;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int q = tid + i * threads, t = (q % kHalf) / kS, n0 = q % kS * kNS;
            const bool is_C = kMode == kScanForward ? q >= kHalf : kBackward;
            const bool on = q < (kMode == kScanForward ? 2 : 1) * kHalf && k0 + t < n_steps;
            const long long token = first + way * (k0 + t);
            const T *from = is_C ? static_cast<const T *>(p.C) + blk.b * p.C_b + token * p.C_l + blk.g * p.C_g + n0
                                 : static_cast<const T *>(p.B) + blk.b * p.B_b + token * p.B_l + blk.g * p.B_g + n0;
            r_BC[i] = load_piece<false, T, kNS>(from, on ? p.states - n0 : 0);
        }
    };
    if (n_steps > 0) fetch(0);
    const Piece<float, 8> bias = load_piece<kWhole, float, 8>(p.delta_bias + c, p.delta_bias ? cn : 0);

    // the lane's channel and states
    const int ch = tid / kS, n0 = (tid % kS) * kNS, d = blk.c0 + ch, col = scan_column(ch);
    const int nn = d < blk.c_end ? max(min(kNS, p.states - n0), 0) : 0;
    float rate[kNS], h[kNS];
    load_floats<kWhole, kNS>(rate, p.A + static_cast<long long>(d) * p.states + n0, nn);
#pragma unroll
    for (int k = 0; k < kNS; ++k) {
        rate[k] = scan_rate(rate[k]);
        h[k] = 0.0f;
    }
    const long long state_at = (static_cast<long long>(blk.b) * p.channels + d) * p.states + n0;
    const long long slot_step = static_cast<long long>(p.batch) * p.channels * p.states;
    if constexpr (kMode == kScanForward) {
        if (blk.chunk > 0) {
            if (nn > 0) scan_fold<kWhole, kNS>(h, rate, p, blk.b, d, n0, nn, 1, blk.chunk + 1, 1);
        } else if (p.state) {
            load_floats<kWhole, kNS>(h, (p.chunks > 1 ? p.slots : p.state) + state_at, nn);
        }
    } else if constexpr (kMode == kScanSum) {
        // chunk 0 starts from the true state; the second launch takes it from a copy, since the final state may replace it
        if (blk.chunk == 0 && p.state) {
            load_floats<kWhole, kNS>(h, p.state + state_at, nn);
            store_floats<kWhole, kNS>(p.slots + state_at, h, nn);
        }
    } else if (blk.chunk == p.chunks - 1 && p.dfinal) {
        load_floats<kWhole, kNS>(h, p.dfinal + state_at, nn);
    }
    float sum_dt = 0.0f;
    T *at_y = static_cast<T *>(p.y) + (static_cast<long long>(blk.b) * p.length + tok) * p.channels + c;
    float *at_kept = nullptr;
    if (kMode == kScanForward && p.history)
        at_kept = p.history +
                  ((blk.b * static_cast<long long>((p.length + kScanHistory - 1) / kScanHistory) + blk.i0 / kScanHistory) * p.channels + d) * p.states + n0;

    float2 *const own = s_pair + row * width;             // the row that the thread fills and finishes
    for (int k0 = 0; k0 < n_steps; k0 += kRows) {
        const bool row_on = k0 + row < n_steps;
        const Piece<T, 8> u = r_u, z = r_z;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float4 pair;
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const float x = r_delta[e + o] + bias[e + o];
                
#ifdef NO_SOFT
 const float dt = !row_on ? 0.0f : x;
#else
 const float dt = !row_on ? 0.0f : softplus ? softplus_f32(x) : x;
#endif

                float in = r_u[e + o];
                if constexpr (kBackward) {
                    if (gated) in *= r_z[e + o] * sigmoid_f32(r_z[e + o]);
                } else {
                    in *= dt;
                }
                (o ? pair.z : pair.x) = dt;
                (o ? pair.w : pair.y) = row_on ? in : 0.0f;
            }
            *reinterpret_cast<float4 *>(own + scan_column(c - blk.c0 + e)) = pair;
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int q = tid + i * threads;
            if (q < (kMode == kScanForward ? 2 : 1) * kHalf) {
                float f[kNS];
#pragma unroll
                for (int k = 0; k < kNS; ++k) f[k] = r_BC[i][k];
                store_floats<true, kNS>(s_B + q * kNS, f, kNS);
            }
        }
        __syncthreads();

#ifdef NO_FETCH
        if (k0 + kRows < n_steps && p.chunks > 1000000) fetch(k0 + kRows);
#else
        if (k0 + kRows < n_steps) fetch(k0 + kRows);
#endif

        const int rows = min(kRows, n_steps - k0);

#ifdef NO_MAIN
 const int rows2 = p.chunks > 1000000 ? rows : 0;
#else
 const int rows2 = rows;
#endif
        for (int t = 0; t < rows2; t += kGroup) {          // rows without a token have dt = 0: the state stays as it is
            if (kMode == kScanForward && at_kept && ((k0 + t) & (kScanHistory - 1)) == 0) {
                store_floats<kWhole, kNS>(at_kept, h, nn);
                at_kept += static_cast<long long>(p.channels) * p.states;
            }
            float o[kGroup];
#pragma unroll
            for (int s = 0; s < kGroup; ++s) {
                const float2 x = s_pair[(t + s) * width + col];
                float in[kNS], a[kNS];
                load_floats<true, kNS>(in, s_B + (t + s) * kNP + n0, kNS);
                scan_decays<kNS>(a, x.x, rate);
                if constexpr (kBackward) {
                    fma_each<kNS>(h, x.y, in, h);
                    mul_each<kNS>(h, a, h);
                } else {
                    mul_each<kNS>(in, x.y, in);
                    fma_each<kNS>(h, a, h, in);
                }
                if constexpr (kMode == kScanForward) {
                    float out[kNS];
                    load_floats<true, kNS>(out, s_B + kHalf * kNS + (t + s) * kNP + n0, kNS);
                    o[s] = dot_each<kNS>(h, out);
                } else {
                    sum_dt += x.x;
                }
            }
            if constexpr (kMode == kScanForward) {
                // every lane of the channel ends up with the sum of one of kS steps
#pragma unroll
                for (int s = 0; s < kGroup; s += kS) {
                    float v[kS];
#pragma unroll
                    for (int i = 0; i < kS; ++i) v[i] = o[s + i];

#ifndef NO_SUMS
                    lane_sums<kS, 1, kS / 2>(v, lane);
#else
                    v[0] = v[0]+v[kS-1]+v[kS/2]+v[kS/4];
#endif

                    __syncwarp();                         // all lanes of the channel have read the steps' pairs
                    s_pair[(t + s + first_sum<kS, 1, kS / 2>(lane)) * width + col].x = v[0];
                }
            }
        }
        __syncthreads();
        if constexpr (kMode == kScanForward) {

#ifdef NO_EPI
            if (row_on && p.chunks > 1000000) {
#else
            if (row_on) {
#endif
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float4 pair = *reinterpret_cast<const float4 *>(own + scan_column(c - blk.c0 + e));
                    y[e] = pair.x;
                    y[e + 1] = pair.z;
                }
                if (p.D) {
                    const Piece<float, 8> skip = load_piece<kWhole, float, 8>(p.D + c, cn);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = fmaf(skip[e], u[e], y[e]);
                }
                if (gated) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] *= z[e] * sigmoid_f32(z[e]);
                }
                store_piece<kWhole, T, 8>(at_y, y, cn);
            }
            at_y += static_cast<long long>(way * kRows) * p.channels;
        }
    }
    if constexpr (kMode == kScanForward) {
        if (p.final_state && blk.chunk == p.chunks - 1) store_floats<kWhole, kNS>(p.final_state + state_at, h, nn);
    } else {
        // forward: slot j + 1 is the state behind chunk j; backward: slot j the gradient in front of chunk j
        store_floats<kWhole, kNS>(p.slots + (blk.chunk + (kBackward ? 0 : 1)) * slot_step + state_at, h, nn);
        if (n0 == 0 && nn > 0)
            p.sums[(static_cast<long long>(blk.chunk + (kBackward ? 0 : 1)) * p.batch + blk.b) * p.channels + d] = sum_dt;
    }
}

// Backward pass of the tiles of kScanHistory steps of a chunk, from the last one to the first.  From the state that the
// forward pass kept in front of the tile the lanes run the recurrence forward once more and hold a h of all its steps in registers; then
// they run
//   G = C dyo + e,   q = G a h,   s = sum_n G B,   r = sum_n rate q,   dA += dt q,   e <- a G         (dyo = dy silu(z))
// backward, a taken again from dt.  Over the channels sum dC = h dyo and dB = G dt u (eight values at a time over the lanes
// of a warp, the warps' sums through shared memory, the CTAs' through global memory, each in a fixed order); over the
// states of a channel o, s and r.  The rows' threads then make du = dt s + D dyo, ddelta = (u s + r ln 2) sigmoid and dz.
// Bound: issue slots (about 24 per state and step, seven of them the sums of dB and dC).
template <typename T, int kNS, int kS, bool kWhole>
__global__ void __launch_bounds__(kScanThreads, 2) ptq_scan_backward_kernel(const ScanParams p)
{
    constexpr int kRows = kScanHistory, kNP = kNS * kS, kE = kRows / kS;     // channels of a row that a thread holds
    constexpr bool kEarly = kE <= 4;                      // the next tile's rows are fetched into registers during this one's recurrence
    constexpr int kHalf = kRows * kS;                     // pieces of B (or of C) in a tile
    constexpr int kLeast = kS == 8 ? kScanThreads : kScanLeast;
    constexpr int kPieces = (2 * kHalf + kLeast - 1) / kLeast;
    constexpr int kSteps = 8 / kNS;                       // steps whose dB (dC) values are summed together: eight values
    constexpr int kLeft = kS >= 4 ? kS / 4 : 1;           // of them left in a lane
    constexpr int kGroup = kSteps > kS ? kSteps : kS;     // steps of an unrolled group
    constexpr int kPairs = kS >= 4 ? kS / 2 : 1;          // steps whose (s, r) are summed together
    extern __shared__ __align__(16) unsigned char scan_smem[];
    const int threads = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
    const int width = threads / kS;
    float2 *s_pair = reinterpret_cast<float2 *>(scan_smem);                       // [kRows][width]: (dt, dt u), later (s, r)
    float *s_do = reinterpret_cast<float *>(s_pair + kRows * width);              // [kRows][width]: dyo
    float *s_o = s_do + kRows * width;                                            // [kRows][width]: o without D u
    float *s_BC = s_o + kRows * width;                                            // [2][kRows][kNP]
    float *s_sum = s_BC + 2 * kRows * kNP;                                        // [warps][kRows][2][kNP]: dB, dC
    const ScanBlock blk(p, blockIdx.x, p.chunks, 0, width);
    const bool softplus = p.flags & kScanSoftplus, reverse = p.flags & kScanReverse;

    const int ch = tid / kS, n0 = (tid % kS) * kNS, d = blk.c0 + ch, col = scan_column(ch);
    const int nn = d < blk.c_end ? max(min(kNS, p.states - n0), 0) : 0;
    const long long state_at = (static_cast<long long>(blk.b) * p.channels + d) * p.states + n0;
    float rate[kNS], e[kNS], dA[kNS];
    load_floats<kWhole, kNS>(rate, p.A + static_cast<long long>(d) * p.states + n0, nn);
#pragma unroll
    for (int k = 0; k < kNS; ++k) {
        rate[k] = scan_rate(rate[k]);
        e[k] = dA[k] = 0.0f;
    }
    if (blk.chunk < p.chunks - 1) {
        if (nn > 0) scan_fold<kWhole, kNS>(e, rate, p, blk.b, d, n0, nn, p.chunks - 1, blk.chunk, -1);
    } else if (p.dfinal) {
        load_floats<kWhole, kNS>(e, p.dfinal + state_at, nn);
    }

    const int row = tid / (width / kE), c = blk.c0 + (tid % (width / kE)) * kE;
    const int cn = max(min(kE, blk.c_end - c), 0);
    float sum_D[kE], sum_bias[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) sum_D[i] = sum_bias[i] = 0.0f;
    struct Rows {
        Piece<T, kE> u, delta, z, dy;
    };
    const long long sequence = static_cast<long long>(blk.b) * p.length;
    const long long kept_rows = (p.length + kScanHistory - 1) / kScanHistory;
    const auto token_of = [&](int i) { return static_cast<long long>(reverse && i < blk.len ? blk.len - 1 - i : i); };
    const auto rows_of = [&](int i0) {
        Rows r;
        const bool on = i0 + row < blk.i1;
        const long long at = on ? token_of(i0 + row) : 0;
        const int n = on ? cn : 0;
        r.u = load_piece<kWhole, T, kE>(static_cast<const T *>(p.u) + blk.b * p.u_b + at * p.u_l + c, n);
        r.delta = load_piece<kWhole, T, kE>(static_cast<const T *>(p.delta) + blk.b * p.delta_b + at * p.delta_l + c, n);
        r.dy = load_piece<kWhole, T, kE>(static_cast<const T *>(p.dy) + (sequence + at) * p.channels + c, n);
        if (p.z) r.z = load_piece<kWhole, T, kE>(static_cast<const T *>(p.z) + blk.b * p.z_b + at * p.z_l + c, n);
        return r;
    };
    Piece<T, kNS> r_BC[kPieces];
    float r_h[kNS];
    const auto fetch = [&](int i0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int q = tid + i * threads, t = (q % kHalf) / kS, n1 = q % kS * kNS;
            const bool on = q < 2 * kHalf && i0 + t < blk.i1;
            const long long tok = on ? token_of(i0 + t) : 0;
            const T *from = q >= kHalf ? static_cast<const T *>(p.C) + blk.b * p.C_b + tok * p.C_l + blk.g * p.C_g + n1
                                       : static_cast<const T *>(p.B) + blk.b * p.B_b + tok * p.B_l + blk.g * p.B_g + n1;
            r_BC[i] = load_piece<false, T, kNS>(from, on ? p.states - n1 : 0);
        }
        load_floats<kWhole, kNS>(r_h, p.kept + ((blk.b * kept_rows + i0 / kScanHistory) * p.channels + d) * p.states + n0, nn);
    };
    const int slot_of_row = row * width;
    const auto column = [&](int i) { return slot_of_row + scan_column(c - blk.c0 + i); };

    const int end = min(blk.i0 + p.chunk_len, p.length);
    int i0 = blk.i0 + (end - 1 - blk.i0) / kRows * kRows;
    // tiles without a token: their gradients are zeros
    for (; i0 >= blk.i0 && i0 >= blk.i1; i0 -= kRows) {
        if (i0 + row < end) {
            float zero[kE];
#pragma unroll
            for (int i = 0; i < kE; ++i) zero[i] = 0.0f;
            const long long at = (sequence + i0 + row) * p.channels + c;
            store_piece<kWhole, T, kE>(static_cast<T *>(p.du) + at, zero, cn);
            store_piece<kWhole, T, kE>(static_cast<T *>(p.ddelta) + at, zero, cn);
            if (p.z) store_piece<kWhole, T, kE>(static_cast<T *>(p.dz) + at, zero, cn);
        }
    }
    // where the thread's sums of dB and dC go: which of the two, which state
    const int out_which = tid / kNP & 1, out_n = tid % kNP, share = blockIdx.x % (p.groups * p.group_blocks);
    const auto put_BC = [&](int i, float v) {
        const long long tok = sequence + token_of(i);
        if (p.part_BC)
            p.part_BC[((static_cast<long long>(share) * p.batch * p.length + tok) * 2 + out_which) * p.states + out_n] = v;
        else
            static_cast<T *>(out_which ? p.dC : p.dB)[(tok * p.groups + blk.g) * p.states + out_n] = from_f32<T>(v);
    };
    const int first_dead = max(i0 + kRows, blk.i0);
    if (out_n < p.states)
        for (int i = first_dead + tid / (2 * kNP); i < end; i += threads / (2 * kNP)) put_BC(i, 0.0f);

    Rows ahead;
    if (i0 >= blk.i0) {
        fetch(i0);
        if (kEarly) ahead = rows_of(i0);
    }
    for (; i0 >= blk.i0; i0 -= kRows) {
        const bool row_on = i0 + row < blk.i1;
        {
            const Rows r = kEarly ? ahead : rows_of(i0);
            const Piece<float, kE> bias = load_piece<kWhole, float, kE>(p.delta_bias + c, p.delta_bias ? cn : 0);
#pragma unroll
            for (int i = 0; i < kE; ++i) {
                const float x = r.delta[i] + bias[i];
                const float dt = !row_on ? 0.0f : softplus ? softplus_f32(x) : x;
                float g = r.dy[i];
                if (p.z) g *= r.z[i] * sigmoid_f32(r.z[i]);
                s_pair[column(i)] = make_float2(dt, row_on ? dt * r.u[i] : 0.0f);
                s_do[column(i)] = row_on ? g : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int q = tid + i * threads;
                if (q < 2 * kHalf) {
                    float f[kNS];
#pragma unroll
                    for (int k = 0; k < kNS; ++k) f[k] = r_BC[i][k];
                    store_floats<true, kNS>(s_BC + q * kNS, f, kNS);
                }
            }
        }
        float h[kNS];
#pragma unroll
        for (int k = 0; k < kNS; ++k) h[k] = r_h[k];
        __syncthreads();
        if (i0 > blk.i0) {
            fetch(i0 - kRows);
            if (kEarly) ahead = rows_of(i0 - kRows);
        }
        float ah[kRows][kNS];
#pragma unroll
        for (int t = 0; t < kRows; t += kGroup) {
            float o[kGroup], dc[kGroup * kNS];
#pragma unroll
            for (int s = 0; s < kGroup; ++s) {
                const float2 x = s_pair[(t + s) * width + col];
                const float g = s_do[(t + s) * width + col];
                float in[kNS], out[kNS], a[kNS], v[kNS];
                load_floats<true, kNS>(in, s_BC + (t + s) * kNP + n0, kNS);
                load_floats<true, kNS>(out, s_BC + (kRows + t + s) * kNP + n0, kNS);
                scan_decays<kNS>(a, x.x, rate);
                mul_each<kNS>(ah[t + s], a, h);
                fma_each<kNS>(h, x.y, in, ah[t + s]);
                o[s] = dot_each<kNS>(h, out);
                mul_each<kNS>(v, g, h);
#pragma unroll
                for (int k = 0; k < kNS; ++k) dc[s * kNS + k] = v[k];
            }
            if (p.z) {
#pragma unroll
                for (int s = 0; s < kGroup; s += kS) {
                    float v[kS];
#pragma unroll
                    for (int i = 0; i < kS; ++i) v[i] = o[s + i];
                    lane_sums<kS, 1, kS / 2>(v, lane);
                    s_o[(t + s + first_sum<kS, 1, kS / 2>(lane)) * width + col] = v[0];
                }
            }
#pragma unroll
            for (int s = 0; s < kGroup; s += kSteps) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = dc[s * kNS + i];
                lane_sums<8, kS, 16>(v, lane);
                if (lane / kS < 8) {
#pragma unroll
                    for (int i = 0; i < kLeft; ++i) {
                        const int idx = first_sum<8, kS, 16>(lane) + i;
                        s_sum[((warp * kRows + t + s + idx / kNS) * 2 + 1) * kNP + n0 + idx % kNS] = v[i];
                    }
                }
            }
        }
#pragma unroll
        for (int t = kRows - kGroup; t >= 0; t -= kGroup) {
            float db[kGroup * kNS], sr[kGroup * 2];
#pragma unroll
            for (int s = kGroup - 1; s >= 0; --s) {
                const float2 x = s_pair[(t + s) * width + col];
                const float g = s_do[(t + s) * width + col];
                float in[kNS], out[kNS], a[kNS], v[kNS], G[kNS];
                load_floats<true, kNS>(in, s_BC + (t + s) * kNP + n0, kNS);
                load_floats<true, kNS>(out, s_BC + (kRows + t + s) * kNP + n0, kNS);
                scan_decays<kNS>(a, x.x, rate);
                fma_each<kNS>(G, g, out, e);
                mul_each<kNS>(e, a, G);
                mul_each<kNS>(v, x.y, G);
#pragma unroll
                for (int k = 0; k < kNS; ++k) db[s * kNS + k] = v[k];
                sr[s * 2] = dot_each<kNS>(G, in);
                mul_each<kNS>(v, G, ah[t + s]);
                sr[s * 2 + 1] = dot_each<kNS>(v, rate);
                fma_each<kNS>(dA, x.x, v, dA);
            }
#pragma unroll
            for (int s = 0; s < kGroup; s += kPairs) {
                float v[kPairs * 2];
#pragma unroll
                for (int i = 0; i < kPairs * 2; ++i) v[i] = sr[s * 2 + i];
                lane_sums<kPairs * 2, 1, kS / 2>(v, lane);
                const int idx = first_sum<kPairs * 2, 1, kS / 2>(lane);
                float2 *at = s_pair + (t + s + idx / 2) * width + col;
                __syncwarp();                             // all lanes of the channel have read the step's pair
                if (kS == 1)
                    *at = make_float2(v[0], v[1]);
                else
                    (idx & 1 ? at->y : at->x) = v[0];
            }
#pragma unroll
            for (int s = 0; s < kGroup; s += kSteps) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = db[s * kNS + i];
                lane_sums<8, kS, 16>(v, lane);
                if (lane / kS < 8) {
#pragma unroll
                    for (int i = 0; i < kLeft; ++i) {
                        const int idx = first_sum<8, kS, 16>(lane) + i;
                        s_sum[(warp * kRows + t + s + idx / kNS) * 2 * kNP + n0 + idx % kNS] = v[i];
                    }
                }
            }
        }
        __syncthreads();
        if (i0 + row < end) {
            const Rows r = rows_of(i0);                    // once more, from the cache: held in registers they would cost occupancy
            const Piece<float, kE> bias = load_piece<kWhole, float, kE>(p.delta_bias + c, p.delta_bias ? cn : 0);
            const Piece<float, kE> skip = load_piece<kWhole, float, kE>(p.D + c, p.D ? cn : 0);
            float du[kE], dd[kE], dz[kE];
#pragma unroll
            for (int i = 0; i < kE; ++i) {
                const float2 sr = s_pair[column(i)];
                const float dyo = s_do[column(i)], D = skip[i], u = r.u[i], x = r.delta[i] + bias[i];
                float dt = x, slope = 1.0f;
                if (softplus) {
                    const float t = exp_minus_abs(x);
                    dt = softplus_of(x, t);
                    slope = __fdividef(x < 0.0f ? t : 1.0f, 1.0f + t);
                }
                du[i] = p.D ? fmaf(dt, sr.x, D * dyo) : dt * sr.x;
                dd[i] = fmaf(u, sr.x, sr.y * kLn2) * slope;
                dz[i] = 0.0f;
                if (p.z) {
                    const float o = p.D ? fmaf(D, u, s_o[column(i)]) : s_o[column(i)], z = r.z[i], gate = sigmoid_f32(z);
                    dz[i] = r.dy[i] * o * gate * fmaf(z, 1.0f - gate, 1.0f);
                }
                if (!row_on) du[i] = dd[i] = dz[i] = 0.0f;
                if (row_on) {
                    sum_D[i] = fmaf(u, dyo, sum_D[i]);
                    sum_bias[i] += dd[i];
                }
            }
            const long long at = (sequence + token_of(i0 + row)) * p.channels + c;
            store_piece<kWhole, T, kE>(static_cast<T *>(p.du) + at, du, cn);
            store_piece<kWhole, T, kE>(static_cast<T *>(p.ddelta) + at, dd, cn);
            if (p.z) store_piece<kWhole, T, kE>(static_cast<T *>(p.dz) + at, dz, cn);
        }
        for (int t = tid / (2 * kNP); t < kRows; t += threads / (2 * kNP)) {
            const int i = i0 + t;
            if (i >= end || out_n >= p.states) break;
            float v = 0.0f;
            if (i < blk.i1) {
                const float *from = s_sum + (t * 2 + out_which) * kNP + out_n;
#pragma unroll 8
                for (int w = 0; w < warps; ++w) v += from[w * kRows * 2 * kNP];
            }
            put_BC(i, v);
        }
        __syncthreads();                                   // s_sum and s_do are written anew
    }
    const long long part = static_cast<long long>(blk.b) * p.chunks + blk.chunk;
    store_floats<kWhole, kNS>(p.part_A + (part * p.channels + d) * p.states + n0, dA, nn);
    if (p.dstate && blk.chunk == 0) store_floats<kWhole, kNS>(p.dstate + state_at, e, nn);
    // the rows' sums of a channel, in the order of the rows
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kE; ++i) {
        s_do[slot_of_row + c - blk.c0 + i] = sum_D[i];
        s_o[slot_of_row + c - blk.c0 + i] = sum_bias[i];
    }
    __syncthreads();
    for (int i = tid; i < width && blk.c0 + i < blk.c_end; i += threads) {
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            a += s_do[r * width + i];
            b += s_o[r * width + i];
        }
        p.part_D[part * p.channels + blk.c0 + i] = a;
        p.part_bias[part * p.channels + blk.c0 + i] = b;
    }
}

// Column sums of the partial results, one output after another: part[rows][cols] -> out[cols].  A CTA takes 32 columns, its
// eight warps every eighth row each.
__device__ __forceinline__ void sum_rows(const float *part, float *out, long long rows, long long cols, long long first, float (&s)[8][33])
{
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const long long col = first + x;
    float v = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (long long r = y; r < rows; r += 8) v += part[r * cols + col];
    }
    s[y][x] = v;
    __syncthreads();
    if (y == 0 && col < cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += s[i][x];
        out[col] = v;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) ptq_scan_finish_kernel(const ScanParams p, float *dA, float *dD, float *dbias, int blocks_A, int blocks_D)
{
    __shared__ float s[8][33];
    const long long rows = static_cast<long long>(p.batch) * p.chunks;
    int block = blockIdx.x;
    if (block < blocks_A) {
        sum_rows(p.part_A, dA, rows, static_cast<long long>(p.channels) * p.states, block * 32ll, s);
        return;
    }
    block -= blocks_A;
    if (block < 2 * blocks_D) {
        float *out = block < blocks_D ? dD : dbias;
        if (out) sum_rows(block < blocks_D ? p.part_D : p.part_bias, out, rows, p.channels, block % blocks_D * 32ll, s);
        return;
    }
    // dB and dC: the shares of the CTAs of a group
    const long long per = static_cast<long long>(p.batch) * p.length * 2 * p.states;
    const long long total = per * p.groups, stride = static_cast<long long>(gridDim.x - blocks_A - 2 * blocks_D) * 256;
    for (long long idx = (block - 2 * blocks_D) * 256ll + threadIdx.x; idx < total; idx += stride) {
        const long long g = idx / per, rest = idx - g * per, tok = rest / (2 * p.states);
        const int q = static_cast<int>(rest - tok * (2 * p.states));
        float v = 0.0f;
        for (int j = 0; j < p.group_blocks; ++j) v += p.part_BC[(g * p.group_blocks + j) * per + rest];
        const long long at = (tok * p.groups + g) * p.states + (q >= p.states ? q - p.states : q);
        static_cast<T *>(q >= p.states ? p.dC : p.dB)[at] = from_f32<T>(v);
    }
}

// One token per sequence.  Bound: the state's bytes, read and written once.  A thread keeps its kNS rates and goes over
// sequences; the lanes of a channel take its token's values alike.
template <typename T, int kNS, int kS, bool kWhole>
__global__ void __launch_bounds__(256) ptq_scan_step_kernel(const ScanParams p)
{
    const int per_cta = 256 / kS;
    const int blocks = (p.channels + per_cta - 1) / per_cta;
    const int d = (blockIdx.x % blocks) * per_cta + threadIdx.x / kS, n0 = (threadIdx.x % kS) * kNS;
    const int nn = d < p.channels ? max(min(kNS, p.states - n0), 0) : 0;
    const bool on = d < p.channels;
    const int g = on ? d / p.group_channels : 0;
    float rate[kNS];
    load_floats<kWhole, kNS>(rate, p.A + static_cast<long long>(d) * p.states + n0, nn);
#pragma unroll
    for (int k = 0; k < kNS; ++k) rate[k] = scan_rate(rate[k]);
    const float bias = on && p.delta_bias ? p.delta_bias[d] : 0.0f, D = on && p.D ? p.D[d] : 0.0f;
#pragma unroll 2
    for (int b = blockIdx.x / blocks; b < p.batch; b += gridDim.x / blocks) {
        const bool token = !p.lengths || p.lengths[b] > 0;
        const long long at = (static_cast<long long>(b) * p.channels + d) * p.states + n0;
        float h[kNS];
#pragma unroll
        for (int k = 0; k < kNS; ++k) h[k] = 0.0f;
        if (p.state) load_floats<kWhole, kNS>(h, p.state + at, nn);
        float o = 0.0f, u = 0.0f;
        if (on && token) {
            u = to_f32<T>(static_cast<const T *>(p.u)[b * p.u_b + d]);
            const float x = to_f32<T>(static_cast<const T *>(p.delta)[b * p.delta_b + d]) + bias;
            const float dt = p.flags & kScanSoftplus ? softplus_f32(x) : x;
            const T *B = static_cast<const T *>(p.B) + b * p.B_b + g * p.B_g + n0, *C = static_cast<const T *>(p.C) + b * p.C_b + g * p.C_g + n0;
            float a[kNS];
            scan_decays<kNS>(a, dt, rate);
#pragma unroll
            for (int k = 0; k < kNS; ++k) {
                const float in = k < nn ? to_f32<T>(B[k]) : 0.0f, out = k < nn ? to_f32<T>(C[k]) : 0.0f;
                h[k] = fmaf(a[k], h[k], dt * u * in);
                o = fmaf(h[k], out, o);
            }
        }
#pragma unroll
        for (int i = 1; i < kS; i *= 2) o += __shfl_xor_sync(0xffffffffu, o, i);
        if (p.final_state) store_floats<kWhole, kNS>(p.final_state + at, h, nn);
        if (on && token && n0 == 0) {
            if (p.D) o = fmaf(D, u, o);
            if (p.z) {
                const float z = to_f32<T>(static_cast<const T *>(p.z)[b * p.z_b + d]);
                o *= z * sigmoid_f32(z);
            }
            static_cast<T *>(p.y)[static_cast<long long>(b) * p.channels + d] = from_f32<T>(o);
        }
    }
}

}  // namespace ptq
