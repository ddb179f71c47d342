// Backward pass of linear attention with a decay for each head (include/ptq_heads.h).
//
// With S the state in front of a chunk, G the gradient of the state behind it, M_ij = e^{L_i - L_j} for j <= i (else 0), P_ij = C_i . B_j
// and R_ij = dy_i . u_j:
//     dC_i = sum_j M_ij R_ij w_j B_j  +  e^{L_i} S^T dy_i                =: .. + dC'_i
//     dB_j = w_j ( sum_i M_ij R_ij C_i  +  e^{L_64 - L_j} G^T u_j )      =: w_j ( .. + dB'_j )
//     du_j = w_j ( sum_i M_ij P_ij dy_i  +  e^{L_64 - L_j} G B_j )  (+ D dy_j)
//     G   <- e^{L_64} G + sum_i e^{L_i} dy_i C_i^T
//     dw_j = sum_i K_ij + B_j . dB'_j,   K = M P R (per element)
//     d(log decay)_t = sum_{j < t <= i} K_ij w_j + sum_{i >= t} C_i . dC'_i + sum_{j < t} w_j B_j . dB'_j + e^{L_64} <G, S>
// The last line sums what passes step t.  (Gradients of the L_i, summed from t on, are the same; but in them each pair of steps on one
// side of t comes twice with opposite signs, and what the roundings leave of them is more than the result of a step near an end.)  Eight warps walk over the chunks from the last to the
// first: four have 16 steps each as rows i (dC, and 16 columns of G in registers, binary32), four as rows j (dB, du); P and R are
// computed both ways, which costs less than an exchange.  S comes from the forward pass's history.  Where S, G and the factors of G's
// update decide states and gradients of parameters they are operands of several 16-bit parts.
//
// What bounds it: latency again, at two CTAs to an SM (up to 64 states, 16 bits; else one), and fetching instructions: issue slots 33 %
// busy, the tensor pipe 20 %, stalls barriers 2.7, no instruction 2.5, fixed latency 1.7, shared memory 1.5 per instruction.  64 x 197 x 12
// heads of 64 columns, 64 states, binary16: 172 us (all kernels of the step, forward included, 249).  Loops that are not unrolled over sets of 16 steps took it from 386 to 320 us
// (the step), shared factors and a second CTA to 295.  binary32: 8 x 784 x 6 heads, 16 states, 188 us for the step; splitting operands into tf32
// parts is most of the instructions.
#pragma once

#include "ptq_heads.cuh"

namespace ptq {

// Factors of a chunk's steps, which one warp forms for all, a chunk ahead.  `pair[r]` refers to the steps' 16 steps r: of steps in front of
// them e^{L_ref - L_j} (ref: the step in front of the 16), of themselves log2 e^{L_j - L_ref}, of steps behind them e^{L_i - L_last} (last: the
// last of the 16).
template <typename T>
struct HeadBackFactors {
    float w[kHeadSteps], into[kHeadSteps];                // e^{L}
    float pair[4][kHeadSteps];
    float low[sizeof(T) == 4 ? kHeadSteps : 2];           // binary32 activations: what is left of the logarithms of the steps
    float rest[4], rest_low[4];                           // log2 e^{L_64 - L_ref}
    float decay, pad;                                     // e^{L_64}
};
template <typename T>
__device__ __forceinline__ void write_back_factors(HeadBackFactors<T> &f, const HeadSteps &st, int lane)
{
    const double all = __shfl_sync(0xffffffffu, st.sum[1], 31);
    reinterpret_cast<float2 *>(f.w)[lane] = make_float2(st.w[0], st.w[1]);
    reinterpret_cast<float2 *>(f.into)[lane] = make_float2(pow2(st.sum[0]), pow2(st.sum[1]));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const double ref = r ? __shfl_sync(0xffffffffu, st.sum[1], 8 * r - 1) : 0.0, last = __shfl_sync(0xffffffffu, st.sum[1], 8 * r + 7);
        float v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
            v[k] = lane < 8 * r ? pow2(ref - st.sum[k]) : lane < 8 * r + 8 ? static_cast<float>(st.sum[k] - ref) : pow2(st.sum[k] - last);
        reinterpret_cast<float2 *>(f.pair[r])[lane] = make_float2(v[0], v[1]);
        if (lane == r) {
            const double x = all - ref;
            f.rest[r] = static_cast<float>(x);
            if constexpr (sizeof(T) == 4) f.rest_low[r] = static_cast<float>(x - static_cast<float>(x));
        }
    }
    if constexpr (sizeof(T) == 4) write_low(f.low, st, lane);
    if (lane == 0) f.decay = pow2(all);
}

template <typename T, int NP>
struct HeadBackSmem {
    static constexpr int kWide = kHeadSteps * (NP + kHeadPad) * static_cast<int>(sizeof(T));
    static constexpr int kNarrow = kHeadSteps * (kHeadCols + kHeadPad) * static_cast<int>(sizeof(T));
    static constexpr int kStage = 2 * kWide + 2 * kNarrow;
    static constexpr int kParts = kHeadParts<T>;                           // of S and G as operands
    static constexpr int kSums = 7 * kHeadSteps * 4;                       // floats: C . dC', dw, B . dB', 4 warps' K
    static constexpr int kOther = 2 * kParts * kWide + 2 * static_cast<int>(sizeof(HeadBackFactors<T>)) + kSums + 16 * 4;
    // two CTAs to an SM where that is possible, else two stages
    static constexpr int kCtas = sizeof(T) == 2 && NP <= 64 ? 2 : 1;
    static constexpr int kStages = 2 * kStage + kOther <= (kCtas == 2 ? 113 : 227) * 1024 ? 2 : 1;
    static constexpr int kS = kStages * kStage;
    static constexpr int kG = kS + kParts * kWide;
    static constexpr int kFactors = kG + kParts * kWide;
    static constexpr int kSum = kFactors + 2 * static_cast<int>(sizeof(HeadBackFactors<T>));
    static constexpr int kSmall = kSum + kSums;                            // floats: largest magnitudes [8], <G, S> [4], dD [4]
    static constexpr int kBytes = kSmall + 16 * 4;
};

// A warp's 16 rows of a state as an operand in its parts, one tile each.
template <int NP, typename T>
__device__ __forceinline__ void store_parts(T *to, const float (&S)[NP / 8][4], float up, int p0, int lane)
{
    constexpr int kWP = NP + kHeadPad;
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NP / 8; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            T *at = to + (p0 + g + 8 * k) * kWP + 8 * n + 2 * t;
            const float x = S[n][2 * k] * up, y = S[n][2 * k + 1] * up;
            if constexpr (sizeof(T) == 2) {
                uint32_t r[kHeadParts<T>];
                head_split<T>(x, y, r);
#pragma unroll
                for (int q = 0; q < kHeadParts<T>; ++q) *reinterpret_cast<uint32_t *>(at + q * kHeadSteps * kWP) = r[q];
            } else {
                *reinterpret_cast<float2 *>(at) = make_float2(x, y);
            }
        }
}
// d[n] += a (rows) times 16 rows k0 .. of a state operand [p][n] in its parts.
template <int NP, typename T>
__device__ __forceinline__ void mma_parts(float (&d)[NP / 8][4], const HeadA<T> &a, const T *state, int k0, int lane)
{
    constexpr int kWP = NP + kHeadPad;
#pragma unroll
    for (int n = 0; n < NP / 16; ++n)
#pragma unroll
        for (int q = kHeadParts<T> - 1; q >= 0; --q) {
            HeadB<T> b[2];
            load_b_t(b, state + q * kHeadSteps * kWP, kWP, 16 * n, k0, lane);
            head_mma(d[2 * n], a, b[0]);
            head_mma(d[2 * n + 1], a, b[1]);
        }
}
// Rows of accumulators times rows of a tile, summed over the columns: what the rows p0 + g and p0 + g + 8 give, in all lanes of a quad.
template <int NP, typename T>
__device__ __forceinline__ float2 row_dots(const float (&d)[NP / 8][4], const T *tile, int p0, int lane)
{
    constexpr int kWP = NP + kHeadPad;
    const int g = lane >> 2, t = lane & 3;
    float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int n = 0; n < NP / 8; ++n) {
        const float2 x = head_pair(tile + (p0 + g) * kWP + 8 * n + 2 * t), y = head_pair(tile + (p0 + g + 8) * kWP + 8 * n + 2 * t);
        v.x = fmaf(d[n][0], x.x, fmaf(d[n][1], x.y, v.x));
        v.y = fmaf(d[n][2], y.x, fmaf(d[n][3], y.y, v.y));
    }
#pragma unroll
    for (int s = 1; s < 4; s <<= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, s);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, s);
    }
    return v;
}
template <int N>
__device__ __forceinline__ void scale_rows(float (&d)[N][4], float s0, float s1)
{
#pragma unroll
    for (int n = 0; n < N; ++n) {
        d[n][0] *= s0;
        d[n][1] *= s0;
        d[n][2] *= s1;
        d[n][3] *= s1;
    }
}
// Two rows of binary32 parts, 8 n + 2 t columns of each.
template <int NP, bool kPairs>
__device__ __forceinline__ void write_part(const float (&d)[NP / 8][4], float *row0, float *row1, int states, int lane)
{
    const int t = lane & 3;
#pragma unroll
    for (int n = 0; n < NP / 8; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float *row = k ? row1 : row0;
            const int c = 8 * n + 2 * t;
            if (!row || c >= states) continue;
            if constexpr (kPairs) {
                *reinterpret_cast<float2 *>(row + c) = make_float2(d[n][2 * k], d[n][2 * k + 1]);
            } else {
                row[c] = d[n][2 * k];
                if (c + 1 < states) row[c + 1] = d[n][2 * k + 1];
            }
        }
}

// Sixteen more steps of M R or M P as an operand: brings `m`, unless it is zero, into binary16's range and `sums`, which it is multiplied into,
// to the same power of two.
template <typename T, int N>
__device__ __forceinline__ void join_scale(float (&m)[2][4], float (&sums)[N][4], HeadScale &sc)
{
    if constexpr (kScaled<T>) {
        const float top = warp_top<2>(m);
        const HeadScale now = top == 0.0f ? sc : scale_for<kScaleSums>(top);
        if (now.up != sc.up) {
            const float by = now.up * sc.down;
            scale_rows(sums, by, by);
            sc = now;
        }
        if (sc.up != 1.0f) scale_rows(m, sc.up, sc.up);
    }
}
// 16 x 16 scores: rows p0 .. of the one tile with rows q0 .. of the other, over kK columns.
template <int kK, typename T>
__device__ __forceinline__ void scores(float (&d)[2][4], const T *rows, const T *cols, int p0, int q0, int lane)
{
#pragma unroll
    for (int k = 0; k < kK / 16; ++k) {
        HeadB<T> b[2];
        load_b(b, cols, kK + kHeadPad, q0, 16 * k, lane);
        const HeadA<T> a = load_a(rows, kK + kHeadPad, p0, 16 * k, lane);
#pragma unroll
        for (int n = 0; n < 2; ++n) head_mma(d[n], a, b[n], k == 0);
    }
}
// d[n] += a times the 16 rows k0 .. of a tile [k][n].
template <int NP, typename T>
__device__ __forceinline__ void mma_rows(float (&d)[NP / 8][4], const HeadA<T> &a, const T *tile, int k0, int lane)
{
#pragma unroll
    for (int n = 0; n < NP / 16; ++n) {
        HeadB<T> b[2];
        load_b_t(b, tile, NP + kHeadPad, 16 * n, k0, lane);
        head_mma(d[2 * n], a, b[0]);
        head_mma(d[2 * n + 1], a, b[1]);
    }
}

template <typename T, int NP, bool kWhole>
__global__ void __launch_bounds__(256, HeadBackSmem<T, NP>::kCtas) ptq_heads_backward_kernel(const HeadParams p)
{
    using M = HeadBackSmem<T, NP>;
    constexpr int kWP = NP + kHeadPad, kXP = kHeadCols + kHeadPad;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = head_warp(), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, r = warp & 3, p0 = 16 * r;
    const bool rows_i = warp < 4;
    if (p.segments > 1) griddep_wait();
    const HeadPlace a = head_place(p, p.segments);
    const int chunks = (a.n + kHeadSteps - 1) / kHeadSteps;
    const int chunk0 = min(chunks, a.seg * p.segment_chunks), chunk1 = min(chunks, chunk0 + p.segment_chunks), count = chunk1 - chunk0;
    const bool reverse = p.flags & kHeadsReverse;
    const auto stage = [&](int s) { return smem + (M::kStages == 2 ? s * M::kStage : 0); };
    const auto tile_u = [&](int s) { return reinterpret_cast<T *>(stage(s)); };
    const auto tile_dy = [&](int s) { return reinterpret_cast<T *>(stage(s) + M::kNarrow); };
    const auto tile_B = [&](int s) { return reinterpret_cast<T *>(stage(s) + 2 * M::kNarrow); };
    const auto tile_C = [&](int s) { return reinterpret_cast<T *>(stage(s) + 2 * M::kNarrow + M::kWide); };
    T *S_op = reinterpret_cast<T *>(smem + M::kS), *G_op = reinterpret_cast<T *>(smem + M::kG);
    HeadBackFactors<T> *factors = reinterpret_cast<HeadBackFactors<T> *>(smem + M::kFactors);
    float *dot_C = reinterpret_cast<float *>(smem + M::kSum), *dw = dot_C + kHeadSteps, *dot_B = dot_C + 2 * kHeadSteps;
    float *pairs = dot_C + 3 * kHeadSteps;                // [4]: what a warp's rows of K w pass over each step
    float *tops = reinterpret_cast<float *>(smem + M::kSmall), *through = tops + 8, *skip_sum = tops + 12;

    const int64_t dy_l = static_cast<int64_t>(p.heads) * p.cols;
    const int64_t dense = (static_cast<int64_t>(a.b) * p.length * p.heads + a.h) * p.cols + a.tile * kHeadCols;
    const T *u = static_cast<const T *>(p.u) + a.b * p.u_b + a.h * p.u_h + a.tile * kHeadCols;
    const T *dy = static_cast<const T *>(p.dy) + dense;
    const T *B = static_cast<const T *>(p.B) + a.b * p.B_b + a.g * p.B_g, *C = static_cast<const T *>(p.C) + a.b * p.C_b + a.g * p.C_g;
    T *du = static_cast<T *>(p.du) + dense;
    const int64_t delta_at = a.b * p.delta_b + a.h * p.delta_h;
    const float bias = p.delta_bias ? __ldg(p.delta_bias + a.h) : 0.0f, skip = p.D ? __ldg(p.D + a.h) : 0.0f;
    const double A2 = static_cast<double>(__ldg(p.A + a.h)) * kLog2e;
    const int64_t part_row = ((static_cast<int64_t>(a.tile) * p.heads + a.h) * p.batch + a.b) * p.length;
    const int64_t head_at = static_cast<int64_t>(a.b) * p.heads + a.h, state_size = static_cast<int64_t>(p.cols) * p.states;
    const int64_t tile_at = static_cast<int64_t>(a.tile) * kHeadCols * p.states;

    // rows of du behind the sequence's end
    {
        const int64_t from = static_cast<int64_t>(a.seg) * p.segment_chunks * kHeadSteps, to = from + static_cast<int64_t>(p.segment_chunks) * kHeadSteps;
        const int first = static_cast<int>(max(from, static_cast<int64_t>(a.n))), last = static_cast<int>(min(to, static_cast<int64_t>(p.length)));
        for (int step = first + warp; step < last; step += 8)
            for (int c = lane; c < a.cols; c += 32) du[step * dy_l + c] = head_round<T>(0.0f);
    }

    const auto token = [&](int step) { return reverse ? a.n - 1 - step : step; };
    const auto load = [&](int chunk, int s) {
        const int first = chunk * kHeadSteps, rows = a.n - first;
        const int64_t sign = reverse ? -1 : 1, at = token(first);
        load_rows<kHeadCols, 256, kWhole>(tile_u(s), u + at * p.u_l, sign * p.u_l, rows, a.cols, p.unit);
        load_rows<kHeadCols, 256, kWhole>(tile_dy(s), dy + at * dy_l, sign * dy_l, rows, a.cols, p.unit);
        load_rows<NP, 256, kWhole>(tile_B(s), B + at * p.B_l, sign * p.B_l, rows, p.states, p.unit);
        load_rows<NP, 256, kWhole>(tile_C(s), C + at * p.C_l, sign * p.C_l, rows, p.states, p.unit);
        cp_async_commit();
    };
    const auto chunk_of = [&](int i) { return chunk1 - 1 - i; };

    // warps of rows i: G; of rows j, between chunks: S of the one that comes
    float H[NP / 8][4];
    float skip_grad = 0.0f;
    if (rows_i) {
        const float *from = nullptr;
        if (a.seg < p.segments - 1)
            from = p.slots + (head_at * p.segments + a.seg + 1) * state_size + tile_at;
        else if (p.dfinal)
            from = p.dfinal + head_at * state_size + tile_at;
        read_state<kWhole>(H, from, p0, 0, a.cols, p.states, lane);
    }
    const bool starts = a.seg == 0 && p.final_state;      // G in front of this segment is wanted
    float delta[2] = {};                                  // of the next chunk, in warp 0, which forms the factors
    if (warp == 0 && count > 0) load_delta<T>(p, delta_at, chunk_of(0) * kHeadSteps, a.n, lane, delta);
    for (int i = -1; i < count; ++i) {
        const int chunk = chunk_of(i), first = chunk * kHeadSteps, s = i & 1;
        const bool next = i + 1 < count;
        const HeadBackFactors<T> &f = factors[s];
        HeadScale scS = {1.0f, 1.0f}, scG = {1.0f, 1.0f};
        if (i >= 0) {
            if constexpr (kScaled<T>) {                   // one power of two for all columns: they are summed over
                const float top = warp_top<NP / 8>(H);
                if (lane == 0) tops[warp] = top;
                __syncthreads();
                scG = scale_for<kScaleState>(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
                scS = scale_for<kScaleState>(fmaxf(fmaxf(tops[4], tops[5]), fmaxf(tops[6], tops[7])));
            }
            store_parts<NP>(rows_i ? G_op : S_op, H, rows_i ? scG.up : scS.up, p0, lane);
            cp_async_wait<0>();
            __syncthreads();
        }
        if (M::kStages == 2 && next) load(chunk_of(i + 1), s ^ 1);
        const int step0 = first + p0 + g, step1 = step0 + 8;
        const int sixteens = (min(a.n - first, kHeadSteps) + 15) / 16;                  // sets of 16 steps that are there
        if (i >= 0 && rows_i) {
            if (r < sixteens) {
            const float *pair = f.pair[r];
            const float l0 = pair[p0 + g], l1 = pair[p0 + g + 8], r0 = fast_exp2(l0), r1 = fast_exp2(l1);
            // what the state gives dC
            float d[NP / 8][4] = {};
#pragma unroll 1
            for (int k = 0; k < kHeadCols / 16; ++k) mma_parts<NP>(d, load_a(tile_dy(s), kXP, p0, 16 * k, lane), S_op, 16 * k, lane);
            scale_rows(d, f.into[p0 + g] * scS.down, f.into[p0 + g + 8] * scS.down);
            const float2 x = row_dots<NP>(d, tile_C(s), p0, lane);
            if (t == 0) {
                dot_C[p0 + g] = x.x;
                dot_C[p0 + g + 8] = x.y;
            }
            // what the steps up to these give it, 16 at a time
            HeadScale sc = {1.0f, 1.0f};
            float run[2] = {};                            // K w of a row summed up to a column
#pragma unroll 1
            for (int j = 0; j <= r; ++j) {
                const bool diagonal = j == r;
                float m[2][4], P[2][4];                   // R, then M R w; P, then K w
                scores<kHeadCols>(m, tile_dy(s), tile_u(s), p0, 16 * j, lane);
                scores<NP>(P, tile_C(s), tile_B(s), p0, 16 * j, lane);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int col = 16 * j + 8 * q + 2 * t;
                    const float2 v = *reinterpret_cast<const float2 *>(pair + col), w = *reinterpret_cast<const float2 *>(f.w + col);
                    float between[4] = {l0 - v.x, l0 - v.y, l1 - v.x, l1 - v.y};
                    if constexpr (sizeof(T) == 4) {
                        if (diagonal) add_low(between, f.low, p0 + g, col);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int at = col + (k & 1), row = p0 + g + (k < 2 ? 0 : 8);
                        const float vk = k & 1 ? v.y : v.x, wk = k & 1 ? w.y : w.x;
                        if (at == row) skip_grad += m[q][k];
                        const float by = (diagonal ? fast_exp2(between[k]) : (k < 2 ? r0 : r1) * vk) * wk;
                        const bool on = !diagonal || at <= row;
                        m[q][k] = on ? m[q][k] * by : 0.0f;
                        P[q][k] = on ? m[q][k] * P[q][k] : 0.0f;
                    }
                    // what passes over step `col`: of each row i >= col its sum up to, not with, col
                    float pass[2] = {};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int row = p0 + g + 8 * k;
                        float v = P[q][2 * k] + P[q][2 * k + 1];
#pragma unroll
                        for (int z = 1; z < 4; z <<= 1) {
                            const float w = __shfl_up_sync(0xffffffffu, v, z, 4);
                            if (t >= z) v += w;
                        }
                        const float before = __shfl_up_sync(0xffffffffu, v, 1, 4), at = run[k] + (t ? before : 0.0f);
                        if (col <= row) pass[0] += at;
                        if (col + 1 <= row) pass[1] += at + P[q][2 * k];
                        run[k] += __shfl_sync(0xffffffffu, v, 3, 4);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int z = 4; z < 32; z <<= 1) pass[k] += __shfl_xor_sync(0xffffffffu, pass[k], z);
                    if (g == 0) *reinterpret_cast<float2 *>(pairs + r * kHeadSteps + col) = make_float2(pass[0], pass[1]);
                }
                join_scale<T>(m, d, sc);
                mma_rows<NP>(d, acc_to_a<T>(m[0], m[1], 1.0f), tile_B(s), 16 * j, lane);
            }
            if (kScaled<T> && sc.down != 1.0f) scale_rows(d, sc.down, sc.down);
            write_part<NP, kWhole>(d, step0 < a.n ? p.part_C + (part_row + token(step0)) * p.states : nullptr,
                                   step1 < a.n ? p.part_C + (part_row + token(step1)) * p.states : nullptr, p.states, lane);
            } else {
                if (lane < 16) dot_C[p0 + lane] = 0.0f;
                reinterpret_cast<float2 *>(pairs + r * kHeadSteps)[lane] = make_float2(0.0f, 0.0f);
            }
            // <G, S> of this warp's columns, and G in front of the chunk
            float z = 0.0f;
#pragma unroll
            for (int n = 0; n < NP / 8; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int at = (p0 + g + 8 * k) * kWP + 8 * n + 2 * t;
                    float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
                    for (int q = kHeadParts<T> - 1; q >= 0; --q) {
                        const float2 x = head_pair(S_op + q * kHeadSteps * kWP + at);
                        v.x += x.x;
                        v.y += x.y;
                    }
                    z = fmaf(H[n][2 * k], v.x, fmaf(H[n][2 * k + 1], v.y, z));
                }
            z *= scS.down;
#pragma unroll
            for (int q = 16; q > 0; q >>= 1) z += __shfl_xor_sync(0xffffffffu, z, q);
            if (lane == 0) through[r] = z * f.decay;
            if (p0 < a.cols && (next || starts)) state_update<NP, NP / 8>(H, tile_dy(s), tile_C(s), f.into, f.decay, p0, 0, sixteens, lane);
        } else if (i >= 0 && r >= sixteens) {
            if (lane < 16) dw[p0 + lane] = dot_B[p0 + lane] = 0.0f;
        } else if (i >= 0) {
            const float *pair = f.pair[r];
            const float l0 = pair[p0 + g], l1 = pair[p0 + g + 8], last = pair[p0 + 15], rest = f.rest[r];
            float to_last[2] = {last - l0, last - l1}, to_end[2] = {rest - l0, rest - l1};
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    to_last[k] += f.low[p0 + 15] - f.low[p0 + g + 8 * k];
                    to_end[k] += f.rest_low[r] - f.low[p0 + g + 8 * k];
                }
            }
            const float r0 = fast_exp2(to_last[0]), r1 = fast_exp2(to_last[1]), e0 = fast_exp2(to_end[0]) * scG.down, e1 = fast_exp2(to_end[1]) * scG.down;
            const float w0 = f.w[p0 + g], w1 = f.w[p0 + g + 8];
            // what the state behind the chunk gives du and dB
            float x[8][4] = {}, d[NP / 8][4] = {};
#pragma unroll 1
            for (int k = 0; k < NP / 16; ++k) {
                const HeadA<T> c = load_a(tile_B(s), kWP, p0, 16 * k, lane);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    HeadB<T> b[2];
                    load_b(b, G_op, kWP, 16 * q, 16 * k, lane);
                    head_mma(x[2 * q], c, b[0]);
                    head_mma(x[2 * q + 1], c, b[1]);
                }
            }
            scale_rows(x, e0, e1);
#pragma unroll 1
            for (int k = 0; k < kHeadCols / 16; ++k) mma_parts<NP>(d, load_a(tile_u(s), kXP, p0, 16 * k, lane), G_op, 16 * k, lane);
            scale_rows(d, e0, e1);
            const float2 b = row_dots<NP>(d, tile_B(s), p0, lane);
            // and what these steps and the ones behind them do, 16 at a time
            HeadScale scx = {1.0f, 1.0f}, scd = {1.0f, 1.0f};
            float k0 = 0.0f, k1 = 0.0f;                   // column sums of K
            // (binary32: a bound that the compiler knows is worth more than the steps that are not there, 141 instead of 157 us of 8 x 784 x 6 heads)
            const int sets = sizeof(T) == 2 ? sixteens : kHeadSteps / 16;
#pragma unroll 1
            for (int j = r; j < sets; ++j) {
                const bool diagonal = j == r;
                float mp[2][4], mr[2][4];                 // M P and M R, transposed
                scores<NP>(mp, tile_B(s), tile_C(s), p0, 16 * j, lane);
                scores<kHeadCols>(mr, tile_u(s), tile_dy(s), p0, 16 * j, lane);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int col = 16 * j + 8 * q + 2 * t;
                    const float2 v = *reinterpret_cast<const float2 *>(pair + col);
                    float between[4] = {l0 - v.x, l0 - v.y, l1 - v.x, l1 - v.y};
                    if constexpr (sizeof(T) == 4) {
                        if (diagonal) add_low(between, f.low, p0 + g, col);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int at = col + (k & 1), row = p0 + g + (k < 2 ? 0 : 8);
                        const float vk = k & 1 ? v.y : v.x;
                        const float by = diagonal ? fast_exp2(-between[k]) : (k < 2 ? r0 : r1) * vk;
                        const bool on = !diagonal || at >= row;
                        mr[q][k] = on ? mr[q][k] * by : 0.0f;
                        const float e = on ? mr[q][k] * mp[q][k] : 0.0f;
                        mp[q][k] = on ? mp[q][k] * by : 0.0f;
                        if (k < 2)
                            k0 += e;
                        else
                            k1 += e;
                    }
                }
                join_scale<T>(mp, x, scx);
                mma_rows<kHeadCols>(x, acc_to_a<T>(mp[0], mp[1], 1.0f), tile_dy(s), 16 * j, lane);
                join_scale<T>(mr, d, scd);
                mma_rows<NP>(d, acc_to_a<T>(mr[0], mr[1], 1.0f), tile_C(s), 16 * j, lane);
            }
#pragma unroll
            for (int q = 1; q < 4; q <<= 1) {
                k0 += __shfl_xor_sync(0xffffffffu, k0, q);
                k1 += __shfl_xor_sync(0xffffffffu, k1, q);
            }
            if (t == 0) {
                dw[p0 + g] = k0 + b.x;
                dw[p0 + g + 8] = k1 + b.y;
                dot_B[p0 + g] = b.x;
                dot_B[p0 + g + 8] = b.y;
            }
            scale_rows(x, w0 * scx.down, w1 * scx.down);
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int c = 8 * n + 2 * t, step = k ? step1 : step0;
                    if (step >= a.n || c >= a.cols) continue;
                    float v0 = x[n][2 * k], v1 = x[n][2 * k + 1];
                    if (p.D) {
                        const float2 y = head_pair(tile_dy(s) + (p0 + g + 8 * k) * kXP + c);
                        v0 = fmaf(skip, y.x, v0);
                        v1 = fmaf(skip, y.y, v1);
                    }
                    T *to = du + token(step) * dy_l + c;
                    if (kWhole || p.out_unit >= 2 * static_cast<int>(sizeof(T))) {
                        head_store_pair(to, v0, v1);
                    } else {
                        to[0] = head_round<T>(v0);
                        if (c + 1 < a.cols) to[1] = head_round<T>(v1);
                    }
                }
            scale_rows(d, w0 * scd.down, w1 * scd.down);
            write_part<NP, kWhole>(d, step0 < a.n ? p.part_B + (part_row + token(step0)) * p.states : nullptr,
                                   step1 < a.n ? p.part_B + (part_row + token(step1)) * p.states : nullptr, p.states, lane);
        }
        if (next) {
            if (!rows_i)
                read_state<kWhole>(H, p.kept + ((static_cast<int64_t>(a.b) * p.chunks + chunk_of(i + 1)) * p.heads + a.h) * state_size + tile_at, p0, 0, a.cols,
                                   p.states, lane);
            if (warp == 0) {
                write_back_factors(factors[s ^ 1], head_steps(p, delta, bias, A2, chunk_of(i + 1) * kHeadSteps, a.n, lane), lane);
                if (i + 2 < count) load_delta<T>(p, delta_at, chunk_of(i + 2) * kHeadSteps, a.n, lane, delta);
            }
        }
        __syncthreads();                                  // the sums; S and G as operands, and the tiles, have been read
        if (M::kStages == 1 && next) load(chunk_of(i + 1), 0);
        if (i >= 0 && warp == 7) {
            // from the last step on C . dC', up to the step w B . dB', the pairs over it and <G, S>
            double v[2], y[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                v[k] = dot_C[2 * lane + k];
                y[k] = static_cast<double>(f.w[2 * lane + k]) * dot_B[2 * lane + k];
            }
            double after = v[0] + v[1], before = y[0] + y[1];
#pragma unroll
            for (int q = 1; q < 32; q <<= 1) {
                const double e = __shfl_down_sync(0xffffffffu, after, q), c = __shfl_up_sync(0xffffffffu, before, q);
                if (lane + q < 32) after += e;
                if (lane >= q) before += c;
            }
            after = __shfl_down_sync(0xffffffffu, after, 1);
            before = __shfl_up_sync(0xffffffffu, before, 1);
            if (lane < 31) v[1] += after;
            v[0] += v[1];
            y[1] = (lane ? before : 0.0) + y[0];
            y[0] = lane ? before : 0.0;
            const double z = static_cast<double>(through[0]) + through[1] + through[2] + through[3];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int j = 2 * lane + k;
                v[k] += y[k] + z;
                for (int q = j / 16; q < 4; ++q) v[k] += pairs[q * kHeadSteps + j];
                if (first + j < a.n) p.part_dt[part_row + token(first + j)] = make_float2(static_cast<float>(v[k]), dw[j]);
            }
        }
    }
    if (rows_i) {
        if (starts) write_state<kWhole>(H, p.final_state + head_at * state_size + tile_at, p0, 0, a.cols, p.states, lane);
#pragma unroll
        for (int q = 16; q > 0; q >>= 1) skip_grad += __shfl_xor_sync(0xffffffffu, skip_grad, q);
        if (lane == 0) skip_sum[r] = skip_grad;
    }
    __syncthreads();
    if (threadIdx.x == 0)
        p.part_D[((static_cast<int64_t>(a.tile) * p.segments + a.seg) * p.batch + a.b) * p.heads + a.h] = skip_sum[0] + skip_sum[1] + skip_sum[2] + skip_sum[3];
    griddep_launch_dependents();
}

}  // namespace ptq
