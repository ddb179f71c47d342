// Norm before or behind a block, with what stands around it in one pass:
//
//   v = x silu(gate)  (gate in front)  or x;   r = residual + scale v;   n = (r - mean) / sqrt(var + eps), or r / rms
//   y = (n weight + bias) silu(gate)  (gate behind)  or n weight + bias;   r and y are written
//
// and the gradients of all of it.  Bound: the bytes of the rows, each read and written once.  A thread owns 8 columns, whose
// parameters (and, backward, whose sums of dweight, dbias and dscale) stay in its registers, a CTA of ceil(D / 256) warps the
// whole row; it goes over the rows kRB at a time, so that one barrier serves the sums of kRB rows.  Mean and variance are
// two passes over the registers.  The norm is taken of the unrounded r, in both directions, so y does not depend on the type of r.
// Measured, 50432 x 768 bfloat16 with a binary32 residual stream: forward 82 us (5.7 TB/s), backward 115 us (6.1 TB/s) and 8 for the column sums;
// backward with the rows in registers 370, binary32 rows in half sectors 160.  16-bit rows alone are bound by issue slots: 50432 x 768 bfloat16 forward 40 us.
#pragma once

#include "ptq_block.cuh"

namespace ptq {

constexpr int kNormMaxWarps = 32;     // 8192 columns
enum { kGateNone = 0, kGateIn = 1, kGateOut = 2 };

// Where a thread's pieces of the rows lie in shared memory, in units of 16 bytes: kRB rows of each tensor that the call has.  The host makes
// it, sizes the launch's shared memory by it and hands it over, so that the two cannot differ.
struct NormStage {
    int x, residual, gate, dy, dresidual, size;
};
inline NormStage norm_stage(bool has_residual, bool has_gate, bool has_dy, bool has_dresidual, int parts, int residual_parts, int rows, int threads)
{
    const int unit = rows * threads;
    NormStage at;
    at.x = 0;
    at.residual = at.x + unit * parts;
    at.gate = at.residual + (has_residual ? unit * residual_parts : 0);
    at.dy = at.gate + (has_gate ? unit * parts : 0);
    at.dresidual = at.dy + (has_dy ? unit * parts : 0);
    at.size = at.dresidual + (has_dresidual ? unit * residual_parts : 0);
    return at;
}

struct NormParams {
    const void *x, *residual, *gate;            // residual and gate may be null
    long long x_l, residual_l, gate_l;          // pitches in elements
    const float *weight, *bias, *scale;         // each may be null
    long long rows;
    int cols, gate_at;
    float eps, inv_cols;
    bool layer;
    int stages;                                 // sets of rows in shared memory
    NormStage at;                               // of one set
    void *y, *residual_out;                     // dense
    // backward
    const void *dy, *dresidual_out;             // dense; dresidual_out may be null
    void *dx, *dresidual, *dgate;               // dense; the last two may be null
    bool sum_scale;                             // dscale is wanted
    float *part;                                // [gridDim.x][3][cols]: dweight, dbias, dscale
};

// Sums over the CTA of kV values per thread, the same in every thread.  `buf` [warps][kV]; a barrier lies between the writes and
// the reads, and the caller gives another buffer the next time.
template <int kV>
__device__ __forceinline__ void row_sums(float (&v)[kV], float *buf, int warp, int warps, int lane)
{
    lane_sums<kV, 1, 16>(v, lane);
    if (lane < kV) buf[warp * kV + first_sum<kV, 1, 16>(lane)] = v[0];
    if (warps == 1)
        __syncwarp();
    else
        __syncthreads();
    load_floats<true, kV>(v, buf, kV);
    for (int w = 1; w < warps; ++w) {
        float more[kV];
        load_floats<true, kV>(more, buf + w * kV, kV);
#pragma unroll
        for (int i = 0; i < kV; ++i) v[i] += more[i];
    }
}

// Stores eight columns of a row per lane.  Two parts of 16 bytes (binary32) would each fill half a sector: they change hands within pairs of
// lanes through `slot` (two 16-byte places of each thread, `apart` from each other), so that an instruction fills whole ones.
// Called by whole warps; `left`: columns from the lane's first one to the end of the row.
template <bool kWhole, typename V>
__device__ __forceinline__ void store_columns(V *at, const float (&f)[8], int left, uint4 *slot, int apart, int lane)
{
    if constexpr (kWhole && sizeof(V) == 4) {
        Piece<float, 8> r;
        r.set(f);
        slot[0] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
        slot[apart] = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
        __syncwarp();
        const int part = lane & 1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int owner = i - part;                    // relative to the lane
            if (left - 8 * owner >= 4 * part + 4) *reinterpret_cast<uint4 *>(at + 8 * owner + 4 * part) = slot[owner + part * apart];
        }
        __syncwarp();
    } else {
        store_piece<kWhole, V, 8>(at, f, max(min(8, left), 0));
    }
}

// kWide: rows of more than 2048 columns, up to 32 warps of 64 registers: the parameters are taken from the cache for every row.
// The rows come through shared memory, one set of kRB under way while the other is worked on (p.stages = 2; 1 where a row is too wide
// for that): held in registers, the loads of two sets would leave too few warps to keep the memory busy.
template <typename T, typename R, int kRB, bool kWide, bool kBackward, bool kWhole>
__global__ void __launch_bounds__(kWide ? 1024 : 256) ptq_norm_kernel(const NormParams p)
{
    constexpr int kStages = 3;
    constexpr int kParts = sizeof(T) / 2, kResidualParts = sizeof(R) / 2;
    __shared__ __align__(16) float s_sum[2][kStages][2 * kRB * (kWide ? kNormMaxWarps : 8)];
    extern __shared__ __align__(16) uint4 norm_rows[];
    if (kBackward) griddep_launch_dependents();
    const int threads = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = threads >> 5;
    const int c = threadIdx.x * 8, left = p.cols - c, cn = max(min(8, left), 0);
    const bool has_dr = kBackward && p.dresidual_out;
    const NormStage &at = p.at;
    float weight[8], bias[8], scale[8];
    const auto parameters = [&] {
        floats_of(weight, load_piece<kWhole, float, 8>(p.weight + c, p.weight ? cn : 0));
        floats_of(bias, load_piece<kWhole, float, 8>(p.bias + c, p.bias ? cn : 0));
        floats_of(scale, load_piece<kWhole, float, 8>(p.scale + c, p.scale ? cn : 0));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (!p.weight) weight[e] = 1.0f;
            if (!p.scale) scale[e] = 1.0f;
        }
    };
    if (!kWide) parameters();
    float sum_w[8], sum_b[8], sum_s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (kBackward) sum_w[e] = sum_b[e] = sum_s[e] = 0.0f;
    const long long step = static_cast<long long>(gridDim.x) * kRB;
    long long m0 = static_cast<long long>(blockIdx.x) * kRB;
    // the thread's part of the next set's first row
    const T *at_x = static_cast<const T *>(p.x) + m0 * p.x_l + c, *at_gate = static_cast<const T *>(p.gate) + m0 * p.gate_l + c,
            *at_dy = static_cast<const T *>(p.dy) + m0 * p.cols + c;
    const R *at_residual = static_cast<const R *>(p.residual) + m0 * p.residual_l + c, *at_dr = static_cast<const R *>(p.dresidual_out) + m0 * p.cols + c;
    const auto fetch = [&](long long m, int stage) {
        uint4 *to = norm_rows + stage * at.size + threadIdx.x;
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            const int n = m + i < p.rows ? cn : 0;
            stage_piece<kWhole, T, 8>(to + at.x + i * kParts * threads, at_x + i * p.x_l, n, threads);
            if (p.residual) stage_piece<kWhole, R, 8>(to + at.residual + i * kResidualParts * threads, at_residual + i * p.residual_l, n, threads);
            if (p.gate) stage_piece<kWhole, T, 8>(to + at.gate + i * kParts * threads, at_gate + i * p.gate_l, n, threads);
            if (kBackward) stage_piece<kWhole, T, 8>(to + at.dy + i * kParts * threads, at_dy + static_cast<long long>(i) * p.cols, n, threads);
            if (has_dr) stage_piece<kWhole, R, 8>(to + at.dresidual + i * kResidualParts * threads, at_dr + static_cast<long long>(i) * p.cols, n, threads);
        }
        stage_group();
        at_x += step * p.x_l;
        at_residual += step * p.residual_l;
        at_gate += step * p.gate_l;
        at_dy += step * p.cols;
        at_dr += step * p.cols;
    };
    if (p.stages == 2 && m0 < p.rows) fetch(m0, 0);
    long long out = m0 * p.cols + c;                      // where the thread's part of the set's first row goes
    for (int parity = 0; m0 < p.rows; m0 += step, out += step * p.cols, parity ^= 1) {
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
        uint4 *from = norm_rows + (p.stages == 2 ? parity * at.size : 0) + threadIdx.x;
        const auto x_of = [&](int i) { return staged_piece<T, 8>(from + at.x + i * kParts * threads, threads); };
        const auto gate_of = [&](int i) { return staged_piece<T, 8>(from + at.gate + i * kParts * threads, threads); };
        if (kWide) parameters();
        float r[kRB][8], mean[kRB], rstd[kRB];
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            floats_of(r[i], x_of(i));
            if (p.gate_at == kGateIn) {
                const Piece<T, 8> g = gate_of(i);
#pragma unroll
                for (int e = 0; e < 8; ++e) r[i][e] *= g[e] * sigmoid_f32(g[e]);
            }
            if (p.residual) {
                float res[8];
                floats_of(res, staged_piece<R, 8>(from + at.residual + i * kResidualParts * threads, threads));
                fma_each<8>(r[i], scale, r[i], res);
            } else if (p.scale) {
                mul_each<8>(r[i], scale, r[i]);
            }
            if (!kBackward && p.residual_out && m0 + i < p.rows) {
                R *to = static_cast<R *>(p.residual_out) + out + static_cast<long long>(i) * p.cols;
                if (p.residual)
                    store_columns<kWhole, R>(to, r[i], left, from + at.residual + i * kResidualParts * threads, threads, lane);
                else
                    store_piece<kWhole, R, 8>(to, r[i], cn);
            }
        }
        if (p.layer) {
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                float s[4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) add_pair(s[e], s[e + 1], r[i][e], r[i][e + 1], r[i][e + 4], r[i][e + 5]);
                add_pair(s[0], s[1], s[0], s[1], s[2], s[3]);
                mean[i] = s[0] + s[1];
            }
            row_sums<kRB>(mean, s_sum[parity][0], warp, warps, lane);
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                const float m = -mean[i] * p.inv_cols;
#pragma unroll
                for (int e = 0; e < 8; e += 2) add_pair(r[i][e], r[i][e + 1], r[i][e], r[i][e + 1], m, m);
                if (cn < 8) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e >= cn) r[i][e] = 0.0f;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kRB; ++i) rstd[i] = dot_each<8>(r[i], r[i]);
        row_sums<kRB>(rstd, s_sum[parity][1], warp, warps, lane);
#pragma unroll
        for (int i = 0; i < kRB; ++i) {
            rstd[i] = rsqrtf(fmaf(rstd[i], p.inv_cols, p.eps));
            if (kBackward && i > 0 && m0 + i >= p.rows) rstd[i] = 0.0f;             // no row: zeros, whose 1 / rms is infinite without eps
            mul_each<8>(r[i], rstd[i], r[i]);                                        // n from here on
        }
        if constexpr (!kBackward) {
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                if (m0 + i >= p.rows) break;
                fma_each<8>(r[i], r[i], weight, bias);
                if (p.gate_at == kGateOut) {
                    const Piece<T, 8> g = gate_of(i);
#pragma unroll
                    for (int e = 0; e < 8; ++e) r[i][e] *= g[e] * sigmoid_f32(g[e]);
                }
                store_columns<kWhole, T>(static_cast<T *>(p.y) + out + static_cast<long long>(i) * p.cols, r[i], left, from + at.x + i * kParts * threads, threads,
                                         lane);
            }
        } else {
            float sums[2 * kRB], dn[kRB][8];
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                floats_of(dn[i], staged_piece<T, 8>(from + at.dy + i * kParts * threads, threads));
                if (p.gate_at == kGateOut) {
                    const Piece<T, 8> g = gate_of(i);
                    float dg[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float z = g[e], s = sigmoid_f32(z);
                        dg[e] = dn[i][e] * fmaf(r[i][e], weight[e], bias[e]) * s * fmaf(z, 1.0f - s, 1.0f);
                        dn[i][e] *= z * s;
                    }
                    if (m0 + i < p.rows) store_piece<kWhole, T, 8>(static_cast<T *>(p.dgate) + out + static_cast<long long>(i) * p.cols, dg, cn);
                }
                fma_each<8>(sum_w, dn[i], r[i], sum_w);
                add_each<8>(sum_b, dn[i], sum_b);
                mul_each<8>(dn[i], dn[i], weight);
                sums[2 * i] = dot_each<8>(dn[i], r[i]);
                float s[4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) add_pair(s[e], s[e + 1], dn[i][e], dn[i][e + 1], dn[i][e + 4], dn[i][e + 5]);
                add_pair(s[0], s[1], s[0], s[1], s[2], s[3]);
                sums[2 * i + 1] = s[0] + s[1];
            }
            row_sums<2 * kRB>(sums, s_sum[parity][2], warp, warps, lane);
#pragma unroll
            for (int i = 0; i < kRB; ++i) {
                if (m0 + i >= p.rows) break;
                const float along = -sums[2 * i] * p.inv_cols, flat = p.layer ? -sums[2 * i + 1] * p.inv_cols : 0.0f;
                const long long row = out + static_cast<long long>(i) * p.cols;
                fma_each<8>(dn[i], along, r[i], dn[i]);
#pragma unroll
                for (int e = 0; e < 8; e += 2) add_pair(dn[i][e], dn[i][e + 1], dn[i][e], dn[i][e + 1], flat, flat);
                float dr[8], v[8], dx[8];
                if (has_dr) {
                    floats_of(dr, staged_piece<R, 8>(from + at.dresidual + i * kResidualParts * threads, threads));
                    fma_each<8>(dr, rstd[i], dn[i], dr);
                } else {
                    mul_each<8>(dr, rstd[i], dn[i]);
                }
                if (p.dresidual) {
                    if (p.residual)
                        store_columns<kWhole, R>(static_cast<R *>(p.dresidual) + row, dr, left, from + at.residual + i * kResidualParts * threads, threads, lane);
                    else
                        store_piece<kWhole, R, 8>(static_cast<R *>(p.dresidual) + row, dr, cn);
                }
                floats_of(v, x_of(i));
                mul_each<8>(dx, dr, scale);
                if (p.gate_at == kGateIn) {
                    const Piece<T, 8> g = gate_of(i);
                    float dg[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float z = g[e], s = sigmoid_f32(z), silu = z * s;
                        dg[e] = dx[e] * v[e] * s * fmaf(z, 1.0f - s, 1.0f);
                        dx[e] *= silu;
                        v[e] *= silu;
                    }
                    store_piece<kWhole, T, 8>(static_cast<T *>(p.dgate) + row, dg, cn);
                }
                if (p.sum_scale) fma_each<8>(sum_s, dr, v, sum_s);
                store_columns<kWhole, T>(static_cast<T *>(p.dx) + row, dx, left, from + at.x + i * kParts * threads, threads, lane);
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
    griddep_wait();
    const int col = blockIdx.x * 32 + (threadIdx.x & 31);
    float *out = blockIdx.y == 0 ? dweight : blockIdx.y == 1 ? dbias : dscale;
    if (!out) return;
    const float v = sum_rows<32>(part + static_cast<long long>(blockIdx.y) * cols + col, rows, 3ll * cols, col < cols, s);
    if (threadIdx.x < 32 && col < cols) out[col] = v;
}

}  // namespace ptq
