// Linear attention with a decay for each head (include/ptq_heads.h): what its kernels share, and the forward pass.
//
// A chunk of 64 steps is taken as matrix products.  With L_i the sum of dt A over the chunk's steps up to i, w_j the factor of
// an input (dt or 1) and S the state in front of the chunk:
//     y_i = sum_{j <= i} e^{L_i - L_j} w_j (C_i . B_j) u_j  +  e^{L_i} S C_i  (+ D u_i)
//     S  <- e^{L_64} S + sum_j e^{L_64 - L_j} w_j u_j B_j^T
// A CTA walks over the chunks of a sequence for 64 columns of a head.  Eight warps: four have 16 steps of each chunk (scores and
// outputs), four 16 columns of the state, which stay in registers in binary32 from chunk to chunk.
//
// The products are mma.sync on 16-bit operands: per chunk they are 64 x 64 x (16 .. 128), the scores go from one product's
// accumulators through exponentials into the next one's operand and the state's update needs its operand in two halves (the
// state is binary32), which all happens in the registers of a warp without a barrier; tcgen05 would move each of these
// matrices through TMEM and shared memory with a hand-over between warps each time.  binary32 activations: the same with tf32
// operands in two parts, three products for one.
//
// e^{L_i - L_j} is formed without a quotient of large numbers: the sums L are binary64, a warp's 16 steps refer to the sum in front
// of them, so that each factor of an earlier step is one exponential per column of scores and one per row, and only the 16 x 16
// block on the diagonal needs one per element.  For that block the sums themselves are kept: behind steps that leave nothing of the state
// they are large and their differences are not.  A step counts as 2^-256 at most, so the sums are below 16 x 256; in binary32 their rounding is
// 2^-15.5 of a factor behind one such step, 2^-12.5 behind fifteen.  That is below half a step of the 16-bit types; binary32 activations
// have what the rounding leaves beside it (in all types: 2 % of the batch's time).
//
// 16-bit activations: scores times decays, and the state where C is multiplied by it, are rounded to the type as operands; each is off by half a step
// of itself, as y is of y.  Against 64 bits y is off by 2.5e-4 of its size in binary16 and 2.1e-3 in bfloat16, where y rounded alone is by 2.1e-4 and
// 1.7e-3; the results of a training step by 2.9e-4 and 2.3e-3.  Operands in two parts would be half as many products again.
//
// What bounds it: the latency of dependent instructions.  128 x 197 x 12 heads of 64 columns, 128 states, binary16: 134 us, 0.7 TB/s of the
// bytes that count and 93 TFLOP/s; issue slots 42 % busy, the tensor pipe 33 %, stalls fixed latency 2.1, barriers 2.0, shared
// memory 1.5 per instruction.  The states and sums of a CTA fill half of an SM's registers, so two CTAs are all there are.  One warp for 16
// steps and 16 columns of the state (four warps to a CTA) took 235 us; roles of warps of their own, factors formed a chunk ahead by
// one warp, 16 earlier steps at a time and separate kernels for aligned rows (instruction cache) made the difference.  The factors on
// a warp of the outputs instead of the states were no gain (1 image 14.4 -> 16.4 us).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "ptx_griddep.cuh"

namespace ptq {

constexpr int kHeadSteps = 64;        // of a chunk
constexpr int kHeadCols = 64;         // columns of a head that a CTA has
constexpr unsigned kHeadsSoftplus = 1u, kHeadsReverse = 2u, kHeadsUnscaled = 4u;
constexpr double kLog2e = 1.4426950408889634074;

struct HeadParams {
    const void *u, *delta, *B, *C, *dy;
    int64_t u_b, u_l, u_h, delta_b, delta_l, delta_h, B_b, B_l, B_g, C_b, C_l, C_g;
    const float *A, *D, *delta_bias, *state;
    const int32_t *lengths;
    void *y;
    float *final_state, *history;
    float *slots, *logs;              // of the segments: states [batch, heads, segments, cols, states], log2 of their decays [batch, heads, segments]
    int batch, length, heads, cols, states, groups, group_heads;
    int col_tiles, segments, segment_chunks, chunks;
    int unit, out_unit;               // bytes that rows of the inputs, of y can be moved at a time
    bool share;                       // forward: the states' warps take some of the outputs' products
    unsigned flags;
    // backward pass
    const float *kept, *dfinal;
    void *du;
    float *part_B, *part_C;           // [col_tiles, heads, batch, length, states]
    float2 *part_dt;                  // [col_tiles, heads, batch, length]: gradients of the log decay and of w
    float *part_D;                    // [col_tiles, segments, batch, heads]
};

// ---------------------------------------------------------------------------------------------------- fragments
// Operands of one 16 x 8 x 16 product as the lanes of a warp hold them (g = lane / 4, t = lane % 4): of the 16 x 16 operand rows g and
// g + 8, columns 2t, 2t + 1, 2t + 8, 2t + 9; of the 16 x 8 one the same rows of its column g.  binary32: two products of 8.
template <typename T>
struct HeadA { uint32_t r[4]; };
template <>
struct HeadA<float> { float v[8]; };
template <typename T>
struct HeadB { uint32_t r[2]; };
template <>
struct HeadB<float> { float v[4]; };

constexpr int kHeadPad = 8;           // elements between the rows of a tile in shared memory, against bank conflicts

// Number of this warp, known to the compiler to be the same for all of its lanes.
__device__ __forceinline__ int head_warp() { return __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x) >> 5, 0); }

__device__ __forceinline__ uint32_t head_smem(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], const void *p)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(head_smem(p)) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], const void *p)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(head_smem(p)) : "memory");
}

// The 16 x 16 operand at rows m0, columns k0 of a tile [m][k].
template <typename T>
__device__ __forceinline__ HeadA<T> load_a(const T *tile, int pitch, int m0, int k0, int lane)
{
    HeadA<T> a;
    if constexpr (sizeof(T) == 2) {
        ldsm4(a.r, tile + (m0 + (lane & 15)) * pitch + k0 + (lane >> 4) * 8);
    } else {
        const T *p = tile + (m0 + (lane >> 2)) * pitch + k0 + 2 * (lane & 3);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 v = *reinterpret_cast<const float2 *>(p + (i & 1) * 8 * pitch + (i >> 1) * 8);
            a.v[2 * i] = v.x;
            a.v[2 * i + 1] = v.y;
        }
    }
    return a;
}
// The same from a tile [k][m].
template <typename T>
__device__ __forceinline__ HeadA<T> load_a_t(const T *tile, int pitch, int m0, int k0, int lane)
{
    HeadA<T> a;
    if constexpr (sizeof(T) == 2) {
        ldsm4t(a.r, tile + (k0 + (lane >> 4) * 8 + (lane & 7)) * pitch + m0 + ((lane >> 3) & 1) * 8);
    } else {
        const T *p = tile + (k0 + 2 * (lane & 3)) * pitch + m0 + (lane >> 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) a.v[i] = p[((i & 1) + (i >> 2) * 8) * pitch + ((i >> 1) & 1) * 8];
    }
    return a;
}
// Two 16 x 8 operands, columns n0 .. n0 + 15, rows k0 .. k0 + 15, of a tile [n][k].
template <typename T>
__device__ __forceinline__ void load_b(HeadB<T> (&b)[2], const T *tile, int pitch, int n0, int k0, int lane)
{
    if constexpr (sizeof(T) == 2) {
        uint32_t r[4];
        ldsm4(r, tile + (n0 + (lane >> 4) * 8 + (lane & 7)) * pitch + k0 + ((lane >> 3) & 1) * 8);
        b[0].r[0] = r[0], b[0].r[1] = r[1], b[1].r[0] = r[2], b[1].r[1] = r[3];
    } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const T *p = tile + (n0 + 8 * j + (lane >> 2)) * pitch + k0 + 2 * (lane & 3);
            const float2 lo = *reinterpret_cast<const float2 *>(p), hi = *reinterpret_cast<const float2 *>(p + 8);
            b[j].v[0] = lo.x, b[j].v[1] = lo.y, b[j].v[2] = hi.x, b[j].v[3] = hi.y;
        }
    }
}
// The same from a tile [k][n].
template <typename T>
__device__ __forceinline__ void load_b_t(HeadB<T> (&b)[2], const T *tile, int pitch, int n0, int k0, int lane)
{
    if constexpr (sizeof(T) == 2) {
        uint32_t r[4];
        ldsm4t(r, tile + (k0 + ((lane >> 3) & 1) * 8 + (lane & 7)) * pitch + n0 + (lane >> 4) * 8);
        b[0].r[0] = r[0], b[0].r[1] = r[1], b[1].r[0] = r[2], b[1].r[1] = r[3];
    } else {
        const T *p = tile + (k0 + 2 * (lane & 3)) * pitch + n0 + (lane >> 2);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) b[j].v[i] = p[((i & 1) + (i >> 1) * 8) * pitch + 8 * j];
    }
}

template <typename T>
__device__ __forceinline__ uint32_t head_pack(float lo, float hi)
{
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
}
template <typename T>
__device__ __forceinline__ float2 head_unpack(uint32_t v)
{
    if constexpr (std::is_same<T, __half>::value)
        return __half22float2(*reinterpret_cast<const __half2 *>(&v));
    else
        return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v));
}
__device__ __forceinline__ float head_f32(float v) { return v; }
__device__ __forceinline__ float head_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float head_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T head_round(float v)
{
    if constexpr (std::is_same<T, __half>::value)
        return __float2half_rn(v);
    else if constexpr (std::is_same<T, __nv_bfloat16>::value)
        return __float2bfloat16_rn(v);
    else
        return v;
}
// Two neighbouring elements.
template <typename T>
__device__ __forceinline__ float2 head_pair(const T *p)
{
    if constexpr (sizeof(T) == 2)
        return head_unpack<T>(*reinterpret_cast<const uint32_t *>(p));
    else
        return *reinterpret_cast<const float2 *>(p);
}
template <typename T>
__device__ __forceinline__ void head_store_pair(T *p, float x, float y)
{
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint32_t *>(p) = head_pack<T>(x, y);
    else
        *reinterpret_cast<float2 *>(p) = make_float2(x, y);
}

// Operand from the accumulators of two 8-column tiles, times `scale`.
template <typename T>
__device__ __forceinline__ HeadA<T> acc_to_a(const float (&lo)[4], const float (&hi)[4], float scale)
{
    HeadA<T> a;
    if constexpr (sizeof(T) == 2) {
        a.r[0] = head_pack<T>(lo[0] * scale, lo[1] * scale);
        a.r[1] = head_pack<T>(lo[2] * scale, lo[3] * scale);
        a.r[2] = head_pack<T>(hi[0] * scale, hi[1] * scale);
        a.r[3] = head_pack<T>(hi[2] * scale, hi[3] * scale);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a.v[i] = lo[i];
            a.v[4 + i] = hi[i];
        }
    }
    return a;
}

__device__ __forceinline__ uint32_t to_tf32(float v)
{
    uint32_t r;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// d = a b + c.  binary32: both operands as two tf32 parts (22 bits), the product of the two lower parts left out (2^-22 of the terms);
// the tensor cores' sums are cut off rather than rounded, so these 16 terms are summed on their own and added to the others rounded.
template <typename T>
__device__ __forceinline__ void head_mma(float (&d)[4], const HeadA<T> &a, const HeadB<T> &b, float c0, float c1, float c2, float c3)
{
    if constexpr (std::is_same<T, __half>::value) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a.r[0]), "r"(a.r[1]), "r"(a.r[2]), "r"(a.r[3]), "r"(b.r[0]), "r"(b.r[1]), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
            : "r"(a.r[0]), "r"(a.r[1]), "r"(a.r[2]), "r"(a.r[3]), "r"(b.r[0]), "r"(b.r[1]), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
    } else {
        uint32_t ah[8], al[8], bh[4], bl[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ah[i] = to_tf32(a.v[i]);
            al[i] = to_tf32(a.v[i] - __uint_as_float(ah[i]));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bh[i] = to_tf32(b.v[i]);
            bl[i] = to_tf32(b.v[i] - __uint_as_float(bh[i]));
        }
        // the order of the inner index is the same on both sides: element 2t in place t, 2t + 1 in place t + 4
        float e[4] = {};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            mma_tf32(e, al[4 * k], al[4 * k + 2], al[4 * k + 1], al[4 * k + 3], bh[2 * k], bh[2 * k + 1]);
            mma_tf32(e, ah[4 * k], ah[4 * k + 2], ah[4 * k + 1], ah[4 * k + 3], bl[2 * k], bl[2 * k + 1]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) mma_tf32(e, ah[4 * k], ah[4 * k + 2], ah[4 * k + 1], ah[4 * k + 3], bh[2 * k], bh[2 * k + 1]);
        d[0] = c0 + e[0];
        d[1] = c1 + e[1];
        d[2] = c2 + e[2];
        d[3] = c3 + e[3];
    }
}
// d += a b; with `fresh` d = a b.
template <typename T>
__device__ __forceinline__ void head_mma(float (&d)[4], const HeadA<T> &a, const HeadB<T> &b, bool fresh = false)
{
    if (fresh)
        head_mma(d, a, b, 0.0f, 0.0f, 0.0f, 0.0f);
    else
        head_mma(d, a, b, d[0], d[1], d[2], d[3]);
}

// Operands of more bits than the activations' type has: two binary16 or three bfloat16 values that add up to one of 22 or 24 bits
// (binary32: head_mma splits).
template <typename T>
constexpr int kHeadParts = std::is_same<T, __half>::value ? 2 : std::is_same<T, __nv_bfloat16>::value ? 3 : 1;
template <typename T>
__device__ __forceinline__ void head_split(float x, float y, uint32_t (&r)[kHeadParts<T>])
{
#pragma unroll
    for (int q = 0; q < kHeadParts<T>; ++q) {
        r[q] = head_pack<T>(x, y);
        const float2 v = head_unpack<T>(r[q]);
        x -= v.x;
        y -= v.y;
    }
}

// ---------------------------------------------------------------------------------------------------- powers of two for binary16
// An operand that is formed here may leave binary16's range; its rows are scaled by a power of two that brings their largest
// magnitude to about 2^13.  (bfloat16 has binary32's range.)
template <typename T>
constexpr bool kScaled = std::is_same<T, __half>::value;

__device__ __forceinline__ float finite_abs(float v)
{
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b < 0x7f800000u ? __uint_as_float(b) : 0.0f;
}
// The largest of a warp's values, none of them negative: their bits are in the same order.
__device__ __forceinline__ float warp_max(float v) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v))); }
// The largest magnitude of a warp's values; if that is infinite, of the finite ones (the others are lost whatever their scale).
template <int N>
__device__ __forceinline__ float warp_top(const float (&d)[N][4])
{
    float top = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        top = fmaxf(top, fmaxf(fabsf(d[n][0]), fabsf(d[n][1])));
        top = fmaxf(top, fmaxf(fabsf(d[n][2]), fabsf(d[n][3])));
    }
    top = warp_max(top);
    if (__float_as_uint(top) >= 0x7f800000u) {
        top = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) top = fmaxf(top, finite_abs(d[n][k]));
        top = warp_max(top);
    }
    return top;
}
struct HeadScale {
    float up, down;
};
// The power of two, within 2^-126 .. 2^most, that brings `top` into 2^to .. 2^(to + 1), and its inverse.
__device__ __forceinline__ HeadScale exact_scale(float top, int to, int most)
{
    const int e = top == 0.0f ? 0 : max(-126, min(most, to + 127 - static_cast<int>(__float_as_uint(top) >> 23)));
    return {__uint_as_float(static_cast<uint32_t>(127 + e) << 23), __uint_as_float(static_cast<uint32_t>(127 - e) << 23)};
}
// Into 2^13 .. 2^14; 1 where `top` is 2^-4 .. 2^15: what binary16 cannot hold is less than 2^-21 of it then, and what need not be scaled is
// not.  `most`: 126 for states, which a growing chunk makes large from however small; 60 for operands whose products join sums that
// are scaled with them (smaller ones vanish beside what binary16 holds in the result).
template <int kMost>
__device__ __forceinline__ HeadScale scale_for(float top)
{
    if (top >= 0.0625f && top < 32768.0f) return {1.0f, 1.0f};
    return exact_scale(top, 13, kMost);
}
constexpr int kScaleSums = 60, kScaleState = 126;

// ---------------------------------------------------------------------------------------------------- loads
__device__ __forceinline__ void cp_async(uint32_t dst, const void *src, int bytes, bool on)
{
    const int n = on ? bytes : 0;                        // what is not copied is filled with zeros
    if (bytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else if (bytes == 8)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// 64 rows of kWidth elements into a tile: row r from src + r * step, zeros from `rows` and from column `cols` on.  kWhole: 16 bytes at a
// time; else in units of 8, 4 or (through registers) 2 bytes that divide the rows.  (Two kernels: what the general one needs
// would crowd the instruction cache of the other.)
template <int kWidth, int kThreads, bool kWhole, typename T>
__device__ __forceinline__ void load_rows(T *tile, const T *src, int64_t step, int rows, int cols, int unit)
{
    constexpr int kPitch = kWidth + kHeadPad;
    const auto go = [&](auto bytes) {
        constexpr int kBytes = decltype(bytes)::value, kElems = kBytes / static_cast<int>(sizeof(T)), kRow = kWidth / kElems, kAt = kThreads / kRow;
        static_assert(kThreads % kRow == 0 && kHeadSteps % kAt == 0, "a thread has one place of all its rows");
        const int r0 = threadIdx.x / kRow, c = threadIdx.x % kRow * kElems;
        const T *from = src + r0 * step + c;
        uint32_t to = head_smem(tile + r0 * kPitch + c);
        int left = c < cols ? rows - r0 : 0;
#pragma unroll
        for (int i = 0; i < kHeadSteps / kAt; ++i) {
            cp_async(to, left > 0 ? from : src, kBytes, left > 0);
            from += kAt * step;
            to += kAt * kPitch * static_cast<int>(sizeof(T));
            left -= kAt;
        }
    };
    if constexpr (kWhole) {
        go(std::integral_constant<int, 16>());
    } else if (unit >= 8) {
        go(std::integral_constant<int, 8>());
    } else if (unit == 4) {
        go(std::integral_constant<int, 4>());
    } else if constexpr (sizeof(T) == 2) {
        for (int i = threadIdx.x; i < kHeadSteps * kWidth; i += kThreads) {
            const int r = i / kWidth, c = i % kWidth;
            tile[r * kPitch + c] = r < rows && c < cols ? src[r * step + c] : head_round<T>(0.0f);
        }
    }
}

// ---------------------------------------------------------------------------------------------------- steps of a chunk
// A lane has steps 2 lane and 2 lane + 1 of a chunk.
struct HeadSteps {
    float dt[2], w[2];
    double sum[2];                    // log2 of the decays up to and with the step
};
__device__ __forceinline__ float head_softplus(float e) { return e > 20.0f ? e : log1pf(expf(e)); }
__device__ __forceinline__ float head_dt(const HeadParams &p, float delta, float bias)
{
    if (!p.delta) return 1.0f;
    const float e = delta + bias;
    return p.flags & kHeadsSoftplus ? head_softplus(e) : e;
}
// delta of the two steps of a lane; n: steps of the sequence
template <typename T>
__device__ __forceinline__ void load_delta(const HeadParams &p, int64_t at, int first, int n, int lane, float (&v)[2])
{
    const T *d = static_cast<const T *>(p.delta);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = first + 2 * lane + k;
        v[k] = d && i < n ? head_f32(d[at + (p.flags & kHeadsReverse ? n - 1 - i : i) * p.delta_l]) : 0.0f;
    }
}
// A2 = A log2 e.  Below 2^-256 a step's decay counts as that: nothing in binary32, whatever growth up to 2^127 is beside it, and -inf does no
// harm in differences.
__device__ __forceinline__ HeadSteps head_steps(const HeadParams &p, const float (&delta)[2], float bias, double A2, int first, int n, int lane)
{
    HeadSteps s;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const bool on = first + 2 * lane + k < n;
        s.dt[k] = on ? head_dt(p, delta[k], bias) : 0.0f;
        s.w[k] = !on ? 0.0f : p.flags & kHeadsUnscaled ? 1.0f : s.dt[k];
        double a = s.dt[k] == 0.0f ? 0.0 : static_cast<double>(s.dt[k]) * A2;
        if (a < -256.0) a = -256.0;
        s.sum[k] = a;
    }
    s.sum[1] += s.sum[0];
    double all = s.sum[1];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double x = __shfl_up_sync(0xffffffffu, all, d);
        if (lane >= d) all += x;
    }
    // not by differences: what comes behind a NaN must not reach what is in front of it
    const double before = __shfl_up_sync(0xffffffffu, all, 1);
    if (lane) {
        s.sum[0] += before;
        s.sum[1] = all;
    }
    return s;
}
__device__ __forceinline__ double sum_at(const HeadSteps &s, int step) { return __shfl_sync(0xffffffffu, s.sum[step & 1], step >> 1); }
// ex2.approx: 2 units in the last place; results below 2^-126 become zero.
__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float pow2(double x) { return fast_exp2(static_cast<float>(x)); }

// What a CTA works on.
struct HeadPlace {
    int b, h, g, tile, seg, n;        // n: steps of the sequence
    int cols;                         // of this tile
};
__device__ __forceinline__ HeadPlace head_place(const HeadParams &p, int segments)
{
    HeadPlace a;
    int i = static_cast<int>(blockIdx.x);
    a.seg = i % segments;
    i /= segments;
    a.tile = i % p.col_tiles;
    i /= p.col_tiles;
    a.h = i % p.heads;
    a.b = i / p.heads;
    a.g = a.h / p.group_heads;
    a.n = p.lengths ? max(0, min(p.length, __ldg(p.lengths + a.b))) : p.length;
    a.cols = min(kHeadCols, p.cols - a.tile * kHeadCols);
    return a;
}

// state[p][n] <- decay state + sum_j f_j x_j[p] z_j[n] over a chunk, for 16 columns p0 .. and 8 kN states n0 ..; x and z are tiles
// [step][..].  The factors make x an operand of more than 16 bits: it goes in in parts.
template <int NP, int kN, typename T>
__device__ __forceinline__ void state_update(float (&S)[kN][4], const T *x, const T *z, const float *f, float decay, int p0, int n0, int sets, int lane)
{
    constexpr int kXP = kHeadCols + kHeadPad, kZP = NP + kHeadPad;
    const int t = lane & 3;
    if constexpr (kScaled<T>) {
        // binary16, 16 steps at a time: of each u is brought to less than 2^8 and the factors to less than 2^7, so that the product stays below 2^15, all
        // bits of what is 2^-22 of the largest u stay, and 2^-31 of the largest factor.  Eight lanes have the powers of two of 16 steps.
        const float2 q = *reinterpret_cast<const float2 *>(f + 2 * lane);
        float top_f = fmaxf(finite_abs(q.x), finite_abs(q.y)), top_u = 0.0f;
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) top_f = fmaxf(top_f, __shfl_xor_sync(0xffffffffu, top_f, d));
#pragma unroll
        for (int k = 0; k < kHeadSteps / 16; ++k) {
            const HeadA<T> a = load_a_t(x, kXP, p0, 16 * k, lane);
            __half2 most = __habs2(*reinterpret_cast<const __half2 *>(&a.r[0]));
#pragma unroll
            for (int i = 1; i < 4; ++i) most = __hmax2(most, __habs2(*reinterpret_cast<const __half2 *>(&a.r[i])));
            const float2 m = __half22float2(most);
            const float top = warp_max(fminf(fmaxf(m.x, m.y), 65504.0f));              // an infinity counts as the largest finite value
            if (lane >> 3 == k) top_u = top;
        }
        const HeadScale scu = exact_scale(top_u, 7, 15), scf = exact_scale(top_f, 6, 126);             // (2^15: a power of two that binary16 holds)
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[n][i] *= decay;
#pragma unroll 1
        for (int k = 0; k < sets; ++k) {
            const HeadA<T> a = load_a_t(x, kXP, p0, 16 * k, lane);
            const float up_u = __shfl_sync(0xffffffffu, scu.up, 8 * k), up_f = __shfl_sync(0xffffffffu, scf.up, 8 * k);
            const float down = __shfl_sync(0xffffffffu, scu.down * scf.down, 8 * k);
            const float2 f0 = *reinterpret_cast<const float2 *>(f + 16 * k + 2 * t), f1 = *reinterpret_cast<const float2 *>(f + 16 * k + 2 * t + 8);
            // u f as two binary16 values in binary16 arithmetic: f in two parts, the product with the upper one and what its
            // rounding left (a fused multiply-add leaves it whole), plus that with the lower one
            uint32_t fh[2], fl[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t r[2];
                head_split<T>((c ? f1.x : f0.x) * up_f, (c ? f1.y : f0.y) * up_f, r);
                fh[c] = r[0];
                fl[c] = r[1];
            }
            const __half2 up = __float2half2_rn(up_u);
            HeadA<T> upper, lower;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __half2 v = __hmul2(*reinterpret_cast<const __half2 *>(&a.r[i]), up);
                const __half2 h = *reinterpret_cast<const __half2 *>(&fh[i >> 1]), l = *reinterpret_cast<const __half2 *>(&fl[i >> 1]);
                const __half2 hi = __hmul2_rn(v, h), lo = __hfma2(v, l, __hfma2(v, h, __hneg2(hi)));
                upper.r[i] = *reinterpret_cast<const uint32_t *>(&hi);
                lower.r[i] = *reinterpret_cast<const uint32_t *>(&lo);
            }
#pragma unroll
            for (int n = 0; n < kN / 2; ++n) {
                HeadB<T> b[2];
                load_b_t(b, z, kZP, n0 + 16 * n, 16 * k, lane);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float sum[4];
                    head_mma(sum, lower, b[j], true);
                    head_mma(sum, upper, b[j]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) S[2 * n + j][i] = fmaf(sum[i], down, S[2 * n + j][i]);
                }
            }
        }
    } else {
        HeadA<T> a[kHeadSteps / 16];
#pragma unroll
        for (int k = 0; k < kHeadSteps / 16; ++k) a[k] = load_a_t(x, kXP, p0, 16 * k, lane);
        // the chunk's sums on their own, joined with the state in binary32: the tensor cores' sums are cut off, not rounded
        // (beside all states of 16 columns three parts of 64 steps are too many registers: 32 steps at a time)
        constexpr int kSet = kHeadParts<T> > 2 && kN > 8 ? 2 : 4;
#pragma unroll
        for (int k0 = 0; k0 < kHeadSteps / 16; k0 += kSet) {
            HeadA<T> part[kSet][kHeadParts<T>];
#pragma unroll
            for (int ks = 0; ks < kSet; ++ks) {
                const int k = k0 + ks;
                const float2 f0 = *reinterpret_cast<const float2 *>(f + 16 * k + 2 * t), f1 = *reinterpret_cast<const float2 *>(f + 16 * k + 2 * t + 8);
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 v = head_unpack<T>(a[k].r[i]), q = i < 2 ? f0 : f1;
                        uint32_t r[kHeadParts<T>];
                        head_split<T>(v.x * q.x, v.y * q.y, r);
#pragma unroll
                        for (int j = 0; j < kHeadParts<T>; ++j) part[ks][j].r[i] = r[j];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) part[ks][0].v[i] = a[k].v[i] * (i < 4 ? (i & 1 ? f0.y : f0.x) : (i & 1 ? f1.y : f1.x));
                }
            }
#pragma unroll
            for (int n = 0; n < kN / 2; ++n) {
                float sum[2][4];
#pragma unroll
                for (int ks = 0; ks < kSet; ++ks) {
                    HeadB<T> b[2];
                    load_b_t(b, z, kZP, n0 + 16 * n, 16 * (k0 + ks), lane);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int q = kHeadParts<T> - 1; q >= 0; --q) head_mma(sum[j], part[ks][q], b[j], ks == 0 && q == kHeadParts<T> - 1);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float &to = S[2 * n + j][i];
                        to = k0 == 0 ? fmaf(decay, to, sum[j][i]) : to + sum[j][i];
                    }
            }
        }
    }
}

// A warp's part of a state in memory [cols][states]: rows p0 + g and p0 + g + 8, columns n0 + 8 n + 2 t of it.
template <int kN, class Fn>
__device__ __forceinline__ void for_state(int p0, int n0, int cols, int states, int lane, Fn fn)
{
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = p0 + g + (i >> 1) * 8, c = n0 + 8 * n + 2 * t + (i & 1);
            fn(n, i, p < cols && c < states, static_cast<int64_t>(p) * states + c);
        }
}
// kWhole: two values at a time.
template <bool kWhole, int kN>
__device__ __forceinline__ void read_state(float (&S)[kN][4], const float *from, int p0, int n0, int cols, int states, int lane)
{
    if constexpr (kWhole) {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = p0 + g + 8 * i, c = n0 + 8 * n + 2 * t;
                float2 v = make_float2(0.0f, 0.0f);
                if (from && p < cols && c < states) v = *reinterpret_cast<const float2 *>(from + static_cast<int64_t>(p) * states + c);
                S[n][2 * i] = v.x;
                S[n][2 * i + 1] = v.y;
            }
    } else {
        for_state<kN>(p0, n0, cols, states, lane, [&](int n, int i, bool on, int64_t at) { S[n][i] = on && from ? from[at] : 0.0f; });
    }
}
template <bool kWhole, int kN>
__device__ __forceinline__ void write_state(const float (&S)[kN][4], float *to, int p0, int n0, int cols, int states, int lane)
{
    if constexpr (kWhole) {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = p0 + g + 8 * i, c = n0 + 8 * n + 2 * t;
                if (p < cols && c < states) *reinterpret_cast<float2 *>(to + static_cast<int64_t>(p) * states + c) = make_float2(S[n][2 * i], S[n][2 * i + 1]);
            }
    } else {
        for_state<kN>(p0, n0, cols, states, lane, [&](int n, int i, bool on, int64_t at) {
            if (on) to[at] = S[n][i];
        });
    }
}

// ---------------------------------------------------------------------------------------------------- forward pass
enum HeadMode {
    kHeadForward,                     // outputs and final states
    kHeadSum,                         // what a segment adds to the state, and its decay
    kHeadGradSum,                     // what a segment's outputs add to the gradient of the state in front of it, and its decay
};

// Factors of a chunk's steps, which one warp forms for all, a chunk ahead.  The sums refer to the step in front of each 16 steps r.
template <typename T>
struct HeadFactors {
    float state[kHeadSteps];          // of an input in the state behind the chunk (gradients: of an output in the one in front)
    float w[kHeadSteps];
    float into[kHeadSteps];           // e^{L}
    float pair[4][kHeadSteps];        // for the 16 steps r: of the steps in front of them e^{L_ref - L_j} w_j, of themselves log2 e^{L_j - L_ref}
    float low[sizeof(T) == 4 ? kHeadSteps : 2];           // binary32 activations: what is left of that logarithm
    float decay, log_decay;           // of the chunk, log2 of it
    float pad[2];
};
// What binary32 leaves of the logarithms of a lane's steps, which refer to the step in front of their 16.
__device__ __forceinline__ void write_low(float *low, const HeadSteps &st, int lane)
{
    const double ref = __shfl_sync(0xffffffffu, st.sum[1], ((lane & 24) - 1) & 31), own = lane < 8 ? 0.0 : ref, x = st.sum[0] - own, y = st.sum[1] - own;
    reinterpret_cast<float2 *>(low)[lane] = make_float2(static_cast<float>(x - static_cast<float>(x)), static_cast<float>(y - static_cast<float>(y)));
}
// d: of the rows row, row + 8 the differences with the columns col, col + 1.
__device__ __forceinline__ void add_low(float (&d)[4], const float *low, int row, int col)
{
    const float2 z = *reinterpret_cast<const float2 *>(low + col);
    const float z0 = low[row], z1 = low[row + 8];
    d[0] += z0 - z.x;
    d[1] += z0 - z.y;
    d[2] += z1 - z.x;
    d[3] += z1 - z.y;
}
template <int kMode, typename T>
__device__ __forceinline__ void write_factors(HeadFactors<T> &f, const HeadSteps &st, int lane)
{
    const double all = __shfl_sync(0xffffffffu, st.sum[1], 31);
    float2 *to = reinterpret_cast<float2 *>(&f) + lane;
    constexpr int kRow = kHeadSteps / 2;
    if constexpr (kMode == kHeadGradSum)
        to[0] = make_float2(pow2(st.sum[0]), pow2(st.sum[1]));
    else
        to[0] = make_float2(pow2(all - st.sum[0]) * st.w[0], pow2(all - st.sum[1]) * st.w[1]);
    if constexpr (kMode == kHeadForward) {
        to[kRow] = make_float2(st.w[0], st.w[1]);
        to[2 * kRow] = make_float2(pow2(st.sum[0]), pow2(st.sum[1]));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const double ref = r ? __shfl_sync(0xffffffffu, st.sum[1], 8 * r - 1) : 0.0;
            to[(3 + r) * kRow] = lane < 8 * r ? make_float2(pow2(ref - st.sum[0]) * st.w[0], pow2(ref - st.sum[1]) * st.w[1])
                                              : make_float2(static_cast<float>(st.sum[0] - ref), static_cast<float>(st.sum[1] - ref));
        }
        if constexpr (sizeof(T) == 4) write_low(f.low, st, lane);
    }
    if (lane == 0) {
        f.decay = pow2(all);
        // nothing of the state in front of the chunk comes through it: no growth behind it in the segment brings that back
        f.log_decay = f.decay == 0.0f ? -1e30f : static_cast<float>(all);
    }
}

// Shared memory of the forward kernel, in bytes: two stages of tiles (u, B, C; sums: u or dy, and one of B and C), the state as an
// operand, staging, factors of two chunks, powers of two of the state's columns.
template <typename T, int NP, int kMode>
struct HeadSmem {
    static constexpr int kWide = kHeadSteps * (NP + kHeadPad) * static_cast<int>(sizeof(T));
    static constexpr int kNarrow = kHeadSteps * (kHeadCols + kHeadPad) * static_cast<int>(sizeof(T));
    static constexpr int kStage = (kMode == kHeadForward ? 2 : 1) * kWide + kNarrow;
    static constexpr int kStages = 2 * kStage + (kMode == kHeadForward ? kWide : 0) <= 200 * 1024 ? 2 : 1;
    static constexpr bool kOverC = NP >= kHeadCols;                        // staging of the outputs: rows as wide as theirs
    static constexpr int kState = kStages * kStage;
    static constexpr int kStaging = kState + (kMode == kHeadForward ? kWide : 0);
    static constexpr int kFactors = kStaging + (kMode == kHeadForward && sizeof(T) == 2 && !kOverC ? kNarrow : 0);
    static constexpr int kPowers = kFactors + 2 * static_cast<int>(sizeof(HeadFactors<T>));
    // what the states' warps add to outputs, 16 x 64 binary32 sums each: over the state's operand where that is large enough
    static constexpr bool kOverState = kWide >= 4 * 4096;
    static constexpr int kHelp = kOverState ? kState : kPowers + 4 * 4;
    static constexpr int kBytes = kPowers + 4 * 4 + (kMode == kHeadForward && !kOverState ? 4 * 4096 : 0);
};

// Whether an operand holds an infinity or NaN (zero times it is not zero).
template <typename T, int N>
__device__ __forceinline__ bool not_finite(const HeadB<T> (&v)[N][2])
{
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 zero = __float2half2_rn(0.0f);
        __half2 sum = zero;
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) sum = __hfma2(*reinterpret_cast<const __half2 *>(&v[i / 4][i / 2 % 2].r[i % 2]), zero, sum);
        const float2 f = __half22float2(sum);
        return f.x + f.y != 0.0f;
    } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        const __nv_bfloat162 zero = __float2bfloat162_rn(0.0f);
        __nv_bfloat162 sum = zero;
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) sum = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&v[i / 4][i / 2 % 2].r[i % 2]), zero, sum);
        const float2 f = __bfloat1622float2(sum);
        return f.x + f.y != 0.0f;
    } else {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8 * N; ++i) sum = fmaf(v[i / 8][i / 4 % 2].v[i % 4], 0.0f, sum);
        return sum != 0.0f;
    }
}

// Zeros in the place of such values.
template <typename T, int N>
__device__ __forceinline__ void only_finite(HeadB<T> (&v)[N][2])
{
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) {
        if constexpr (sizeof(T) == 2) {
            constexpr uint32_t kExp = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
            uint32_t &x = v[i / 4][i / 2 % 2].r[i % 2];
            if ((x & kExp) == kExp) x &= 0xffff0000u;
            if ((x >> 16 & kExp) == kExp) x &= 0x0000ffffu;
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float &x = v[i / 4][i / 2 % 2].v[2 * (i % 2) + k];
                x = isfinite(x) ? x : 0.0f;
            }
        }
    }
}

template <typename T, int NP, int kMode, bool kWhole>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) ptq_heads_kernel(const HeadParams p)
{
    using M = HeadSmem<T, NP, kMode>;
    constexpr int kWP = NP + kHeadPad, kXP = kHeadCols + kHeadPad;
    constexpr int kN = NP / (kMode == kHeadForward ? 8 : 16);                            // 8-column tiles of a warp's states
    constexpr bool kOut = kMode == kHeadForward, kGrad = kMode == kHeadGradSum;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = head_warp(), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // Outputs: warps 0 .. 3 have 16 steps each, 4 .. 7 16 columns of the state.  (The last steps have four times the first ones' scores: in the
    // CTAs that share an SM, as many apart as there are SMs, on different schedulers.)  Sums: two warps 16 columns, half of the states each.
    const bool outputs = kOut && warp < 4;
    const int r = outputs && (blockIdx.x / 148) & 1 ? 3 - warp : warp & 3, p0 = 16 * r, n0 = kOut ? 0 : (warp >> 2) * (NP / 2);
    if (kOut && p.segments > 1) griddep_wait();
    const HeadPlace a = head_place(p, kOut ? p.segments : p.segments - 1);
    const int seg = kGrad ? a.seg + 1 : a.seg;            // sums: of all segments but the last, of gradients: but the first
    const int chunks = (a.n + kHeadSteps - 1) / kHeadSteps;
    const int chunk0 = min(chunks, seg * p.segment_chunks), chunk1 = min(chunks, chunk0 + p.segment_chunks);
    const bool reverse = p.flags & kHeadsReverse;
    const auto tile_u = [&](int s) { return reinterpret_cast<T *>(smem + (M::kStages == 2 ? s * M::kStage : 0)); };
    const auto tile_B = [&](int s) { return reinterpret_cast<T *>(smem + (M::kStages == 2 ? s * M::kStage : 0) + M::kNarrow); };
    const auto tile_C = [&](int s) { return reinterpret_cast<T *>(smem + (M::kStages == 2 ? s * M::kStage : 0) + M::kNarrow + M::kWide); };
    T *state_s = reinterpret_cast<T *>(smem + M::kState);
    HeadFactors<T> *factors = reinterpret_cast<HeadFactors<T> *>(smem + M::kFactors);
    float *powers = reinterpret_cast<float *>(smem + M::kPowers);
    float4 *help = reinterpret_cast<float4 *>(smem + M::kHelp);

    const T *u = static_cast<const T *>(kGrad ? p.dy : p.u) +
                 (kGrad ? (static_cast<int64_t>(a.b) * p.length * p.heads + a.h) * p.cols : a.b * p.u_b + a.h * p.u_h) + a.tile * kHeadCols;
    const int64_t u_l = kGrad ? static_cast<int64_t>(p.heads) * p.cols : p.u_l;
    const T *B = static_cast<const T *>(kGrad ? p.C : p.B) + (kGrad ? a.b * p.C_b + a.g * p.C_g : a.b * p.B_b + a.g * p.B_g);
    const int64_t B_l = kGrad ? p.C_l : p.B_l;
    const T *C = static_cast<const T *>(p.C) + a.b * p.C_b + a.g * p.C_g;
    const int64_t delta_at = a.b * p.delta_b + a.h * p.delta_h;
    const float bias = p.delta_bias ? __ldg(p.delta_bias + a.h) : 0.0f, skip = p.D ? __ldg(p.D + a.h) : 0.0f;
    const double A2 = static_cast<double>(__ldg(p.A + a.h)) * kLog2e;
    const int64_t y_l = static_cast<int64_t>(p.heads) * p.cols;
    T *y_at = static_cast<T *>(p.y) + (static_cast<int64_t>(a.b) * p.length * p.heads + a.h) * p.cols + a.tile * kHeadCols;

    const auto token = [&](int step) { return reverse ? a.n - 1 - step : step; };
    const auto load = [&](int chunk, int s) {
        const int first = chunk * kHeadSteps, rows = a.n - first;
        const int64_t sign = reverse ? -1 : 1, at = token(first);
        load_rows<kHeadCols, 256, kWhole>(tile_u(s), u + at * u_l, sign * u_l, rows, a.cols, p.unit);
        load_rows<NP, 256, kWhole>(tile_B(s), B + at * B_l, sign * B_l, rows, p.states, p.unit);
        if (kOut) load_rows<NP, 256, kWhole>(tile_C(s), C + at * p.C_l, sign * p.C_l, rows, p.states, p.unit);
        cp_async_commit();
    };

    const int64_t head_at = (static_cast<int64_t>(a.b) * p.heads + a.h);
    const int64_t state_size = static_cast<int64_t>(p.cols) * p.states, tile_at = static_cast<int64_t>(a.tile) * kHeadCols * p.states;
    const int count = chunk1 - chunk0;
    const auto chunk_of = [&](int i) { return kGrad ? chunk1 - 1 - i : chunk0 + i; };
    float S[kN][4];
    {
        const float *from = nullptr;
        // with segments the first one's start is a copy: the last one may be writing final_state over it
        if (kOut && p.segments > 1 && (seg > 0 || p.state))
            from = p.slots + (head_at * p.segments + (seg > 0 ? seg : p.segments) - 1) * state_size + tile_at;
        else if (kOut && p.state)
            from = p.state + head_at * state_size + tile_at;
        if (!outputs) read_state<kWhole>(S, from, p0, n0, a.cols, p.states, lane);
    }
    const bool started = kOut && (seg > 0 || p.state);    // else the state in front of the first chunk is zero
    // this segment holds the last step (or is the first one of an empty sequence): its state is the final one
    const bool ends = kOut && p.final_state && seg == (chunks > 0 ? (chunks - 1) / p.segment_chunks : 0);
    double log_decay = 0.0;
    const bool busy = !outputs && p0 < a.cols;            // this warp has columns of the state
    // the state as an operand: its columns brought into binary16's range
    const auto publish = [&](int chunk) {
        if (p.history && busy)
            write_state<kWhole>(S, p.history + ((static_cast<int64_t>(a.b) * p.chunks + chunk) * p.heads + a.h) * state_size + tile_at, p0, n0, a.cols, p.states, lane);
        HeadScale sc = {1.0f, 1.0f};
        if constexpr (kScaled<T>) {
            sc = scale_for<kScaleState>(warp_top<kN>(S));
            if (lane == 0) powers[r] = sc.down;
        }
        const auto store = [&](float by) {
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                head_store_pair(state_s + (p0 + g) * kWP + 8 * n + 2 * t, S[n][0] * by, S[n][1] * by);
                head_store_pair(state_s + (p0 + g + 8) * kWP + 8 * n + 2 * t, S[n][2] * by, S[n][3] * by);
            }
        };
        if (sc.up == 1.0f)
            store(1.0f);
        else
            store(sc.up);
    };
    // Tiles come a chunk ahead.  Of warps 4 .. 7 the one with the number of the chunk forms the factors of its steps a chunk ahead; it has read
    // delta a chunk before that.
    float delta[2] = {};
    if (warp == 4 && count > 0) load_delta<T>(p, delta_at, chunk_of(0) * kHeadSteps, a.n, lane, delta);
    for (int i = -1; i < count; ++i) {
        const int chunk = chunk_of(i), first = chunk * kHeadSteps, s = i & 1;
        const bool next = i + 1 < count;
        if (i >= 0) {
            cp_async_wait<0>();
            __syncthreads();                              // the tiles, their steps' factors, and the state as an operand; the last chunk is done
        }
        if (M::kStages == 2 && next) load(chunk_of(i + 1), s ^ 1);
        const HeadFactors<T> &f = factors[s];
        const int sixteens = (min(a.n - first, kHeadSteps) + 15) / 16;                  // sets of 16 steps that are there
        if (outputs && i >= 0) {
            const float *pair = f.pair[r];
            const float l0 = pair[p0 + g], l1 = pair[p0 + g + 8], r0 = fast_exp2(l0), r1 = fast_exp2(l1);
            float y[8][4] = {};
            if ((i > 0 || started) && r < sixteens) {      // what the state gives these 16 steps
#pragma unroll 2
                for (int k = 0; k < NP / 16; ++k) {
                    const HeadA<T> c = load_a(tile_C(s), kWP, p0, 16 * k, lane);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        HeadB<T> b[2];
                        load_b(b, state_s, kWP, 16 * j, 16 * k, lane);
                        head_mma(y[2 * j], c, b[0]);
                        head_mma(y[2 * j + 1], c, b[1]);
                    }
                }
                const float R0 = f.into[p0 + g], R1 = f.into[p0 + g + 8];
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const float down = kScaled<T> ? powers[n / 2] : 1.0f;
                    y[n][0] *= R0 * down;
                    y[n][1] *= R0 * down;
                    y[n][2] *= R1 * down;
                    y[n][3] *= R1 * down;
                }
            }
            asm volatile("bar.arrive 1, 256;" ::: "memory");           // the state and its powers have been read
            // and what the steps up to them give, 16 at a time, the ones on the diagonal last
            const int j0 = p.share ? (r + 1) / 2 : 0;      // the ones before: by the states' warps
            HeadScale sc = {1.0f, 1.0f};
#pragma unroll 1
            for (int j = j0; j <= r && r < sixteens; ++j) {
                const bool diagonal = j == r;
                float m[2][4], odd[2][4];                  // two chains of products each
#pragma unroll
                for (int k = 0; k < NP / 16; k += 2) {
                    HeadB<T> b[2], e[2];
                    load_b(b, tile_B(s), kWP, 16 * j, 16 * k, lane);
                    const HeadA<T> c = load_a(tile_C(s), kWP, p0, 16 * k, lane);
                    load_b(e, tile_B(s), kWP, 16 * j, 16 * k + 16, lane);
                    const HeadA<T> d = load_a(tile_C(s), kWP, p0, 16 * k + 16, lane);
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        head_mma(m[n], c, b[n], k == 0);
                        head_mma(odd[n], d, e[n], k == 0);
                    }
                }
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const int col = 16 * j + 8 * n + 2 * t;
                    const float2 v = *reinterpret_cast<const float2 *>(pair + col);
                    float f00, f01, f10, f11;              // factors of the rows p0 + g and p0 + g + 8
                    if (!diagonal) {
                        f00 = r0 * v.x;
                        f01 = r0 * v.y;
                        f10 = r1 * v.x;
                        f11 = r1 * v.y;
                    } else {
                        const float2 w = *reinterpret_cast<const float2 *>(f.w + col);
                        float d[4] = {l0 - v.x, l0 - v.y, l1 - v.x, l1 - v.y};
                        if constexpr (sizeof(T) == 4) add_low(d, f.low, p0 + g, col);
                        f00 = fast_exp2(d[0]) * w.x;
                        f01 = fast_exp2(d[1]) * w.y;
                        f10 = fast_exp2(d[2]) * w.x;
                        f11 = fast_exp2(d[3]) * w.y;
                    }
                    const int row = diagonal ? p0 + g : kHeadSteps;                    // in front of the diagonal all count
                    m[n][0] = col <= row ? (m[n][0] + odd[n][0]) * f00 : 0.0f;
                    m[n][1] = col + 1 <= row ? (m[n][1] + odd[n][1]) * f01 : 0.0f;
                    m[n][2] = col <= row + 8 ? (m[n][2] + odd[n][2]) * f10 : 0.0f;
                    m[n][3] = col + 1 <= row + 8 ? (m[n][3] + odd[n][3]) * f11 : 0.0f;
                }
                if constexpr (kScaled<T>) {                // y goes along to the units of these scores, unless they are all zero
                    const float top = warp_top<2>(m);
                    const HeadScale now = top == 0.0f ? sc : scale_for<kScaleSums>(top);
                    if (now.up != sc.up) {
                        const float by = now.up * sc.down;
#pragma unroll
                        for (int n = 0; n < 8; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k) y[n][k] *= by;
                        sc = now;
                    }
                }
                if (kScaled<T> && sc.up != 1.0f) {
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) m[n][k] *= sc.up;
                }
                HeadB<T> v[4][2];
#pragma unroll
                for (int q = 0; q < 4; ++q) load_b_t(v[q], tile_u(s), kXP, 16 * q, 16 * j, lane);
                // On the diagonal columns of later steps have the factor zero; where u is not finite there, zero times it is not zero: it stays out
                // of the product and goes where it belongs by itself, so that the other rows and columns are the same as without it.
                const bool odd_u = diagonal && __any_sync(0xffffffffu, not_finite<T>(v));
                if (odd_u) only_finite<T>(v);
                const HeadA<T> w = acc_to_a<T>(m[0], m[1], 1.0f);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    head_mma(y[2 * q], w, v[q][0]);
                    head_mma(y[2 * q + 1], w, v[q][1]);
                }
                if (odd_u) {
#pragma unroll 1
                    for (int c = 0; c < 16; ++c) {
                        const int from = (lane & 28) + (c & 7) / 2;
                        const float e0 = c < 8 ? (c & 1 ? m[0][1] : m[0][0]) : (c & 1 ? m[1][1] : m[1][0]);
                        const float e1 = c < 8 ? (c & 1 ? m[0][3] : m[0][2]) : (c & 1 ? m[1][3] : m[1][2]);
                        const float w0 = __shfl_sync(0xffffffffu, e0, from), w1 = __shfl_sync(0xffffffffu, e1, from);
#pragma unroll
                        for (int n = 0; n < 8; ++n) {
                            const float2 x = head_pair(tile_u(s) + (16 * j + c) * kXP + 8 * n + 2 * t);
                            const bool on0 = !isfinite(x.x), on1 = !isfinite(x.y);
                            if (c <= g && on0) y[n][0] = fmaf(w0, x.x, y[n][0]);
                            if (c <= g && on1) y[n][1] = fmaf(w0, x.y, y[n][1]);
                            if (c <= g + 8 && on0) y[n][2] = fmaf(w1, x.x, y[n][2]);
                            if (c <= g + 8 && on1) y[n][3] = fmaf(w1, x.y, y[n][3]);
                        }
                    }
                }
            }
            if (kScaled<T> && sc.down != 1.0f) {
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[n][k] *= sc.down;
            }
            if (p.share) {
                asm volatile("bar.sync 2, 256;" ::: "memory");         // the others' sums are there
                const auto add = [&](int from) {
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        const float4 v = help[from * 256 + n * 32 + lane];
                        y[n][0] += v.x;
                        y[n][1] += v.y;
                        y[n][2] += v.z;
                        y[n][3] += v.w;
                    }
                };
                if (r > 0) add(r == 3 ? 0 : 4 - r);
                if (r == 3) add(1);
                if (M::kOverState) asm volatile("bar.arrive 3, 256;" ::: "memory");
            }
            const int step0 = first + p0 + g, step1 = step0 + 8;
            // through shared memory (16-bit values: over this warp's rows of C) to whole 16-byte stores.  Of the states' warps, which read these rows
            // where they share the work, barrier 2 has come after that; they read no others' rows of C otherwise.
            T *stage = M::kOverC ? tile_C(s) + p0 * kWP : reinterpret_cast<T *>(smem + M::kStaging) + p0 * kXP;
            if (M::kOverC) __syncwarp();
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int c = 8 * n + 2 * t, step = k ? step1 : step0;
                    float v0 = y[n][2 * k], v1 = y[n][2 * k + 1];
                    if (p.D) {
                        const float2 x = head_pair(tile_u(s) + (p0 + g + 8 * k) * kXP + c);
                        v0 = fmaf(skip, x.x, v0);
                        v1 = fmaf(skip, x.y, v1);
                    }
                    if (sizeof(T) == 2 && kWhole) {
                        head_store_pair(stage + (g + 8 * k) * kXP + c, v0, v1);
                    } else if (step < a.n && c < a.cols) {
                        T *to = y_at + token(step) * y_l + c;
                        if (kWhole || p.out_unit >= 2 * static_cast<int>(sizeof(T))) {
                            head_store_pair(to, v0, v1);
                        } else {
                            to[0] = head_round<T>(v0);
                            if (c + 1 < a.cols) to[1] = head_round<T>(v1);
                        }
                    }
                }
            if (sizeof(T) == 2 && kWhole) {
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int row = 4 * q + (lane >> 3), c = 8 * (lane & 7), step = first + p0 + row;
                    if (step < a.n && c < a.cols)
                        *reinterpret_cast<uint4 *>(y_at + token(step) * y_l + c) = *reinterpret_cast<const uint4 *>(stage + row * kXP + c);
                }
            }
        }
        if (kOut && !outputs && i >= 0 && p.share) {
            // The last steps have four sets of 16 steps up to them, the first ones one: the states' warps take one each, of the steps
            // 48 .. 63 the first two, of 32 .. 47 and of 16 .. 31 the first.  A chunk is shorter for it (1 image 16.4 -> 14.4 us; 128 x 197 x 12 heads,
            // binary16, 144.7 -> 141.6), but with operands in three parts and two CTAs to an SM the states' warps are the slower ones
            // (bfloat16, 2 x 20011 x 16 heads: 349 -> 368 us): not there.
            const int hr = r == 0 ? 3 : 4 - r, hj = r == 1 ? 1 : 0;
            if (hr < sixteens) {
                const float *pair = f.pair[hr];
                float m[2][4];
#pragma unroll
                for (int k = 0; k < NP / 16; ++k) {
                    HeadB<T> b[2];
                    load_b(b, tile_B(s), kWP, 16 * hj, 16 * k, lane);
                    const HeadA<T> c = load_a(tile_C(s), kWP, 16 * hr, 16 * k, lane);
                    head_mma(m[0], c, b[0], k == 0);
                    head_mma(m[1], c, b[1], k == 0);
                }
                const float r0 = fast_exp2(pair[16 * hr + g]), r1 = fast_exp2(pair[16 * hr + g + 8]);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float2 v = *reinterpret_cast<const float2 *>(pair + 16 * hj + 8 * n + 2 * t);
                    m[n][0] *= r0 * v.x;
                    m[n][1] *= r0 * v.y;
                    m[n][2] *= r1 * v.x;
                    m[n][3] *= r1 * v.y;
                }
                HeadScale sc = {1.0f, 1.0f};
                if constexpr (kScaled<T>) sc = scale_for<kScaleSums>(warp_top<2>(m));
                const HeadA<T> w = acc_to_a<T>(m[0], m[1], sc.up);
                if (M::kOverState) asm volatile("bar.sync 1, 256;" ::: "memory");              // the outputs' warps have read the state
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    HeadB<T> b[2];
                    load_b_t(b, tile_u(s), kXP, 16 * q, 16 * hj, lane);
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        float x[4];
                        head_mma(x, w, b[n], true);
                        help[r * 256 + (2 * q + n) * 32 + lane] = make_float4(x[0] * sc.down, x[1] * sc.down, x[2] * sc.down, x[3] * sc.down);
                    }
                }
            } else if (M::kOverState) {
                asm volatile("bar.sync 1, 256;" ::: "memory");
            }
            asm volatile("bar.arrive 2, 256;" ::: "memory");
        }
        if (i >= 0) {
            log_decay += f.log_decay;
            if (busy && (!kOut || next || ends)) state_update<NP, kN>(S, tile_u(s), tile_B(s), f.state, f.decay, p0, n0, sixteens, lane);
            // the outputs' warps have read the state, or what lies over it
            if (kOut && !outputs) asm volatile("bar.sync %0, 256;" ::"r"(M::kOverState && p.share ? 3 : 1) : "memory");
        }
        if (kOut && !outputs && next) publish(chunk_of(i + 1));
        if (warp == 4 + ((i + 1) & 3) && next)
            write_factors<kMode>(factors[s ^ 1], head_steps(p, delta, bias, A2, chunk_of(i + 1) * kHeadSteps, a.n, lane), lane);
        if (warp == 4 + ((i + 2) & 3) && i + 2 < count) load_delta<T>(p, delta_at, chunk_of(i + 2) * kHeadSteps, a.n, lane, delta);
        if (M::kStages == 1 && next) {
            __syncthreads();
            load(chunk_of(i + 1), 0);
        }
    }
    if constexpr (kOut) {
        if (!outputs && ends)
            write_state<kWhole>(S, p.final_state + head_at * state_size + tile_at, p0, n0, a.cols, p.states, lane);
    } else {
        write_state<kWhole>(S, p.slots + (head_at * p.segments + seg) * state_size + tile_at, p0, n0, a.cols, p.states, lane);
        if (threadIdx.x == 0 && a.tile == 0) p.logs[head_at * p.segments + seg] = static_cast<float>(log_decay);
        griddep_launch_dependents();
    }
}

// ---------------------------------------------------------------------------------------------------- single tokens
// One step of many sequences: bound by reading and writing the binary32 states once.  kLanes lanes have a row of a state (4 values
// each), a CTA 32 rows of one head (8 rows of 128 states in flight per warp); everything is binary32.  256 sequences of 24 heads, 64
// columns, 128 states: 70 us in a loop, 5.8 TB/s, 76 between other work, 5.3 TB/s (92 us without the streaming loads and stores, which leave the L2 to the rest).
template <typename T, int kLanes, bool kWhole>
__global__ void __launch_bounds__(128) ptq_heads_step_kernel(const HeadParams p)
{
    constexpr int kAt = 128 / kLanes, kRows = kLanes / 4;                               // rows at a time, times
    const int tiles = (p.cols + kAt * kRows - 1) / (kAt * kRows);
    int i = static_cast<int>(blockIdx.x);
    const int col0 = i % tiles * (kAt * kRows) + threadIdx.x / kLanes;
    i /= tiles;
    const int h = i % p.heads, b = i / p.heads, g = h / p.group_heads, n0 = threadIdx.x % kLanes * 4;
    const bool on = !p.lengths || __ldg(p.lengths + b) > 0;
    const int64_t head = static_cast<int64_t>(b) * p.heads + h, base = head * p.cols * p.states;
    const float *from = p.state ? p.state + base : nullptr;
    float v[kRows][4];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int c = col0 + r * kAt;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[r][k] = 0.0f;
        if (!from || c >= p.cols) continue;
        const float *row = from + static_cast<int64_t>(c) * p.states + n0;
        if constexpr (kWhole) {
            if (n0 < p.states) {
                const float4 x = __ldcs(reinterpret_cast<const float4 *>(row));
                v[r][0] = x.x, v[r][1] = x.y, v[r][2] = x.z, v[r][3] = x.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (n0 + k < p.states) v[r][k] = row[k];
        }
    }
    const float delta = p.delta && on ? head_f32(static_cast<const T *>(p.delta)[b * p.delta_b + h * p.delta_h]) : 0.0f;
    const float dt = on ? head_dt(p, delta, p.delta_bias ? __ldg(p.delta_bias + h) : 0.0f) : 0.0f;
    const float decay = dt == 0.0f ? 1.0f : expf(dt * __ldg(p.A + h)), w = !on ? 0.0f : p.flags & kHeadsUnscaled ? 1.0f : dt;
    const T *Bp = static_cast<const T *>(p.B) + b * p.B_b + g * p.B_g + n0, *Cp = static_cast<const T *>(p.C) + b * p.C_b + g * p.C_g + n0;
    float B[4], C[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const bool in = on && n0 + k < p.states;
        B[k] = in ? head_f32(Bp[k]) : 0.0f;
        C[k] = in ? head_f32(Cp[k]) : 0.0f;
    }
    const T *u = static_cast<const T *>(p.u) + b * p.u_b + h * p.u_h;
    const float skip = p.D ? __ldg(p.D + h) : 0.0f;
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int c = col0 + r * kAt;
        const float x = on && c < p.cols ? head_f32(u[c]) : 0.0f, wx = w * x;
        float y = 0.0f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (on) v[r][k] = from ? fmaf(decay, v[r][k], wx * B[k]) : wx * B[k];
            y = n0 + k < p.states ? fmaf(v[r][k], C[k], y) : y;
        }
#pragma unroll
        for (int d = kLanes / 2; d > 0; d >>= 1) y += __shfl_xor_sync(0xffffffffu, y, d);
        if (c >= p.cols) continue;
        if (p.final_state) {
            float *row = p.final_state + base + static_cast<int64_t>(c) * p.states + n0;
            if constexpr (kWhole) {
                if (n0 < p.states) __stcs(reinterpret_cast<float4 *>(row), make_float4(v[r][0], v[r][1], v[r][2], v[r][3]));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (n0 + k < p.states) row[k] = v[r][k];
            }
        }
        if (on && n0 == 0) static_cast<T *>(p.y)[head * p.cols + c] = head_round<T>(p.D ? fmaf(skip, x, y) : y);
    }
}

}  // namespace ptq
