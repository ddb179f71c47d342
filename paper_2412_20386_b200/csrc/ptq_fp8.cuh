// Linears in e4m3 with a scale for each block of 128 values (include/ptq_fp8.h): quantize kernels and the product on the
// tensor cores.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "ptx_sm100.cuh"

namespace ptq {

constexpr int kFp8Block = 128;                 // values that share a scale; one k-block of the product
constexpr float kFp8Max = 448.0f;
constexpr float kFp8Least = 0x1p-100f;         // a block's largest magnitude counts as this at least: both quotients stay finite

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// max(a, |b|) that keeps a NaN of either side.
__device__ __forceinline__ float max_abs_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}

// Eight values of a row from column c on, zeros from `cols` on, as they are stored.  kWhole: 16 bytes at a time; rows begin on multiples of
// 16 bytes and cols is a multiple of 8.
template <typename T>
struct Eight {
    uint4 q[sizeof(T) / 2];
};
template <bool kWhole, typename T>
__device__ __forceinline__ Eight<T> load8(const T *row, int c, int cols)
{
    Eight<T> v;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) v.q[i] = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (kWhole) {
        if (c < cols) {
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) v.q[i] = __ldcs(reinterpret_cast<const uint4 *>(row + c) + i);
        }
    } else {
        T *t = reinterpret_cast<T *>(&v);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < cols) t[i] = row[c + i];
    }
    return v;
}
template <typename T>
__device__ __forceinline__ void unpack8(const Eight<T> &e, float (&v)[8])
{
    const T *t = reinterpret_cast<const T *>(&e);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(t[i]);
}

// The largest magnitude of the 128 values that 16 neighbouring lanes hold, not below kFp8Least; a NaN stays one.
template <typename T>
__device__ __forceinline__ float block_top(const Eight<T> &e)
{
    float top = kFp8Least;
    if constexpr (sizeof(T) == 2) {                       // two at a time, in the type itself
        using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        const T2 *t = reinterpret_cast<const T2 *>(&e);
        const T2 m = __hmax2_nan(__hmax2_nan(__habs2(t[0]), __habs2(t[1])), __hmax2_nan(__habs2(t[2]), __habs2(t[3])));
        top = max_abs_nan(max_abs_nan(top, to_f32(m.x)), to_f32(m.y));
    } else {
        const float *t = reinterpret_cast<const float *>(&e);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max_abs_nan(top, t[i]);
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) top = max_abs_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
    return top;
}
// Of N blocks that 16 neighbouring lanes hold, one division for all: lane i gets 448 / top[i], lane 8 + i top[i] / 448.
template <int N>
__device__ __forceinline__ float block_scales(const float (&top)[N], int l)
{
    static_assert(N <= 8, "two divisions of each block in 16 lanes");
    float t = top[0];
#pragma unroll
    for (int i = 1; i < N; ++i) t = (l & 7) == i ? top[i] : t;
    return (l < 8 ? kFp8Max : t) / (l < 8 ? t : kFp8Max);
}
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inverse)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * h] * inverse, v[4 * h + 1] * inverse), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * h + 2] * inverse, v[4 * h + 3] * inverse), __NV_SATFINITE, __NV_E4M3);
        w[h] = lo | hi << 16;
    }
    return make_uint2(w[0], w[1]);
}
template <bool kWhole>
__device__ __forceinline__ void store_codes8(uint8_t *row, int c, int cols, uint2 w)
{
    if (kWhole ? c < cols : c + 8 <= cols) {
        *reinterpret_cast<uint2 *>(row + c) = w;
    } else {
        for (int i = 0; i < 8 && c + i < cols; ++i) row[c + i] = static_cast<uint8_t>((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    }
}

// ---------------------------------------------------------------------------------------------------- quantize
// Bound by memory: 16-bit values are read, codes and a scale for each 128 of them written, once each.  Half a warp holds a block
// (16 bytes of 16-bit values a lane), kSet neighbouring ones of a row at a time; the 16 half-warps of a CTA take 16 neighbouring rows,
// whose scales lie next to each other in the layout that the product reads.  CTAs, as many as the SMs hold, go over the rows with the loads
// of the next set under way while one is worked on; one division makes all scales of a step.  (One set per CTA and a division per block:
// 26.7 us where this takes 20.7.)  50432 rows of 768 bfloat16 channels: 20.7 us where the same rows come again, 5.7 TB/s, 22.7 to 24.0 on others each time,
// 4.9 to 5.2 TB/s; of 1536 channels 41.3 and 43.0 us, 5.7 and 5.5 TB/s.
struct Fp8QuantizeParams {
    const void *x;
    int64_t x_pitch, codes_pitch, scale_row, scale_block;
    int64_t rows;
    int cols, blocks;                 // blocks of a row
    FastDiv sets;                     // sets of kSet blocks of a row
    unsigned items;                   // sets of 16 rows
    uint8_t *codes;
    float *scales;
};
constexpr int kFp8QuantizeRows = 16;
template <typename T, int kSet, bool kWhole>
__global__ void __launch_bounds__(256) ptq_fp8_quantize_kernel(const Fp8QuantizeParams p)
{
    const int h = threadIdx.x >> 4, l = threadIdx.x & 15;
    griddep_launch_dependents();
    int64_t row, next_row;
    int b0, next_b0;
    Eight<T> e[kSet], next[kSet];
    const auto load = [&](unsigned item) {
        const unsigned group = fd_div(item, p.sets);
        next_row = static_cast<int64_t>(group) * kFp8QuantizeRows + h;
        next_b0 = static_cast<int>(item - group * p.sets.d) * kSet;
        const bool on = item < p.items && next_row < p.rows;
        const T *x = static_cast<const T *>(p.x) + (on ? next_row : 0) * p.x_pitch;
#pragma unroll
        for (int i = 0; i < kSet; ++i) next[i] = load8<kWhole>(x, (next_b0 + i) * kFp8Block + 8 * l, on ? p.cols : 0);
    };
    load(blockIdx.x);
    for (unsigned item = blockIdx.x; item < p.items; item += gridDim.x) {
        row = next_row;
        b0 = next_b0;
#pragma unroll
        for (int i = 0; i < kSet; ++i) e[i] = next[i];
        load(item + gridDim.x);
        const bool on = row < p.rows;                   // the others go along: the shuffles are the warp's
        float top[kSet];
#pragma unroll
        for (int i = 0; i < kSet; ++i) top[i] = block_top(e[i]);
        const float q = block_scales(top, l);
        uint8_t *codes = p.codes + row * p.codes_pitch;
#pragma unroll
        for (int i = 0; i < kSet; ++i) {
            float v[8];
            unpack8(e[i], v);
            const uint2 w = codes8(v, __shfl_sync(0xffffffffu, q, i, 16));
            store_codes8<kWhole>(codes, (b0 + i) * kFp8Block + 8 * l, on ? p.cols : 0, w);
        }
        if (on && l >= 8 && l < 8 + kSet && b0 + l - 8 < p.blocks) p.scales[row * p.scale_row + (b0 + l - 8) * p.scale_block] = q;
    }
}

// Weights: one CTA goes over a block of 128 x 128 twice (it stays in L1), element by element.  Done once per layer.  8192 x 4096 in bfloat16: 43 us,
// 2.3 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) ptq_fp8_quantize_weight_kernel(const Fp8QuantizeParams p)
{
    __shared__ float tops[8];
    const int l = threadIdx.x & 15, h = threadIdx.x >> 4, c = blockIdx.x * kFp8Block + 8 * l;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * kFp8Block;
    float v[8], top = kFp8Least;
    for (int r = h; r < kFp8Block; r += 16) {
        const int64_t row = row0 + r;
        top = max_abs_nan(top, block_top(load8<false>(static_cast<const T *>(p.x) + (row < p.rows ? row : 0) * p.x_pitch, c, row < p.rows ? p.cols : 0)));
    }
    top = max_abs_nan(top, __shfl_xor_sync(0xffffffffu, top, 16));
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    for (int i = 0; i < 8; ++i) top = max_abs_nan(top, tops[i]);
    for (int r = h; r < kFp8Block; r += 16) {
        const int64_t row = row0 + r;
        if (row >= p.rows) break;
        unpack8(load8<false>(static_cast<const T *>(p.x) + row * p.x_pitch, c, p.cols), v);
        store_codes8<false>(p.codes + row * p.codes_pitch, c, p.cols, codes8(v, kFp8Max / top));
    }
    if (threadIdx.x == 0) p.scales[static_cast<int64_t>(blockIdx.y) * p.blocks + blockIdx.x] = top / kFp8Max;
}

// ---------------------------------------------------------------------------------------------------- product
// One k-block of 128 is one chain of four tcgen05.mma (kind::f8f6f4, binary32 accumulators in TMEM) into one of two
// accumulator buffers; the epilogue warps read the buffer, multiply it by the block's scales and add it to sums that they
// keep in registers, while the tensor pipe fills the other one.  The scales cannot go into the operands (they are not powers
// of two) nor be put off to the end (they change with every k-block).
//
// Warp 0 issues the TMA loads, warp 1 the MMAs, warps 4 .. 11 read: 32 TMEM lanes each, the two teams of four half of the
// columns each.  A tile is 128 (TMEM lanes, operand P) x BN (TMEM columns, operand Q):
//   many rows   P = activations, Q = weights.  Persistent CTAs.
//   few rows    P = weights, Q = the tokens (BN = 16, 32 or 64): no lane is wasted on rows that are not there.
// Where there are fewer tiles than SMs the k-blocks of a tile are split over a cluster of up to eight CTAs, which add their
// parts through distributed shared memory in the order of the parts.
//
// What bounds it.  8192 x 4096 -> 8192: 241 us alone (2280 TFLOP/s, 68 % of twice the library's bf16 rate; the library's bf16 product of
// this size takes 332), 285 in a long loop under the power limit: a k-block of a 128 x 256 tile is 128 columns of TMEM reads and as many fused
// multiply-adds for each of 8 warps, beside operands from L2.  Pairs of CTAs on one tile took twice as long, packed
// multiply-adds and one accumulator for each team of warps no faster.  1 x 4096 -> 4096: 6.6 us, launch and one chain of loads (2.5 TB/s
// of weights); 2048 x 2048 -> 2048 12.2 us.
struct Fp8Params {
    const float *a_scales, *w_scales, *bias;
    int64_t scale_row, scale_block;   // of a_scales
    void *y;
    int64_t y_pitch;
    const void *x;                    // fused: the activations before they are quantized
    int64_t x_pitch;
    int rows, cols, outputs, blocks;  // blocks: k-blocks
    int p_tiles, q_tiles, split;
    int stages;
    bool whole;                       // rows of y can be moved 16 bytes at a time
    unsigned *status;
};

constexpr int kFp8Threads = 384;                           // warps 0 TMA, 1 MMA, 4 .. 11 read
constexpr int kFp8MaxStages = 8;
constexpr int kFp8PTile = 128 * kFp8Block;                 // bytes of one k-block of operand P
constexpr int kFp8Staging = 4096;                          // bytes of an epilogue warp's staging: 32 rows of 128 bytes
constexpr int kFp8FusedRows = 16;                          // tokens that the CTAs quantize themselves, at most
constexpr int kFp8MaxFused = 64;                           // k-blocks of them that a CTA may hold (2 KB each)
constexpr int kFp8MaxScales = 8192;                        // scales of tokens (k-blocks x BN) that a CTA may hold

// The four MMAs of a k-block into a fresh accumulator; called by a whole warp, one lane issues.
__device__ __forceinline__ void mma_f8_kblock(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc)
{
    asm volatile(
        "{\n\t"
        ".reg .pred p, q, e;\n\t"
        "elect.sync _|e, 0xffffffff;\n\t"
        ".reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "setp.ne.b32 p, 0, 0;\n\t"
        "setp.eq.b32 q, 0, 0;\n\t"
        "add.u64 a1, %1, 2;\n\t"
        "add.u64 a2, %1, 4;\n\t"
        "add.u64 a3, %1, 6;\n\t"
        "add.u64 b1, %2, 2;\n\t"
        "add.u64 b2, %2, 4;\n\t"
        "add.u64 b3, %2, 6;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a1, b1, %3, q;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a2, b2, %3, q;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a3, b3, %3, q;\n\t"
        "}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc)
        : "memory");
}
// Instruction descriptor of kind::f8f6f4 with e4m3 operands, both K-major, and binary32 accumulators: D format [4,6) = 1,
// A and B formats [7,10), [10,13) = 0, N>>3 at [17,23), M>>4 at [24,29).
__host__ __device__ constexpr uint32_t make_idesc_e4m3(int M, int N)
{
    return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// 32 lanes x N columns (8, 16 or 32).
template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&v)[N])
{
    if constexpr (N == 32) {
        tmem_ld_32x32(taddr, v);
    } else if constexpr (N == 16) {
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
            : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
              "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
            : "r"(taddr)
            : "memory");
    } else {
        static_assert(N == 8, "8, 16 or 32 columns");
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                     : "r"(taddr)
                     : "memory");
    }
}

// Waits for this thread's TMEM loads; the values are named so that nothing reads them before.
template <int N>
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&v)[N])
{
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(v[i]));
}

// Floats of the shared memory of the CTA `rank` of the cluster, at the address that they have here.
__device__ __forceinline__ void ld_cluster(uint32_t local_addr, uint32_t rank, float (&v)[1])
{
    asm volatile(
        "{\n\t"
        ".reg .b32 ra;\n\t"
        "mapa.shared::cluster.u32 ra, %1, %2;\n\t"
        "ld.shared::cluster.f32 %0, [ra];\n\t"
        "}"
        : "=f"(v[0])
        : "r"(local_addr), "r"(rank)
        : "memory");
}
__device__ __forceinline__ void ld_cluster(uint32_t local_addr, uint32_t rank, float (&v)[4])
{
    asm volatile(
        "{\n\t"
        ".reg .b32 ra;\n\t"
        "mapa.shared::cluster.u32 ra, %4, %5;\n\t"
        "ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [ra];\n\t"
        "}"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
        : "r"(local_addr), "r"(rank)
        : "memory");
}

// Shared memory: stages of (P tile, Q tile) or, fused, stages of P tiles and all Q tiles of the CTA; staging of the epilogue
// warps (persistent kernels only); few rows: scales [k-block][BN]; barriers.
struct Fp8Layout {
    int stage, q, staging, scales, bars, bytes;
};
template <int BN, bool kSwap, bool kOneTile, bool kFused>
__host__ __device__ constexpr Fp8Layout fp8_layout(int stages, int blocks)
{
    Fp8Layout l = {};
    l.stage = kFp8PTile + (kFused ? 0 : BN * kFp8Block);
    l.q = stages * l.stage;
    l.staging = l.q + (kFused ? blocks * BN * kFp8Block : 0);
    l.scales = l.staging + (kOneTile ? 0 : 8 * kFp8Staging);
    l.bars = l.scales + (kSwap ? blocks * BN * 4 : 0);
    l.bytes = l.bars + 8 * (2 * kFp8MaxStages + 5) + 16;
    // the parts of a split tile lie over the stages, with 4 floats between the rows
    const int parts = kOneTile ? 4 * (kSwap ? BN * (128 + 4) : 128 * (BN + 4)) : 0;
    if (kOneTile && l.bars < parts) {
        l.bars = parts;
        l.bytes = l.bars + 8 * (2 * kFp8MaxStages + 5) + 16;
    }
    return l;
}

// kOneTile: one tile, or one part of one, per CTA; else persistent.  kFused: operand Q is quantized here from x; kWhole: 16 bytes at a
// time.
template <typename Y, int BN, bool kSwap, bool kOneTile, bool kFused, bool kWhole>
__global__ void __launch_bounds__(kFp8Threads, 1)
ptq_fp8_matmul_kernel(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmQ, const Fp8Params p)
{
    static_assert(!kFused || (kSwap && kOneTile), "tokens are quantized in the kernel for few rows");
    static_assert(!kSwap || kOneTile, "few rows make few tiles");
    constexpr int kCols = BN / 2;                          // columns of an epilogue warp
    constexpr int kLd = kCols < 32 ? kCols : 32;           // columns of one TMEM load
    constexpr uint32_t kTmem = 2 * BN;
    constexpr uint32_t kIdesc = make_idesc_e4m3(128, BN);
    // The sums of 128 columns and a TMEM load want more registers than 384 threads can have alike: 168 each at the launch,
    // then 4 x 32 x 40 + 8 x 32 x 232 = 64512, as many.
    constexpr bool kMoreRegs = kCols == 128;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const uint32_t base = smem_u32(smem_raw);
    if ((base & 1023u) != 0u) {                            // never expected; the same in all CTAs of a cluster
        if (threadIdx.x == 0) atomicOr(p.status, PTQ_DEV_SMEM_ALIGN);
        return;
    }
    const int rank = kOneTile ? static_cast<int>(blockIdx.x) % p.split : 0;
    const int first_tile = static_cast<int>(blockIdx.x) / (kOneTile ? p.split : 1);
    const int stride = static_cast<int>(gridDim.x) / (kOneTile ? p.split : 1);         // one tile: all of them
    const int tiles = p.p_tiles * p.q_tiles;
    // the k-blocks of this CTA
    const int kb0 = kOneTile ? static_cast<int>(static_cast<int64_t>(p.blocks) * rank / p.split) : 0;
    const int kb1 = kOneTile ? static_cast<int>(static_cast<int64_t>(p.blocks) * (rank + 1) / p.split) : p.blocks;
    const Fp8Layout at = fp8_layout<BN, kSwap, kOneTile, kFused>(p.stages, (p.blocks + p.split - 1) / p.split);
    const uint32_t nstages = static_cast<uint32_t>(p.stages);
    const uint32_t bar_base = base + at.bars;
    auto full_bar = [&](uint32_t s) { return bar_base + 8u * s; };
    auto empty_bar = [&](uint32_t s) { return bar_base + 8u * (kFp8MaxStages + s); };
    auto tfull_bar = [&](uint32_t b) { return bar_base + 8u * (2 * kFp8MaxStages + b); };
    auto tempty_bar = [&](uint32_t b) { return bar_base + 8u * (2 * kFp8MaxStages + 2 + b); };
    const uint32_t q_bar = bar_base + 8u * (2 * kFp8MaxStages + 4);
    volatile uint32_t *tmem_holder = reinterpret_cast<volatile uint32_t *>(smem_raw + at.bars + 8 * (2 * kFp8MaxStages + 5));
    volatile uint32_t *abort_flag = tmem_holder + 1;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < nstages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (uint32_t b = 0; b < 2; ++b) {
            mbar_init(tfull_bar(b), 1);
            mbar_init(tempty_bar(b), 8);
        }
        mbar_init(q_bar, 8);
        *abort_flag = 0u;
        fence_mbar_init();
        prefetch_tensormap(&tmP);
        if (!kFused) prefetch_tensormap(&tmQ);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_holder)), kTmem);
        tmem_relinquish_alloc_permit();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_holder, 0);

    // Twelve P tiles, then the next Q tile: the CTAs that run together share the operands of about 12 x 12 tiles.
    auto tile_at = [&](int tile, int &pt, int &qt) {
        const int group = tile / (12 * p.q_tiles), r = tile - group * 12 * p.q_tiles;
        const int in_group = min(12, p.p_tiles - group * 12);
        pt = group * 12 + r % in_group;
        qt = r / in_group;
    };

    if (warp < 4) {
        if constexpr (kMoreRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0) {
            // -------------------------------------------------------------- TMA producer
            uint32_t stage = 0, phase = 0, issued = 0;
            bool ok = true;
            const uint32_t tx = static_cast<uint32_t>(at.stage);       // boxes count whole, also beyond the ends
            griddep_wait();
            for (int tile = first_tile; tile < tiles && ok; tile += stride) {
                int pt, qt;
                tile_at(tile, pt, qt);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!mbar_wait_warp(empty_bar(stage), phase ^ 1u, abort_flag, p.status)) {
                        ok = false;
                        break;
                    }
                    const uint32_t dst = base + stage * static_cast<uint32_t>(at.stage);
                    mbar_arrive_expect_tx_warp(full_bar(stage), tx);
                    tma_load_2d_warp(dst, &tmP, kb * kFp8Block, pt * 128, full_bar(stage));
                    if (!kFused) tma_load_2d_warp(dst + kFp8PTile, &tmQ, kb * kFp8Block, qt * BN, full_bar(stage));
                    ++issued;
                    if (++stage == nstages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
            }
            if (!ok) {
                // Error path only: the loads in flight land before the CTA gives up its shared memory (bounded).
                for (uint32_t s = 0; s < nstages; ++s) {
                    const uint32_t uses = (issued + nstages - 1u - s) / nstages;
                    if (uses == 0u) continue;
                    for (int i = 0; i < 200000 && !mbar_try_wait(full_bar(s), (uses - 1u) & 1u); ++i) {
                    }
                }
            }
        } else if (warp == 1) {
            // -------------------------------------------------------------- MMA issuer
            uint32_t stage = 0, phase = 0, buf = 0, bphase = 0;
            bool ok = !kFused || mbar_wait_warp(q_bar, 0u, abort_flag, p.status);
            for (int tile = first_tile; tile < tiles && ok; tile += stride) {
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = mbar_wait_warp(tempty_bar(buf), bphase ^ 1u, abort_flag, p.status) &&
                         mbar_wait_warp(full_bar(stage), phase, abort_flag, p.status);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint32_t addr = base + stage * static_cast<uint32_t>(at.stage);
                    const uint32_t q_addr = kFused ? base + at.q + static_cast<uint32_t>(kb - kb0) * BN * kFp8Block : addr + kFp8PTile;
                    mma_f8_kblock(tmem_base + buf * BN, make_smem_desc_sw128(addr), make_smem_desc_sw128(q_addr), kIdesc);
                    mma_commit(empty_bar(stage));
                    mma_commit(tfull_bar(buf));
                    if (++stage == nstages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                    buf ^= 1u;
                    if (buf == 0u) bphase ^= 1u;
                }
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue warps
        if constexpr (kMoreRegs) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
        griddep_wait();
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t tmem_row = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + half * kCols;
        float *scales_s = reinterpret_cast<float *>(smem_raw + at.scales);
        const int et = static_cast<int>(threadIdx.x) - 128;            // 0 .. 255 among the epilogue threads
        if constexpr (kFused) {
            // 16 half-warps quantize the tokens of this tile, four blocks at a time each, into the layout that the MMAs read
            // (rows of 128 bytes, 16-byte units exchanged by the row's place among eight); rows that are not there are zeros
            const int l = et & 15, tokens = p.rows, items = (kb1 - kb0) * tokens;          // tokens <= BN: one Q tile
            const Y *x = static_cast<const Y *>(p.x);
            for (int i = et; i < (kb1 - kb0) * BN * (kFp8Block / 16); i += 256)
                *reinterpret_cast<uint4 *>(smem_raw + at.q + 16 * i) = make_uint4(0u, 0u, 0u, 0u);
            for (int i = et; i < (kb1 - kb0) * BN; i += 256) scales_s[i] = 0.0f;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            for (int i0 = 0; i0 < items; i0 += 64) {
                Eight<Y> e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int item = i0 + 16 * i + (et >> 4), kb = item / tokens, r = item - kb * tokens;
                    const bool on = item < items;
                    e[i] = load8<kWhole>(x + (on ? r : 0) * p.x_pitch, (kb0 + kb) * kFp8Block + 8 * l, on ? p.cols : 0);
                }
                float top[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) top[i] = block_top(e[i]);
                const float q = block_scales(top, l);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int item = i0 + 16 * i + (et >> 4), kb = item / tokens, r = item - kb * tokens;
                    float v[8];
                    unpack8(e[i], v);
                    const uint2 w = codes8(v, __shfl_sync(0xffffffffu, q, i, 16));
                    if (item < items) {
                        const int off = kb * BN * kFp8Block + r * 128 + (((l >> 1) ^ (r & 7)) << 4) + (l & 1) * 8;
                        *reinterpret_cast<uint2 *>(smem_raw + at.q + off) = w;
                        if (l == 8 + i) scales_s[kb * BN + r] = q;
                    }
                }
            }
            fence_proxy_async_smem();
            asm volatile("bar.sync 1, 256;" ::: "memory");             // the scales are read by all epilogue warps
            if (lane == 0) mbar_arrive(q_bar);
        } else if constexpr (kSwap) {
            int pt, qt;
            tile_at(first_tile, pt, qt);
            for (int i = et; i < (kb1 - kb0) * BN; i += 256) {
                const int kb = i / BN, m = qt * BN + i % BN;
                scales_s[i] = m < p.rows ? p.a_scales[m * p.scale_row + (kb0 + kb) * p.scale_block] : 0.0f;
            }
            asm volatile("bar.sync 1, 256;" ::: "memory");
        }
        uint32_t buf = 0, bphase = 0;
        for (int tile = first_tile; tile < tiles; tile += stride) {
            int pt, qt;
            tile_at(tile, pt, qt);
            const int p_row0 = pt * 128 + quarter * 32;            // this warp's rows of operand P; a thread has one
            const int q_col = qt * BN + half * kCols;                  // its first row of operand Q
            const float *a_scales = kSwap ? nullptr : p.a_scales + static_cast<int64_t>(min(p_row0 + lane, p.rows - 1)) * p.scale_row;
            const int w_block = (kSwap ? pt : q_col / kFp8Block);
            // beyond the last output there is no scale; the sums there are not stored
            const float *w_scales = p.w_scales + static_cast<int64_t>(min(w_block, (p.outputs - 1) / kFp8Block)) * p.blocks;
            float acc[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[c] = 0.0f;
            bool got = true;
            // Scales on their way: the next k-block's of the weights, the next three's of the activations, which come from L2.
            float sw = __ldg(w_scales + kb0), sa[3];
#pragma unroll
            for (int i = 0; i < 3; ++i) sa[i] = !kSwap && kb0 + i < kb1 ? a_scales[(kb0 + i) * p.scale_block] : 0.0f;
            for (int kb = kb0; kb < kb1; ++kb) {
                const float factor = kSwap ? sw : sw * sa[0];
                sa[0] = sa[1];
                sa[1] = sa[2];
                if (!kSwap && kb + 3 < kb1) sa[2] = a_scales[(kb + 3) * p.scale_block];
                if (kb + 1 < kb1) sw = __ldg(w_scales + kb + 1);
                const float *col_scales = scales_s + (kb - kb0) * BN + half * kCols;
                if (!mbar_wait_warp(tfull_bar(buf), bphase, abort_flag, p.status)) {
                    got = false;
                    break;
                }
                tc_fence_after_sync();
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += kLd) {
                    uint32_t v[kLd];
                    tmem_ld_cols<kLd>(tmem_row + buf * BN + c0, v);
                    tmem_ld_wait_for(v);
                    if (c0 + kLd == kCols) {                           // all read: the MMAs may have the buffer
                        tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(tempty_bar(buf));
                    }
#pragma unroll
                    for (int c = 0; c < kLd; ++c)
                        acc[c0 + c] = fmaf(kSwap ? factor * col_scales[c0 + c] : factor, __uint_as_float(v[c]), acc[c0 + c]);
                }
                buf ^= 1u;
                if (buf == 0u) bphase ^= 1u;
            }
            if constexpr (kOneTile) {
                // this CTA's part, over the stages: all its loads have landed and all its MMAs are done
                float *part = reinterpret_cast<float *>(smem_raw);
                asm volatile("bar.sync 1, 256;" ::: "memory");         // every warp has seen the last MMA's end (or gave up)
                if (!got) break;
                if constexpr (kSwap) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c) part[(half * kCols + c) * (128 + 4) + quarter * 32 + lane] = acc[c];
                } else {
                    float4 *row = reinterpret_cast<float4 *>(part + (quarter * 32 + lane) * (BN + 4) + half * kCols);
#pragma unroll
                    for (int c = 0; c < kCols; c += 4) row[c / 4] = make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]);
                }
            } else {
                if (!got) break;
                // through this warp's staging, 128 bytes of each of its 32 rows at a time, so that whole sectors are written
                constexpr int kStep = 128 / sizeof(Y), kUnit = 16 / sizeof(Y);
                uint8_t *stage = smem_raw + at.staging + (warp - 4) * kFp8Staging;
                Y *y = static_cast<Y *>(p.y);
                const int row0 = p_row0;
                if (p.bias) {
#pragma unroll
                    for (int c = 0; c < kCols; ++c) acc[c] += __ldg(p.bias + min(q_col + c, p.outputs - 1));
                }
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += kStep) {
                    if (q_col + c0 >= p.outputs || row0 >= p.rows) continue;               // the same for the whole warp
                    __syncwarp();
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        uint4 out;
                        if constexpr (sizeof(Y) == 4) {
                            const float *f = acc + c0 + 4 * u;
                            out = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                        } else {
                            const float *f = acc + c0 + 8 * u;
                            out = make_uint4(pack2<Y>(f[0], f[1]), pack2<Y>(f[2], f[3]), pack2<Y>(f[4], f[5]), pack2<Y>(f[6], f[7]));
                        }
                        *reinterpret_cast<uint4 *>(stage + lane * 128 + ((u ^ (lane & 7)) << 4)) = out;
                    }
                    __syncwarp();
                    if (p.whole) {
                        const int u = lane & 7, n = q_col + c0 + u * kUnit;
#pragma unroll
                        for (int r0 = 0; r0 < 32; r0 += 4) {
                            const int r = r0 + (lane >> 3);
                            if (row0 + r >= p.rows) continue;
                            const uint4 v = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((u ^ (r & 7)) << 4));
                            Y *to = y + static_cast<int64_t>(row0 + r) * p.y_pitch + n;
                            if (n + kUnit <= p.outputs) {
                                *reinterpret_cast<uint4 *>(to) = v;
                            } else {
                                for (int i = 0; i < kUnit && n + i < p.outputs; ++i) to[i] = reinterpret_cast<const Y *>(&v)[i];
                            }
                        }
                    } else {                                           // row by row, neighbouring lanes neighbouring columns
                        for (int r = 0; r < 32 && row0 + r < p.rows; ++r) {
#pragma unroll
                            for (int c = lane; c < kStep; c += 32) {
                                const int n = q_col + c0 + c;
                                if (n < p.outputs)
                                    y[static_cast<int64_t>(row0 + r) * p.y_pitch + n] =
                                        reinterpret_cast<const Y *>(stage + r * 128 + (((c / kUnit) ^ (r & 7)) << 4))[c % kUnit];
                            }
                        }
                    }
                }
            }
        }
    }

    if constexpr (kOneTile) {
        // A part that gave up leaves what lies there: its error is in the status word, and nobody waits for it in vain.
        if (p.split > 1)
            cluster_sync_all();
        else
            __syncthreads();
        int pt, qt;
        tile_at(first_tile, pt, qt);
        constexpr int kMajor = kSwap ? BN : 128, kMinor = kSwap ? 128 : BN, kPitch = kMinor + 4;
        const int major0 = kMajor * rank / p.split, major1 = kMajor * (rank + 1) / p.split;
        const int m0 = kSwap ? qt * BN : pt * 128, n0 = kSwap ? pt * 128 : qt * BN;
        Y *y = static_cast<Y *>(p.y);
        // four columns at a time, or one where rows of y begin anywhere
        const auto sum = [&](auto wide) {
            constexpr int kWide = decltype(wide)::value;
            for (int i = major0 * (kMinor / kWide) + static_cast<int>(threadIdx.x); i < major1 * (kMinor / kWide); i += kFp8Threads) {
                const int r = i / (kMinor / kWide), c = i % (kMinor / kWide) * kWide, m = m0 + r, n = n0 + c;
                if (m >= p.rows) break;
                if (n >= p.outputs) continue;
                float v[kWide] = {};
                const uint32_t from = base + 4u * static_cast<uint32_t>(r * kPitch + c);
                if (p.split > 1) {
                    float part[8][kWide];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
#pragma unroll
                        for (int j = 0; j < kWide; ++j) part[q][j] = 0.0f;
                        if (q < p.split) ld_cluster(from, q, part[q]);
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q)
#pragma unroll
                        for (int j = 0; j < kWide; ++j) v[j] += part[q][j];
                } else {
#pragma unroll
                    for (int j = 0; j < kWide; ++j) v[j] = reinterpret_cast<const float *>(smem_raw + (from - base))[j];
                }
                if (p.bias) {
#pragma unroll
                    for (int j = 0; j < kWide; ++j) v[j] += __ldg(p.bias + min(n + j, p.outputs - 1));
                }
                Y *to = y + static_cast<int64_t>(m) * p.y_pitch + n;
                if constexpr (kWide == 4) {
                    if (n + 4 <= p.outputs) {
                        if constexpr (sizeof(Y) == 4)
                            *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
                        else
                            *reinterpret_cast<uint2 *>(to) = make_uint2(pack2<Y>(v[0], v[1]), pack2<Y>(v[2], v[3]));
                        continue;
                    }
                }
#pragma unroll
                for (int j = 0; j < kWide; ++j)
                    if (n + j < p.outputs) to[j] = from_f32<Y>(v[j]);
            }
        };
        if (p.whole)
            sum(std::integral_constant<int, 4>());
        else
            sum(std::integral_constant<int, 1>());
        if (p.split > 1) cluster_sync_all();               // nobody leaves while its part is read
    }
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, kTmem);
    }
}

}  // namespace ptq
