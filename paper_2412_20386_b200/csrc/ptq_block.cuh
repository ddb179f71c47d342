// Element types of the operators between a block's linears (gated scan, block norm, short convolution): rows of binary16,
// bfloat16 or binary32 values with any pitch, read and written in pieces of up to 16 bytes where the pointers allow it.
// All arithmetic is binary32; a value is rounded to its type once, when it is stored.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>
#include <type_traits>

namespace ptq {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T>
__device__ __forceinline__ float to_f32(T v)
{
    if constexpr (sizeof(T) == 4)
        return v;
    else if constexpr (std::is_same_v<T, __half>)
        return __half2float(v);
    else
        return __bfloat162float(v);
}
template <typename T>
__device__ __forceinline__ T from_f32(float v)
{
    if constexpr (sizeof(T) == 4)
        return v;
    else if constexpr (std::is_same_v<T, __half>)
        return __float2half_rn(v);
    else
        return __float2bfloat16_rn(v);
}

// kE consecutive elements as they lie in memory.
template <typename T, int kE>
struct alignas(kE * sizeof(T) >= 16 ? 16 : kE * sizeof(T)) Piece {
    T v[kE];
    __device__ __forceinline__ float operator[](int e) const { return to_f32<T>(v[e]); }
};

// `n` of the kE elements exist.  `whole`: the address allows accesses of up to 16 bytes.  Plain loads: some kernels replace what they
// have read (a state), which loads through the read-only path must not see.
template <typename T, int kE>
__device__ __forceinline__ Piece<T, kE> load_piece(const T *p, int n, bool whole)
{
    Piece<T, kE> r;
    if (whole && n >= kE) {
        constexpr int kWords = kE * static_cast<int>(sizeof(T)) / 4;
        if constexpr (kWords >= 4) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) reinterpret_cast<uint4 *>(&r)[i] = reinterpret_cast<const uint4 *>(p)[i];
        } else if constexpr (kWords == 2) {
            *reinterpret_cast<uint2 *>(&r) = *reinterpret_cast<const uint2 *>(p);
        } else {
            *reinterpret_cast<uint32_t *>(&r) = *reinterpret_cast<const uint32_t *>(p);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kE; ++e) r.v[e] = e < n ? p[e] : from_f32<T>(0.0f);
    }
    return r;
}
template <typename T, int kE>
__device__ __forceinline__ void store_piece(T *p, const float (&f)[kE], int n, bool whole)
{
    Piece<T, kE> r;
#pragma unroll
    for (int e = 0; e < kE; ++e) r.v[e] = from_f32<T>(f[e]);
    if (whole && n >= kE) {
        constexpr int kWords = kE * static_cast<int>(sizeof(T)) / 4;
        if constexpr (kWords >= 4) {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) reinterpret_cast<uint4 *>(p)[i] = reinterpret_cast<const uint4 *>(&r)[i];
        } else if constexpr (kWords == 2) {
            *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(&r);
        } else {
            *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(&r);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kE; ++e)
            if (e < n) p[e] = r.v[e];
    }
}

// kN consecutive floats, of which n exist (16-byte accesses where `whole`).
template <int kN>
__device__ __forceinline__ void load_floats(float (&f)[kN], const float *p, int n, bool whole)
{
    if (kN == 4 && whole && n >= 4) {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        f[0] = v.x;
        f[1 % kN] = v.y;
        f[2 % kN] = v.z;
        f[3 % kN] = v.w;
    } else {
#pragma unroll
        for (int k = 0; k < kN; ++k) f[k] = k < n ? p[k] : 0.0f;
    }
}
template <int kN>
__device__ __forceinline__ void store_floats(float *p, const float (&f)[kN], int n, bool whole)
{
    if (kN == 4 && whole && n >= 4) {
        *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1 % kN], f[2 % kN], f[3 % kN]);
    } else {
#pragma unroll
        for (int k = 0; k < kN; ++k)
            if (k < n) p[k] = f[k];
    }
}

// 1 / (1 + e^-x): 0 and 1 where e^-x over- or underflows.
__device__ __forceinline__ float sigmoid_f32(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }

__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Sums over the lanes whose numbers differ in the bits kLow, 2 kLow, ..., kHigh of V values per lane: every level that
// still has two values or more sends one half and keeps the other, so that V values over P lanes take about V (1 - 1/P)
// shuffles instead of V log2 P.  Returns how many values are left per lane; they are those from index_of on.
template <int kV, int kLow, int kHigh>
__device__ __forceinline__ void lane_sums(float (&v)[kV], int lane)
{
    if constexpr (kLow <= kHigh) {
        if constexpr (kV >= 2) {
            const bool up = lane & kLow;
            float half[kV / 2];
#pragma unroll
            for (int i = 0; i < kV / 2; ++i) {
                const float keep = up ? v[i + kV / 2] : v[i];
                const float send = up ? v[i] : v[i + kV / 2];
                half[i] = keep + __shfl_xor_sync(0xffffffffu, send, kLow);
            }
            lane_sums<kV / 2, kLow * 2, kHigh>(half, lane);
#pragma unroll
            for (int i = 0; i < kV / 2; ++i) v[i] = half[i];
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], kLow);
            lane_sums<1, kLow * 2, kHigh>(v, lane);
        }
    }
}
// Which of the V values the first one left in a lane is.
template <int kV, int kLow, int kHigh>
__device__ __forceinline__ int first_sum(int lane)
{
    if constexpr (kLow <= kHigh && kV >= 2)
        return ((lane & kLow) ? kV / 2 : 0) + first_sum<kV / 2, kLow * 2, kHigh>(lane);
    else
        return 0;
}

}  // namespace ptq
