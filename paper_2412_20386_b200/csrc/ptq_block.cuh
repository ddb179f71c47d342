// Element types of the operators between a block's linears (gated scan, block norm, short convolution): rows of binary16,
// bfloat16 or binary32 values with any pitch, read and written in pieces of up to 16 bytes where the pointers allow it.
// All arithmetic is binary32; a value is rounded to its type once, when it is stored.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>
#include <type_traits>

#include "ptx_griddep.cuh"

namespace ptq {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

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

// kE consecutive elements as they lie in memory, in whole registers: held as 16-bit values, they would be taken apart, and
// waited for, where they are loaded.
template <typename T, int kE>
struct Piece {
    static constexpr int kWords = (kE * static_cast<int>(sizeof(T)) + 3) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(w[e]);
        } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
        } else {
            const __half2 h = *reinterpret_cast<const __half2 *>(&w[e / 2]);
            return e & 1 ? __high2float(h) : __low2float(h);
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ void set(const float (&f)[kE])
    {
        zero();
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            if constexpr (sizeof(T) == 4) {
                w[e] = __float_as_uint(f[e]);
            } else if constexpr (kE % 2 == 0) {
                if (e & 1) continue;
                if constexpr (std::is_same_v<T, __half>) {
                    const __half2 h = __floats2half2_rn(f[e], f[(e + 1) % kE]);
                    w[e / 2] = *reinterpret_cast<const uint32_t *>(&h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(f[e], f[(e + 1) % kE]);
                    w[e / 2] = *reinterpret_cast<const uint32_t *>(&h);
                }
            } else {
                const T t = from_f32<T>(f[e]);
                w[e / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(&t)) << 16 * (e & 1);
            }
        }
    }
};

template <typename T, int kE>
__device__ __forceinline__ void floats_of(float (&f)[kE], const Piece<T, kE> &r)
{
#pragma unroll
    for (int e = 0; e < kE; ++e) f[e] = r[e];
}

// Words of the accesses that move a piece, and how many elements one of them holds.
template <typename T, int kE>
constexpr int kAccessWords = kE * sizeof(T) >= 16 ? 4 : kE * sizeof(T) >= 8 ? 2 : 1;

// `n` of the kE elements exist, the others are zeros.  kWhole: the pointer allows accesses of up to 16 bytes, and n ends between two of
// them; otherwise of `unit` elements (4, 2 or 1), of which 16-bit types make use.  Plain loads: some kernels replace what they have read (a state), which loads through the read-only path must not see.
template <bool kWhole, typename T, int kE>
__device__ __forceinline__ Piece<T, kE> load_piece(const T *p, int n, int unit = 1)
{
    Piece<T, kE> r;
    r.zero();
    if constexpr (kWhole && kE * sizeof(T) >= 4) {
        constexpr int kStep = kAccessWords<T, kE>, kElems = kStep * 4 / static_cast<int>(sizeof(T));
#pragma unroll
        for (int i = 0; i < Piece<T, kE>::kWords / kStep; ++i) {
            if (n < (i + 1) * kElems) continue;
            if constexpr (kStep == 4) {
                const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
                r.w[4 * i] = v.x;
                r.w[4 * i + 1] = v.y;
                r.w[4 * i + 2] = v.z;
                r.w[4 * i + 3] = v.w;
            } else if constexpr (kStep == 2) {
                const uint2 v = reinterpret_cast<const uint2 *>(p)[i];
                r.w[2 * i] = v.x;
                r.w[2 * i + 1] = v.y;
            } else {
                r.w[i] = reinterpret_cast<const uint32_t *>(p)[i];
            }
        }
    } else {
        if constexpr (sizeof(T) == 2 && kE % 4 == 0) {
            if (unit >= 4) {
#pragma unroll
                for (int i = 0; i < kE / 4; ++i) {
                    if (n < 4 * i + 4) continue;
                    const uint2 v = reinterpret_cast<const uint2 *>(p)[i];
                    r.w[2 * i] = v.x;
                    r.w[2 * i + 1] = v.y;
                }
                return r;
            }
        }
        if constexpr (sizeof(T) == 2 && kE % 2 == 0) {
            if (unit >= 2) {
#pragma unroll
                for (int i = 0; i < kE / 2; ++i)
                    if (n >= 2 * i + 2) r.w[i] = reinterpret_cast<const uint32_t *>(p)[i];
                return r;
            }
        }
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            if (e >= n) continue;
            if constexpr (sizeof(T) == 4)
                r.w[e] = reinterpret_cast<const uint32_t *>(p)[e];
            else
                r.w[e / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[e]) << 16 * (e & 1);
        }
    }
    return r;
}
template <bool kWhole, typename T, int kE>
__device__ __forceinline__ void store_piece(T *p, const Piece<T, kE> &r, int n, int unit = 1)
{
    if constexpr (kWhole && kE * sizeof(T) >= 4) {
        constexpr int kStep = kAccessWords<T, kE>, kElems = kStep * 4 / static_cast<int>(sizeof(T));
#pragma unroll
        for (int i = 0; i < Piece<T, kE>::kWords / kStep; ++i) {
            if (n < (i + 1) * kElems) continue;
            if constexpr (kStep == 4)
                reinterpret_cast<uint4 *>(p)[i] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
            else if constexpr (kStep == 2)
                reinterpret_cast<uint2 *>(p)[i] = make_uint2(r.w[2 * i], r.w[2 * i + 1]);
            else
                reinterpret_cast<uint32_t *>(p)[i] = r.w[i];
        }
    } else {
        if constexpr (sizeof(T) == 2 && kE % 4 == 0) {
            if (unit >= 4) {
#pragma unroll
                for (int i = 0; i < kE / 4; ++i)
                    if (n >= 4 * i + 4) reinterpret_cast<uint2 *>(p)[i] = make_uint2(r.w[2 * i], r.w[2 * i + 1]);
                return;
            }
        }
        if constexpr (sizeof(T) == 2 && kE % 2 == 0) {
            if (unit >= 2) {
#pragma unroll
                for (int i = 0; i < kE / 2; ++i)
                    if (n >= 2 * i + 2) reinterpret_cast<uint32_t *>(p)[i] = r.w[i];
                return;
            }
        }
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            if (e >= n) continue;
            if constexpr (sizeof(T) == 4)
                reinterpret_cast<uint32_t *>(p)[e] = r.w[e];
            else
                reinterpret_cast<uint16_t *>(p)[e] = static_cast<uint16_t>(r.w[e / 2] >> 16 * (e & 1));
        }
    }
}
template <bool kWhole, typename T, int kE>
__device__ __forceinline__ void store_piece(T *p, const float (&f)[kE], int n, int unit = 1)
{
    Piece<T, kE> r;
    r.set(f);
    store_piece<kWhole, T, kE>(p, r, n, unit);
}

// Copies kBytes to shared memory without waiting for them; zeros, and nothing is read, unless `on`.
template <int kBytes>
__device__ __forceinline__ void copy_async(uint32_t to, const void *from, bool on)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(kBytes), "r"(on ? kBytes : 0) : "memory");
}

// A piece on its way to shared memory, its 16-byte parts at to[0], to[apart], ... (one thread's of a row of threads, so that no two of them
// meet a bank).  The thread that asked for it may read it after staged().  General rows are copied in units of 8 or 4 bytes; what is
// aligned to 2 bytes only is loaded and stored.
template <bool kWhole, typename T, int kE>
__device__ __forceinline__ void stage_piece(uint4 *to, const T *p, int n, int apart = 32, int unit = 1)
{
    static_assert(kE * sizeof(T) % 16 == 0, "whole parts");
    constexpr int kParts = kE * static_cast<int>(sizeof(T)) / 16, kElems = 16 / static_cast<int>(sizeof(T));
    const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(to));
    if constexpr (kWhole) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int bytes = n >= (i + 1) * kElems ? 16 : 0;      // the rest of the 16 is filled with zeros, nothing is read for none
            if constexpr (kParts == 1)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at + 16 * apart * i), "l"(p + i * kElems), "r"(bytes) : "memory");
            else                                           // half a sector: the other part finds it in the first-level cache
                copy_async<16>(at + 16 * apart * i, p + i * kElems, bytes > 0);
        }
    } else if (sizeof(T) == 4 || unit == 2) {
        constexpr int kStep = 4 / static_cast<int>(sizeof(T));
#pragma unroll
        for (int e = 0; e < kE; e += kStep) copy_async<4>(at + 16 * apart * (e / kElems) + e % kElems * static_cast<int>(sizeof(T)), p + e, n >= e + kStep);
    } else if (unit >= 4) {
        constexpr int kStep = 8 / static_cast<int>(sizeof(T));
#pragma unroll
        for (int e = 0; e < kE; e += kStep) copy_async<8>(at + 16 * apart * (e / kElems) + e % kElems * static_cast<int>(sizeof(T)), p + e, n >= e + kStep);
    } else {
        const Piece<T, kE> r = load_piece<false, T, kE>(p, n);
#pragma unroll
        for (int i = 0; i < kParts; ++i) to[apart * i] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
    }
}
template <typename T, int kE>
__device__ __forceinline__ Piece<T, kE> staged_piece(const uint4 *from, int apart = 32)
{
    Piece<T, kE> r;
#pragma unroll
    for (int i = 0; i < Piece<T, kE>::kWords / 4; ++i) {
        const uint4 v = from[apart * i];
        r.w[4 * i] = v.x;
        r.w[4 * i + 1] = v.y;
        r.w[4 * i + 2] = v.z;
        r.w[4 * i + 3] = v.w;
    }
    return r;
}
__device__ __forceinline__ void staged() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// Copies in groups: staged_but<n>() waits for all groups but the last n.
__device__ __forceinline__ void stage_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kGroups>
__device__ __forceinline__ void staged_but()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(kGroups) : "memory");
}

// kN consecutive floats, of which n exist; kWhole: the address allows accesses of 16 bytes (8, if kN is 2), and n ends between
// two of them.
template <bool kWhole, int kN>
__device__ __forceinline__ void load_floats(float (&f)[kN], const float *p, int n)
{
    if constexpr (kN % 4 == 0 && kWhole) {
#pragma unroll
        for (int k = 0; k < kN; k += 4) {
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (n >= k + 4) v = *reinterpret_cast<const float4 *>(p + k);
            f[k] = v.x;
            f[k + 1] = v.y;
            f[k + 2] = v.z;
            f[k + 3] = v.w;
        }
    } else if constexpr (kN == 2 && kWhole) {
        float2 v = make_float2(0.0f, 0.0f);
        if (n >= 2) v = *reinterpret_cast<const float2 *>(p);
        f[0] = v.x;
        f[1] = v.y;
    } else {
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            f[k] = 0.0f;
            if (k < n) f[k] = p[k];
        }
    }
}
template <bool kWhole, int kN>
__device__ __forceinline__ void store_floats(float *p, const float (&f)[kN], int n)
{
    if constexpr (kN % 4 == 0 && kWhole) {
#pragma unroll
        for (int k = 0; k < kN; k += 4)
            if (n >= k + 4) *reinterpret_cast<float4 *>(p + k) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
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

// Two binary32 operations in one instruction (it occupies the pipe for two cycles and leaves the other issue slot free).
__device__ __forceinline__ void fma_pair(float &d0, float &d1, float a0, float a1, float b0, float b1, float c0, float c1)
{
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void mul_pair(float &d0, float &d1, float a0, float a1, float b0, float b1)
{
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void add_pair(float &d0, float &d1, float a0, float a1, float b0, float b1)
{
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
template <int kN>
__device__ __forceinline__ void add_each(float (&d)[kN], const float (&a)[kN], const float (&b)[kN])
{
    static_assert(kN % 2 == 0, "pairs");
#pragma unroll
    for (int k = 0; k < kN; k += 2) add_pair(d[k], d[k + 1], a[k], a[k + 1], b[k], b[k + 1]);
}
// d[k] = a[k] b[k] + c[k], and with one factor for all k; d may be any of the operands.
template <int kN>
__device__ __forceinline__ void fma_each(float (&d)[kN], const float (&a)[kN], const float (&b)[kN], const float (&c)[kN])
{
    if constexpr (kN == 1) d[0] = fmaf(a[0], b[0], c[0]);
#pragma unroll
    for (int k = 0; k + 1 < kN; k += 2) fma_pair(d[k], d[k + 1], a[k], a[k + 1], b[k], b[k + 1], c[k], c[k + 1]);
}
template <int kN>
__device__ __forceinline__ void fma_each(float (&d)[kN], float a, const float (&b)[kN], const float (&c)[kN])
{
    if constexpr (kN == 1) d[0] = fmaf(a, b[0], c[0]);
#pragma unroll
    for (int k = 0; k + 1 < kN; k += 2) fma_pair(d[k], d[k + 1], a, a, b[k], b[k + 1], c[k], c[k + 1]);
}
template <int kN>
__device__ __forceinline__ void mul_each(float (&d)[kN], const float (&a)[kN], const float (&b)[kN])
{
    if constexpr (kN == 1) d[0] = a[0] * b[0];
#pragma unroll
    for (int k = 0; k + 1 < kN; k += 2) mul_pair(d[k], d[k + 1], a[k], a[k + 1], b[k], b[k + 1]);
}
template <int kN>
__device__ __forceinline__ void mul_each(float (&d)[kN], float a, const float (&b)[kN])
{
    if constexpr (kN == 1) d[0] = a * b[0];
#pragma unroll
    for (int k = 0; k + 1 < kN; k += 2) mul_pair(d[k], d[k + 1], a, a, b[k], b[k + 1]);
}

// sum_k a[k] b[k]
template <int kN>
__device__ __forceinline__ float dot_each(const float (&a)[kN], const float (&b)[kN])
{
    if constexpr (kN == 1) return a[0] * b[0];
    float s[2];
    mul_pair(s[0], s[1], a[0], a[1 % kN], b[0], b[1 % kN]);
#pragma unroll
    for (int k = 2; k + 1 < kN; k += 2) fma_pair(s[0], s[1], a[k], a[k + 1], b[k], b[k + 1], s[0], s[1]);
    return s[0] + s[1];
}

// Sums over the lanes whose numbers differ in the bits kLow, 2 kLow, ..., kHigh of V values per lane: every level that
// still has two values or more sends one half and keeps the other, so that V values over P lanes take about V (1 - 1/P)
// shuffles instead of V log2 P.  V / P values, or one, are left in a lane, at the front of v: those from first_sum on.
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

// Column sums of the partial results of other CTAs, in the order of the rows: the sum of part[r * pitch] for r < rows.  Called by all of
// a CTA of kWarps warps, one column per lane (`on`: it has one), every kWarps-th row per warp; the result is the first warp's.
template <int kWarps>
__device__ __forceinline__ float sum_rows(const float *part, long long rows, long long pitch, bool on, float (&s)[kWarps][33])
{
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    float v = 0.0f;
    if (on) {
#pragma unroll 8
        for (long long r = y; r < rows; r += kWarps) v += part[r * pitch];
    }
    s[y][x] = v;
    __syncthreads();
    v = 0.0f;
    if (y == 0) {
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += s[i][x];
    }
    return v;
}

}  // namespace ptq
