// What the host files of the operators of include/ptq_block.h, ptq_heads.h and ptq_fp8.h share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <initializer_list>
#include <type_traits>

#include "../../include/ptq_block.h"
#include "ptq_host.h"

namespace ptq_host {

constexpr int kSms = 148;             // of the one GPU that the library is for; only cuts of the work go by it
constexpr long long kMaxGrid = 0x7fffffffll;

#define PTQ_TRY(...)                                  \
    do {                                              \
        const ptq_status_t st_ = (__VA_ARGS__);       \
        if (st_ != PTQ_OK) return st_;                \
    } while (0)

inline ptq_status_t launched()
{
    g_launches.fetch_add(1, std::memory_order_relaxed);
    PTQ_CUDA(cudaGetLastError());
    return PTQ_OK;
}

// Launch of a call's second or third kernel: it may begin while the one before it drains, and waits for its end (griddep_wait) before it
// touches memory.  The first kernel of a call is launched the ordinary way.
template <typename... KArgs, typename... Args>
ptq_status_t launch_next(void (*kern)(KArgs...), dim3 grid, int threads, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    PTQ_CUDA(cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...));
    return launched();
}

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Calls fn with the flag as a constant.
template <class Fn>
ptq_status_t with_flag(bool flag, Fn fn)
{
    return flag ? fn(std::true_type()) : fn(std::false_type());
}

inline ptq_status_t check_arch()
{
    constexpr int kMaxDevices = 64;
    static std::atomic<int> known[kMaxDevices] = {};      // 0: not asked yet, 1: sm_100, 2: another one
    int dev = -1;
    PTQ_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= kMaxDevices) return fail(PTQ_ERR_CUDA, "device index %d out of range", dev);
    int k = known[dev].load(std::memory_order_relaxed);
    if (k == 0) {
        int major = 0, minor = 0;
        PTQ_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
        PTQ_CUDA(cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev));
        k = major == 10 && minor == 0 ? 1 : 2;
        known[dev].store(k, std::memory_order_relaxed);
    }
    return k == 1 ? PTQ_OK : fail(PTQ_ERR_ARCH, "device %d is not compute capability 10.0", dev);
}

inline int elem_bytes(int dtype) { return dtype == PTQ_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == PTQ_F16 || dtype == PTQ_BF16 || dtype == PTQ_F32; }

// Every pointer that is given on a multiple of `bytes`.
inline bool aligned(std::initializer_list<const void *> ps, int bytes)
{
    for (const void *p : ps)
        if (reinterpret_cast<uintptr_t>(p) % bytes) return false;
    return true;
}
inline bool multiples(std::initializer_list<int64_t> pitches, int unit)
{
    for (int64_t v : pitches)
        if (v % unit) return false;
    return true;
}
inline bool not_negative(std::initializer_list<int64_t> pitches)
{
    for (int64_t v : pitches)
        if (v < 0) return false;
    return true;
}
inline size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

template <class Fn>
ptq_status_t with_type(int dtype, Fn fn)
{
    if (dtype == PTQ_F16) return fn(__half());
    if (dtype == PTQ_BF16) return fn(__nv_bfloat16());
    return fn(0.0f);
}

inline ptq_status_t check_space(const void *workspace, size_t have, size_t need)
{
    if (need == 0) return PTQ_OK;
    if (!workspace) return fail(PTQ_ERR_NULL, "workspace is NULL");
    if (!aligned({workspace}, 16)) return fail(PTQ_ERR_ALIGN, "workspace is not 16-byte aligned");
    if (have < need) return fail(PTQ_ERR_SHAPE, "workspace has %zu bytes, %zu are needed", have, need);
    return PTQ_OK;
}

}  // namespace ptq_host
