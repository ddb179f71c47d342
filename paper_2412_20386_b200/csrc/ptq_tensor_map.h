// Tensor maps of the TMA loads and stores.
#pragma once

#include <cuda.h>

#include <mutex>

#include "ptq_host.h"

namespace ptq_host {

// cuTensorMapEncodeTiled is reached through the runtime's driver entry point query, so the
// library has no link-time dependency on libcuda and loads on machines without a driver.
typedef CUresult (*encode_tiled_fn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                    const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                    CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                    CUtensorMapFloatOOBfill);

inline encode_tiled_fn get_encode_tiled()
{
    static encode_tiled_fn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<encode_tiled_fn>(p);
    });
    return fn;
}

// 2-D row-major tensor [rows, cols] with `pitch_bytes` between rows; box [box_rows, box_cols];
// the swizzle mode follows the box's row bytes (128 or 64, which box_cols * elem_bytes must equal);
// out-of-range elements read as zero and are skipped on stores.
inline ptq_status_t make_map_2d(CUtensorMap *map, CUtensorMapDataType dt, int elem_bytes, const void *ptr,
                         unsigned long long cols, unsigned long long rows, unsigned long long pitch_bytes,
                         unsigned box_cols, unsigned box_rows)
{
    encode_tiled_fn enc = get_encode_tiled();
    if (!enc) return fail(PTQ_ERR_CUDA, "cuTensorMapEncodeTiled entry point not available");
    const unsigned row_bytes = box_cols * elem_bytes;
    if ((row_bytes != 128 && row_bytes != 64) || box_rows == 0 || box_rows > 256)
        return fail(PTQ_ERR_SHAPE, "internal: bad TMA box %u x %u", box_rows, box_cols);
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {pitch_bytes};
    cuuint32_t box[2] = {box_cols, box_rows};
    cuuint32_t estr[2] = {1, 1};
    CUresult r = enc(map, dt, 2, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     row_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS)
        return fail(PTQ_ERR_CUDA, "cuTensorMapEncodeTiled failed with CUresult %d (cols %llu rows %llu pitch %llu)",
                    static_cast<int>(r), cols, rows, pitch_bytes);
    return PTQ_OK;
}

}  // namespace ptq_host
