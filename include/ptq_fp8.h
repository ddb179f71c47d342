/*
 * ptq_fp8.h -- C ABI of linears in 8-bit floating point (e4m3) with a scale for each block of 128 (B200, sm_100a), in the library
 * of ptq_linear.h and under its conventions: status codes, thread-local error text, the caller's stream, nothing allocated,
 * nothing synchronised, no exception, abort or trap.
 *
 * Activations [rows, cols] share a scale among 128 neighbouring values of a row, weights [outputs, cols] among 128 x 128;
 * the last blocks may be smaller.  Scales are found from the data of the call, nothing is calibrated:
 *     top   = max(2^-100, max over the block |x|)
 *     scale = top / 448,  code = e4m3(x (448 / top))          (binary32, each quotient rounded once; ties to even codes)
 *     y[m,n] = sum_b a_scale[m,b] w_scale[n / 128, b] sum_{k in block b} a[m,k] w[n,k]  (+ bias[n])
 * The products of a block of 128 are summed on the tensor cores in binary32, the blocks in binary32 in their order (where a
 * sum is split over several CTAs: parts in their order); the same call gives the same bits.  A block that holds an
 * infinity or NaN makes the row of the result NaN (of weights: its 128 columns).  The two scales are multiplied first: beyond binary32's range that
 * makes infinities and NaN, below its normal values it is inexact or zero.
 *
 * Codes lie in rows on 16-byte boundaries: base and pitch are multiples of 16.  What lies between cols and the pitch is not read.
 */
#ifndef PTQ_FP8_H_
#define PTQ_FP8_H_

#include "ptq_block.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PTQ_FP8_BLOCK       128
#define PTQ_FP8_MAX_ROWS    (1 << 30)
#define PTQ_FP8_MAX_COLS    65536
#define PTQ_FP8_MAX_OUTPUTS (1 << 20)

/* Activations of a call, before they are quantized. */
typedef struct {
    int dtype;                        /* ptq_dtype_t of x */
    int cols;
    int64_t rows;
    const void *x;                    /* device, [rows, cols] */
    int64_t x_pitch;                  /* elements between rows, not negative */
} ptq_fp8_input_t;

/* codes device [rows, cols], codes_pitch bytes between rows; scales device: that of block b of row m at
 * scales[m * scales_pitch[0] + b * scales_pitch[1]], each in a place of its own.  Outputs overlap no input. */
ptq_status_t ptq_fp8_quantize(const ptq_fp8_input_t *in, void *codes, int64_t codes_pitch, float *scales, const int64_t scales_pitch[2],
                              void *stream);
/* The same for weights (rows: outputs, at most PTQ_FP8_MAX_OUTPUTS); scales dense [ceil(rows/128), ceil(cols/128)]. */
ptq_status_t ptq_fp8_quantize_weight(const ptq_fp8_input_t *in, void *codes, int64_t codes_pitch, float *scales, void *stream);

typedef struct {
    int cols, outputs;
    const void *codes;                /* device, [outputs, cols] */
    int64_t codes_pitch;              /* bytes between rows */
    const float *scales;              /* device, dense [ceil(outputs/128), ceil(cols/128)] */
    const float *bias;                /* device, [outputs], or NULL */
} ptq_fp8_weight_t;

/* y device [rows, outputs] of type y_dtype, y_pitch elements between rows; overlaps no input. */
ptq_status_t ptq_fp8_matmul(const ptq_fp8_weight_t *w, int64_t rows, const void *a, int64_t a_pitch, const float *a_scales,
                            const int64_t a_scales_pitch[2], void *y, int y_dtype, int64_t y_pitch, void *stream);

/* Both: quantizes the input and multiplies; y has the input's type.  workspace device, 16-byte aligned, at least
 * ptq_fp8_linear_workspace_bytes(rows, cols, outputs) bytes (0 for few rows: then it may be NULL).  Gives the bits that the
 * two calls give where the sums are cut alike: with up to 16 rows they may be cut otherwise. */
size_t ptq_fp8_linear_workspace_bytes(int64_t rows, int cols, int outputs);
ptq_status_t ptq_fp8_linear(const ptq_fp8_weight_t *w, const ptq_fp8_input_t *in, void *y, int64_t y_pitch, void *workspace,
                            size_t workspace_bytes, void *stream);

/* Whether a kernel of this header gave up a bounded wait on the current device since the last call of this function, whose
 * output is then undefined: PTQ_OK or PTQ_ERR_TIMEOUT.  Synchronises the device; not for captured streams. */
ptq_status_t ptq_fp8_device_status(void);

#ifdef __cplusplus
}
#endif
#endif /* PTQ_FP8_H_ */
