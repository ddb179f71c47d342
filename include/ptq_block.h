/*
 * ptq_block.h -- C ABI of the operators between the quantized linears of a Mamba block (B200, sm_100a), in the
 * library of ptq_linear.h and under its conventions: status codes, thread-local error text, the caller's stream,
 * nothing allocated, nothing synchronised, no exception, abort or trap.
 *
 *   ptq_norm_*   norm in front of in_proj (with residual and scale) or behind the scan (with its gate)
 *   ptq_conv_*   short causal depthwise convolution behind in_proj
 *   ptq_scan_*   gated linear recurrence between dt_proj and out_proj
 *
 * Activations are token-major, [batch, token, channel], of one type per call, with the channels of a token next to
 * each other and any pitch between tokens and between sequences (in elements, not negative): the halves of in_proj's
 * output and the columns of x_proj's are passed as they lie.  Pointers are aligned to their type; rows whose
 * pointers and pitches are multiples of 16 bytes are moved 16 bytes at a time.  The pitches of an input that is NULL
 * are ignored.  Parameters, states of the recurrence and gradients of parameters are binary32.  Arithmetic is binary32
 * throughout; a result is rounded to its type once.  Outputs are dense unless their pitch is an argument, and overlap no input but
 * where a function says so.  Sums have a fixed order: the same call gives the same bits.
 *
 * Sequences are processed from the first token to the last or, with PTQ_SEQ_REVERSE, from the last to the first.
 * `lengths` (device, [batch] int32, or NULL) gives the number of tokens of each sequence of a padded batch; values are
 * clamped to 0 .. length.  What lies behind a sequence's end is not read; outputs there are left as they are, gradients are
 * set to zero.
 *
 * An infinity or NaN in a token reaches what the formulas make of it and, in the backward passes, all gradients of the parameters
 * of its channel (in B or C: of the group's channels).
 */
#ifndef PTQ_BLOCK_H_
#define PTQ_BLOCK_H_

#include "ptq_linear.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PTQ_F16 = 0, PTQ_BF16 = 1, PTQ_F32 = 2 } ptq_dtype_t;

#define PTQ_SEQ_REVERSE     2u   /* scan, conv: process from the last token to the first */
#define PTQ_SCAN_SOFTPLUS   1u   /* dt = log(1 + e^(delta + delta_bias)); without: dt = delta + delta_bias */
#define PTQ_CONV_SILU       1u   /* y = pre / (1 + e^-pre); without: y = pre */
#define PTQ_NORM_LAYER      1u   /* subtract the mean (layer norm); without: root mean square only */
#define PTQ_NORM_GATE_OUT   2u   /* the gate multiplies the norm's result; without: its input */

#define PTQ_MAX_LENGTH      (1 << 30)
#define PTQ_MAX_CHANNELS    65536
#define PTQ_MAX_STATES      32
#define PTQ_MAX_NORM_COLS   8192
#define PTQ_SCAN_HISTORY    8    /* steps between two states that the backward pass starts from */

/*
 * Gated linear recurrence.  For step i of a sequence (token p), channel d of group g = d / (channels / groups), state n:
 *     e = delta[p,d] + delta_bias[d];  dt = log(1 + exp(e)), or e
 *     h[d,n] <- exp(dt A[d,n]) h[d,n] + dt u[p,d] B[p,g,n]
 *     o[p,d] = sum_n h[d,n] C[p,g,n] + D[d] u[p,d];   y[p,d] = o[p,d] z[p,d] / (1 + exp(-z[p,d])), or o[p,d]
 * The decay is the exact solution over a step, the input's factor the first-order dt B, as Mamba blocks are trained (not the
 * (exp(dt A) - 1) / A B of an input that is held over the step).  A is negative in a trained model; any finite value is computed, and -inf
 * (no memory where dt > 1e-36; a step with dt = 0 keeps the state with any A).
 */
typedef struct {
    int dtype;                        /* ptq_dtype_t of u, delta, z, B, C, y and their gradients */
    int batch, length, channels, states, groups;
    unsigned flags;                   /* PTQ_SCAN_SOFTPLUS, PTQ_SEQ_REVERSE */
    const void *u, *delta;            /* device, [batch, length, channels] */
    const void *z;                    /* device, the gate, like u, or NULL */
    const void *B, *C;                /* device, [batch, length, groups, states] */
    int64_t u_pitch[2], delta_pitch[2], z_pitch[2];       /* between sequences, between tokens */
    int64_t B_pitch[3], C_pitch[3];                       /* between sequences, tokens, groups */
    const float *A;                   /* device, [channels, states] */
    const float *D, *delta_bias;      /* device, [channels], each or NULL */
    const float *state;               /* device, [batch, channels, states]: h in front of the first step, or NULL (zeros) */
    const int32_t *lengths;           /* device, [batch], or NULL */
} ptq_scan_t;

/*
 * Forward pass.
 *   y            device, [batch, length, channels]
 *   final_state  device, [batch, channels, states]: h behind the last step, or NULL; may be `state` itself
 *   history      device, [batch, ceil(length / PTQ_SCAN_HISTORY), channels, states], or NULL: the state in front of every
 *                8th step, for ptq_scan_backward; entries behind a sequence's end are left as they are
 *   workspace    device, 16-byte aligned, at least ptq_scan_workspace_bytes(s, 0) bytes (may be 0: then it may be NULL)
 * Length 1 (a token of a generating model) takes a kernel of its own.
 */
size_t ptq_scan_workspace_bytes(const ptq_scan_t *s, int backward);      /* 0 too where a dimension is out of range */
ptq_status_t ptq_scan_forward(const ptq_scan_t *s, void *y, float *final_state, float *history, void *workspace,
                              size_t workspace_bytes, void *stream);

/* Gradients with respect to everything that the forward pass read.  dB and dC are dense and hold one value for every
 * token, whatever the pitches of B and C.  The pointers marked * may be NULL (not wanted, or the input was not given). */
typedef struct {
    void *du, *ddelta, *dz;           /* [batch, length, channels]; dz NULL exactly where z is */
    void *dB, *dC;                    /* [batch, length, groups, states] */
    float *dA;                        /* [channels, states] */
    float *dD, *ddelta_bias;          /* [channels]  * */
    float *dstate;                    /* [batch, channels, states]  * */
} ptq_scan_grads_t;

/*
 * Backward pass.
 *   s         as for the forward pass (state: the one it started from, unchanged)
 *   history   as the forward pass wrote it
 *   dy        device, [batch, length, channels], dense
 *   dfinal    device, [batch, channels, states], gradient of final_state, or NULL (zeros)
 *   workspace device, 16-byte aligned, at least ptq_scan_workspace_bytes(s, 1) bytes
 */
ptq_status_t ptq_scan_backward(const ptq_scan_t *s, const float *history, const void *dy, const float *dfinal,
                               const ptq_scan_grads_t *grads, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Norm with residual, scale and gate.  Per row:
 *     v = x silu(gate), or x;   r = residual + scale v;   n = (r - mean(r)) / sqrt(var(r) + eps), or r / sqrt(mean(r^2) + eps)
 *     y = n weight + bias, times silu(gate) with PTQ_NORM_GATE_OUT
 * The norm is taken of r before it is rounded to residual_out's type.
 */
typedef struct {
    int dtype;                        /* ptq_dtype_t of x, gate, y and their gradients */
    int residual_dtype;               /* of residual, residual_out and their gradients: dtype or PTQ_F32 */
    int64_t rows;
    int cols;
    unsigned flags;                   /* PTQ_NORM_LAYER, PTQ_NORM_GATE_OUT */
    float eps;                        /* >= 0 */
    const void *x, *residual, *gate;  /* device, [rows, cols]; the last two each or NULL */
    int64_t x_pitch, residual_pitch, gate_pitch;
    const float *weight, *bias, *scale;       /* device, [cols], each or NULL (1, 0, 1) */
} ptq_norm_t;

/* y device [rows, cols]; residual_out device [rows, cols] or NULL: r; may be `residual` itself where that is dense. */
ptq_status_t ptq_norm_forward(const ptq_norm_t *n, void *y, void *residual_out, void *stream);

typedef struct {
    void *dx;                         /* [rows, cols] */
    void *dgate;                      /* [rows, cols]; NULL exactly where gate is */
    void *dresidual;                  /* [rows, cols]  * */
    float *dweight, *dbias, *dscale;  /* [cols]  *; of an input that is NULL: the gradient at 1, 0 and 1 */
} ptq_norm_grads_t;

/* n as for the forward pass (residual unchanged); dy, dresidual_out device, dense [rows, cols], the latter or NULL (zeros);
 * workspace device, 16-byte aligned, ptq_norm_workspace_bytes(n) bytes. */
size_t ptq_norm_workspace_bytes(const ptq_norm_t *n);
ptq_status_t ptq_norm_backward(const ptq_norm_t *n, const void *dy, const void *dresidual_out, const ptq_norm_grads_t *grads,
                               void *workspace, size_t workspace_bytes, void *stream);

/*
 * Short causal depthwise convolution of `taps` (2 .. 4) taps.  For step i of a sequence:
 *     pre[i,d] = bias[d] + sum_j weight[d,j] x[i - (taps-1) + j, d],   y = pre / (1 + exp(-pre)), or pre
 * The taps - 1 steps in front of the first one are the rows of `state`.
 */
typedef struct {
    int dtype;                        /* ptq_dtype_t of x, state, y and their gradients */
    int batch, length, channels, taps;
    unsigned flags;                   /* PTQ_CONV_SILU, PTQ_SEQ_REVERSE */
    const void *x;                    /* device, [batch, length, channels] */
    int64_t x_pitch[2];               /* between sequences, between tokens */
    const float *weight;              /* device, [channels, taps] */
    const float *bias;                /* device, [channels], or NULL */
    const void *state;                /* device, [batch, taps-1, channels] in the order of the steps, or NULL (zeros) */
    const int32_t *lengths;           /* device, [batch], or NULL */
} ptq_conv_t;

/* y device [batch, length, channels]; final_state device [batch, taps-1, channels] or NULL: the last taps-1 rows, for the
 * next piece of the sequences or their next token; may be `state` itself. */
ptq_status_t ptq_conv_forward(const ptq_conv_t *c, void *y, void *final_state, void *stream);

typedef struct {
    void *dx;                         /* [batch, length, channels] */
    void *dstate;                     /* [batch, taps-1, channels]  * */
    float *dweight;                   /* [channels, taps] */
    float *dbias;                     /* [channels]  * */
} ptq_conv_grads_t;

/* c as for the forward pass (state unchanged); dy device, dense; dfinal device, [batch, taps-1, channels], or NULL (zeros);
 * workspace device, 16-byte aligned, ptq_conv_workspace_bytes(c) bytes. */
size_t ptq_conv_workspace_bytes(const ptq_conv_t *c);
ptq_status_t ptq_conv_backward(const ptq_conv_t *c, const void *dy, const void *dfinal, const ptq_conv_grads_t *grads, void *workspace,
                               size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PTQ_BLOCK_H_ */
