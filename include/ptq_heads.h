/*
 * ptq_heads.h -- C ABI of linear attention with a decay for each head (B200, sm_100a), the recurrence of blocks whose state is a
 * matrix per head, in the library of ptq_linear.h and under its conventions: status codes, thread-local error text, the caller's
 * stream, nothing allocated, nothing synchronised, no exception, abort or trap.
 *
 * Activations are token-major, [batch, token, head, column], of one type per call, with the columns of a head (of a group) next
 * to each other and any other pitches (in elements, not negative): the columns of a projection's output are passed as they lie.
 * Pointers are aligned to their type; rows whose pointers and pitches are multiples of 16 bytes are moved 16 bytes at a time.
 * Parameters, states and gradients of parameters are binary32.  Outputs are dense and overlap no input but where a function says
 * so.  Sums have a fixed order: the same call gives the same bits.
 *
 * Sequences are processed from the first token to the last or, with PTQ_SEQ_REVERSE, from the last to the first.  `lengths`
 * (device, [batch] int32, or NULL) gives the number of tokens of each sequence of a padded batch; values are clamped to
 * 0 .. length.  What lies behind a sequence's end is not read; outputs there are left as they are, gradients are set to zero.
 */
#ifndef PTQ_HEADS_H_
#define PTQ_HEADS_H_

#include "ptq_block.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PTQ_HEADS_SOFTPLUS   1u   /* dt = log(1 + e^(delta + delta_bias)); without: dt = delta + delta_bias */
                                  /* PTQ_SEQ_REVERSE (2u) as for ptq_scan */
#define PTQ_HEADS_UNSCALED   4u   /* the input is u B^T; without: dt u B^T */

#define PTQ_MAX_HEADS        4096
#define PTQ_MAX_HEAD_COLS    256  /* columns of a head */
#define PTQ_MAX_HEAD_STATES  128  /* states of a column */
#define PTQ_HEADS_HISTORY    64   /* steps between two states that the backward pass starts from */

/*
 * For step i of a sequence (token t), head h of group g = h / (heads / groups), column p, state n:
 *     e = delta[t,h] + delta_bias[h];  dt = log(1 + exp(e)), or e, or 1 where delta is NULL
 *     S[h,p,n] <- exp(dt A[h]) S[h,p,n] + dt u[t,h,p] B[t,g,n]
 *     y[t,h,p] = sum_n S[h,p,n] C[t,g,n] + D[h] u[t,h,p]
 * Decays are at most 1 in a trained model (A <= 0, dt >= 0); growth is computed as long as it, and products of operands times it, stay in
 * binary32's range over 64 steps.  A decay below 2^-126 over up to 64 steps counts as zero.  A may be -inf.
 *
 * Accuracy: steps are taken 64 at a time as matrix products.  16-bit operands enter the tensor cores as they are, sums are
 * binary32; products of two operands and the state are rounded to the activations' type where they become operands themselves
 * for y and the gradients of activations, and split into two or three such values where they go into states and gradients of
 * parameters.  (binary16: the state and products of operands are rounded relative to the largest of 16 columns or steps and scaled
 * by powers of two, so that they neither overflow nor vanish.)  binary32 operands are split in two throughout.
 *
 * An infinity or NaN in a token reaches what the formulas make of it (an infinity perhaps as NaN in the state), in the forward
 * pass no earlier token, in the backward pass all gradients of the 64 steps around it, the earlier ones' and the parameters'.
 */
typedef struct {
    int dtype;                        /* ptq_dtype_t of u, delta, B, C, y and their gradients */
    int batch, length, heads, cols, states, groups;
    unsigned flags;                   /* PTQ_HEADS_SOFTPLUS, PTQ_SEQ_REVERSE, PTQ_HEADS_UNSCALED */
    const void *u;                    /* device, [batch, length, heads, cols] */
    const void *delta;                /* device, [batch, length, heads], or NULL (dt = 1; delta_bias is NULL too) */
    const void *B, *C;                /* device, [batch, length, groups, states] */
    int64_t u_pitch[3], B_pitch[3], C_pitch[3];           /* between sequences, tokens, heads (groups) */
    int64_t delta_pitch[3];                               /* between sequences, tokens, heads */
    const float *A;                   /* device, [heads] */
    const float *D, *delta_bias;      /* device, [heads], each or NULL */
    const float *state;               /* device, [batch, heads, cols, states]: S in front of the first step, or NULL (zeros) */
    const int32_t *lengths;           /* device, [batch], or NULL */
} ptq_heads_t;

/*
 * Forward pass.
 *   y            device, [batch, length, heads, cols]
 *   final_state  device, like state: S behind the last step, or NULL; may be `state` itself
 *   history      device, [batch, ceil(length / PTQ_HEADS_HISTORY), heads, cols, states], or NULL: the state in front of every 64th
 *                step, for ptq_heads_backward; entries behind a sequence's end are left as they are
 *   workspace    device, 16-byte aligned, at least ptq_heads_workspace_bytes(s, 0) bytes (may be 0: then it may be NULL)
 * Length 1 (a token of a generating model) takes a kernel of its own, in binary32 throughout.
 */
size_t ptq_heads_workspace_bytes(const ptq_heads_t *s, int backward);    /* 0 too where a dimension is out of range */
ptq_status_t ptq_heads_forward(const ptq_heads_t *s, void *y, float *final_state, float *history, void *workspace, size_t workspace_bytes,
                               void *stream);

/* The pointers marked * may be NULL (not wanted, or the input was not given). */
typedef struct {
    void *du;                         /* [batch, length, heads, cols] */
    void *ddelta;                     /* [batch, length, heads]; NULL exactly where delta is */
    void *dB, *dC;                    /* [batch, length, groups, states] */
    float *dA;                        /* [heads] */
    float *dD, *ddelta_bias;          /* [heads]  * */
    float *dstate;                    /* [batch, heads, cols, states]  * */
} ptq_heads_grads_t;

/*
 * Backward pass.
 *   s         as for the forward pass (state: the one it started from, unchanged)
 *   history   as the forward pass wrote it
 *   dy        device, [batch, length, heads, cols], dense
 *   dfinal    device, [batch, heads, cols, states], gradient of final_state, or NULL (zeros)
 *   workspace device, 16-byte aligned, at least ptq_heads_workspace_bytes(s, 1) bytes (8 for each token, head and state, for each 64 columns of
 *             a head, and some more)
 */
ptq_status_t ptq_heads_backward(const ptq_heads_t *s, const float *history, const void *dy, const float *dfinal, const ptq_heads_grads_t *grads,
                                void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* PTQ_HEADS_H_ */
