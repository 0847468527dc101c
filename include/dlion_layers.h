/*
 * dlion_layers.h -- C ABI of the layer operators that make the gradients the optimizer step of
 * dlion.h consumes: a product with bias, activation and residual in its epilogue, its gradient,
 * activation checkpoints in 8 bits, and the loss over a large vocabulary with its gradient.
 *
 *   forward   z = x W + b ;  y = act(z) + r                     dlion_linear_forward
 *   backward  of y = act(u) W + b, u the saved input:           dlion_linear_backward
 *             du = (dy W^T) * act'(u) + r ;  dW = act(u)^T dy ;  db = sum over rows of dy
 *   8 bits    blocks of 32 values of a row share a power of two dlion_checkpoint8, dlion_restore8
 *   loss      L_t = log sum_v exp(x_t . w_v) - x_t . w_{y_t}    dlion_lm_loss
 *             d_tv = g (softmax_tv - [v = y_t]) ;  dx = d W ;  dW = d^T x
 *
 * Conventions:
 *   - operands of a product are bf16; products are summed in binary32 on the tensor cores; what
 *     follows a sum (bias, activation, residual, softmax statistics) is binary32, and an output
 *     is rounded once, when it is stored (bf16: nearest, ties to even);
 *   - the tensor cores drop what their accumulator does not hold: a binary32 result is off by about 1e-6 of the
 *     products' sizes; one rounded to bf16, and the loss's dw, may come out low by up to 2^-28 of itself a product
 *     (k products of one sign, k up to 131072; from there on as a binary32 result);
 *   - act(u) is rounded to bf16 as an operand of dW (the forward product read the same values), and
 *     so is softmax_tv - [v = y_t] as an operand of dx and dW (g multiplies their sums); between the two the
 *     logits are held as 16-bit distances below a group's largest, 3.4e-4 relative in exp at most, exact where
 *     the distance is 0, and softmax below 5e-20 of its group's largest counts as 0.  The losses do not
 *     go through the codes.  dx is bf16;
 *   - gelu is the tanh form z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))); silu is z/(1 + exp(-z));
 *   - NaN and infinities go through as the formulas say; relu(NaN) = NaN.  In the loss, words may be masked by -infinity or by
 *     any finite value; a row with a logit that is NaN or +infinity, or with none above -infinity, has a loss and gradients
 *     of NaN.
 *
 * Every buffer is DEVICE memory owned by the caller.  A matrix is a pointer and two strides in
 * ELEMENTS; strides are non-negative, rows and columns at most 2^30 (2^24 - 256 columns of u and of the
 * 8-bit form).  Where a parameter has one stride ("ld", between rows) its columns are adjacent.  x, w, dy
 * take any strides: an operand that the copy engine cannot read in place (neither stride 1, a base or the
 * other stride off the 16-byte grid) is packed into the workspace first.  m = 0 (no rows) is allowed: sums over
 * no rows are zero.  Inputs and outputs must not overlap, except that residual may equal y or dx.
 *
 * Calls are asynchronous on the given stream, never synchronise, allocate nothing and keep no state:
 * the workspace (16-byte aligned, of at least the queried size, its contents arbitrary) is in use
 * until the stream has passed the call.  Results do not depend on what the workspace held and are
 * the same from call to call.  Nothing here throws, aborts or traps.  Calls may come from any
 * thread; a device must be current.  No CPU fallback exists.
 */
#ifndef DLION_LAYERS_H_
#define DLION_LAYERS_H_

#include "dlion.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { DLION_ACT_NONE = 0, DLION_ACT_RELU = 1, DLION_ACT_GELU = 2, DLION_ACT_SILU = 3 } dlion_act;
typedef enum { DLION_KEEP_NONE = 0, DLION_KEEP_BF16 = 1, DLION_KEEP_8BIT = 2 } dlion_keep;

#define DLION_BLOCK8 32 /* values of a row that share an exponent in the 8-bit form */

/* A matrix in the 8-bit form: q[row * q_ld + col] is an int8, e[(col / 32) * e_ld + row] a byte, and
 * the value is q * 2^(e - 127), exact in bf16.  2^(e-127) is the smallest power of two, 2^-126 at
 * least and 2^121 at most, with max|v| <= 127 * 2^(e-127) over the block; q is v / 2^(e-127) to the
 * nearest integer, ties to even, and 127 or -127 for what lies beyond (above 127 * 2^121, where a larger
 * power would restore the type's largest value as infinity).  e = 255 marks a block that held a NaN or an
 * infinity: its values are NaN. */

typedef struct {
    int64_t m, k, n;                       /* rows (tokens), inputs, outputs; k, n >= 1 */
    const void* x; int64_t x_rs, x_cs;     /* bf16 [m][k] */
    const void* w; int64_t w_rs, w_cs;     /* bf16 [k][n] */
    const void* bias; int32_t bias_type;   /* nullable [n]; dlion_gdtype */
    int32_t act;                           /* dlion_act */
    const void* residual; int64_t r_ld;    /* nullable, bf16 [m][n] */
    void* y; int64_t y_ld; int32_t y_type; /* [m][n]; dlion_gdtype */
    int32_t keep;                          /* what is kept of z: dlion_keep */
    void* kept; int64_t kept_ld;           /* bf16 or int8 [m][n] */
    uint8_t* kept_e; int64_t kept_e_ld;    /* 8 bits only: [ceil(n/32)][m] */
} dlion_linear_fwd;

typedef struct {
    int64_t m, k, n;
    const void* dy; int64_t dy_rs, dy_cs;  /* bf16 [m][n] */
    const void* w; int64_t w_rs, w_cs;     /* bf16 [k][n]; needed for dx only */
    int32_t act;                           /* dlion_act applied to u before the product */
    int32_t saved;                         /* DLION_KEEP_BF16 or DLION_KEEP_8BIT */
    const void* u; int64_t u_ld;           /* bf16 or int8 [m][k] */
    const uint8_t* u_e; int64_t u_e_ld;    /* 8 bits only: [ceil(k/32)][m] */
    const void* residual; int64_t r_ld;    /* nullable, bf16 [m][k]: added to dx */
    void* dx; int64_t dx_ld;               /* nullable, bf16 [m][k] */
    void* dw; int64_t dw_rs, dw_cs;        /* nullable [k][n], one stride 1; dlion_gdtype grad_type.  dx and dw have the
                                              same bits alone as together if grad_type and these strides are the same;
                                              db may be added in another order */
    void* db;                              /* nullable [n]; grad_type */
    int32_t grad_type;                     /* dlion_gdtype, that of the optimizer's gradient arena */
} dlion_linear_bwd;

typedef struct {
    int64_t m, h, v;                       /* rows (tokens), width, words; h, v >= 1 */
    const void* x; int64_t x_rs, x_cs;     /* bf16 [m][h] */
    const void* w; int64_t w_rs, w_cs;     /* bf16 [v][h] */
    const int64_t* targets;                /* [m]; a target outside [0, v) that is not ignore_index makes
                                              its row's loss, and so the loss, and its gradients NaN */
    int64_t ignore_index;                  /* such a row has loss and gradients 0 (its x is multiplied by 0 for dw,
                                              not left out: NaN there stays NaN) */
    int32_t mean;                          /* 1: g = scale / (rows with a target); 0: g = scale */
    float scale;                           /* factor of the gradients only (loss scaling) */
    float* loss;                           /* [1]: sum or mean of the rows' losses; 0 when no row has a target */
    float* rows;                           /* [m]: each row's loss, 0 where the target is ignored */
    void* dx; int64_t dx_ld;               /* nullable together with dw: bf16 [m][h] */
    void* dw; int64_t dw_ld;               /* [v][h]; grad_type */
    int32_t grad_type;                     /* dlion_gdtype */
    int64_t piece;                         /* rows whose logits are held at a time, as 16-bit codes; 0: 4096;
                                              rounded up to a multiple of 8 where x_cs is not 1.  Without
                                              gradients no logits are held, and 32768 rows at least are one */
} dlion_loss;

/* Bytes of workspace that the call needs (0 also for arguments that the call refuses). */
uint64_t dlion_linear_forward_workspace(const dlion_linear_fwd* p);
uint64_t dlion_linear_backward_workspace(const dlion_linear_bwd* p);
uint64_t dlion_lm_loss_workspace(const dlion_loss* p);

/* DLION_EINVAL: a null pointer that is needed, a size or an enumerator out of range, a workspace too
 * small; DLION_EALIGN: a pointer off its element's size, a workspace off 16 bytes; DLION_ECUDA: the
 * runtime or the driver refused a launch. */
dlion_status dlion_linear_forward(const dlion_linear_fwd* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream);
dlion_status dlion_linear_backward(const dlion_linear_bwd* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream);
dlion_status dlion_lm_loss(const dlion_loss* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream);

/* x (bf16 [m][k]) into the 8-bit form, and back. */
dlion_status dlion_checkpoint8(const void* x, int64_t x_ld, int64_t m, int64_t k, int8_t* q, int64_t q_ld,
                               uint8_t* e, int64_t e_ld, void* cuda_stream);
dlion_status dlion_restore8(const int8_t* q, int64_t q_ld, const uint8_t* e, int64_t e_ld, int64_t m, int64_t k,
                            void* x, int64_t x_ld, void* cuda_stream);

/* Every wait inside the kernels ends after a time limit; a kernel whose wait ran out ends, its outputs
 * undefined, and leaves a mark on the device.  Synchronises the stream and returns DLION_OK, DLION_ESTATE
 * if a mark was left since the last call (and clears it), or DLION_ECUDA. */
dlion_status dlion_layers_check(void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* DLION_LAYERS_H_ */
