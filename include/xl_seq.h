/*
 * xl sequence operators for AMD MI355X (gfx950 / CDNA4): the layers of a scan block, the mixer
 * behind a convolutional stem whose feature map is read as a sequence of positions.
 *
 * C ABI of libxl_seq.so.  Plain C types only; a stream is passed as `void*` holding a hipStream_t.
 * Statuses are those of xl.h; xl_seq_last_error gives the message of the calling thread's last failure.
 *
 *   xl_causal_conv       depthwise convolution over time, each token and the few before it
 *   xl_selective_scan    state-space recurrence whose step and input/output vectors depend on the token
 *   xl_quantize_blocks   numbers -> 8-bit floating point (e4m3) with one scale for each block of 128
 *   xl_block_matmul      product of two such operands
 *
 * Every call takes one struct of 64-bit numbers and DEVICE pointers, enqueues one kernel (a large
 * product and a scan with a workspace two, sizes that take 2^32 threads and more several) on `stream` and returns without synchronising: it may be recorded into a HIP graph.  The library allocates
 * nothing and keeps nothing between calls.  Calls never throw or abort.  The current HIP device must be a gfx950 (XL_E_DEVICE) that can reach the
 * pointers.  Inference only: there are no gradients.
 *
 * Sequences.  Activations are [batch, length, channels], channels next to each other, the steps between tokens and
 * between sequences free (in elements; a half of a wider tensor needs no copy) but not negative.  Sequences of a batch may have
 * lengths of their own: `lengths` (int32 per sequence, NULL: all are `length` long; values outside [0, length] are taken as the nearer end).  Tokens past a
 * sequence's end are never read, and come out as zeros.
 * States.  A sequence's state is what one call leaves for the next: with it, a prompt may be run in pieces and
 * continued token by token.  `state` may be NULL (a sequence begins: zeros) and `new_state` may be NULL (nobody goes on); they may
 * be the same memory and must not overlap otherwise.  Row `slots[i]` (int32; NULL: row i) of `nslots` rows belongs to sequence i; a row
 * outside [0, nslots) marks a sequence that is absent: its outputs are zeros and no state is touched.  Two sequences of a call
 * must not share a row.
 * A call with an empty batch, no channels, rows or columns does nothing.  With a length of zero the states are carried over.
 */
#ifndef XL_SEQ_H
#define XL_SEQ_H

#include "xl.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { XL_F32 = 0, XL_F16 = 1, XL_BF16 = 2 };

#define XL_SCALE_BLOCK   128    /* numbers along a row that share a scale           */
#define XL_MAX_TAPS      4
#define XL_MAX_STATES    128

/*
 * y[b,t,c] = act(bias[c] + sum over j < taps of weight[c,j] * x[b, t - (taps - 1) + j, c]),  act = v * sigmoid(v) or none.
 * Inputs before the first token are the rows of `state` [nslots, taps - 1, channels], oldest first, of x's type;
 * `new_state` gets the last taps - 1 inputs.  taps is 2 to 4.  Sums are fp32.
 * y must not overlap x.
 */
typedef struct xl_causal_conv_args {
    long long batch, length, channels, taps;
    long long dtype;                        /* XL_F32, XL_F16, XL_BF16: x, y, states    */
    long long silu;
    long long x_batch, x_token;             /* elements between sequences / tokens      */
    long long y_batch, y_token;
    long long nslots;
    const void *x;
    const float *weight;                    /* [channels, taps]                         */
    const float *bias;                      /* [channels] or NULL                       */
    const void *state;
    void *new_state;
    const int *lengths, *slots;
    void *y;
} xl_causal_conv_args;
xl_status xl_causal_conv(const xl_causal_conv_args *args, void *stream);

/*
 * For every sequence and channel c, with states h[n], n < states (1 to 128):
 *   d    = softplus(delta[t,c] + delta_bias[c])           (without `softplus`: the sum itself)
 *   h[n] = exp(d * A[c,n]) * h[n] + d * u[t,c] * B[t,n]
 *   y    = (sum over n of C[t,n] * h[n]  +  D[c] * u[t,c]) * z[t,c] * sigmoid(z[t,c])
 * delta_bias, D and z may be NULL (left out).  u, delta, B, C, z and y are of type `dtype`; A, D, delta_bias and the
 * states [nslots, channels, states] are fp32, and so is all arithmetic.  y may be u's, delta's or z's memory with
 * the same steps, and must not overlap the inputs otherwise.
 * A token's factor exp(d * A) has to be an fp32 number.  States may grow: without `softplus` by as much as fp32 holds; with it, where A is positive, by up to 2^128 within 16
 * tokens (a state of zero stays zero whatever the growth).  What an infinite or NaN input makes of its channel is not finite from its token on; infinity or NaN is not said.
 */
typedef struct xl_scan_args {
    long long batch, length, channels, states;
    long long dtype;
    long long softplus;
    long long u_batch, u_token, delta_batch, delta_token, z_batch, z_token, y_batch, y_token;
    long long b_batch, b_token, c_batch, c_token;
    long long nslots;
    long long workspace_bytes;
    const void *u, *delta;
    const float *A;                         /* [channels, states]                       */
    const void *B, *C;                      /* [batch, length, states]                  */
    const float *D, *delta_bias;            /* [channels] or NULL                       */
    const void *z;
    const float *state;
    float *new_state;
    const int *lengths, *slots;
    void *y;
    void *workspace;
} xl_scan_args;
xl_status xl_selective_scan(const xl_scan_args *args, void *stream);

/* Bytes of device memory (aligned to 16) with which xl_selective_scan is faster for arguments of these sizes: where there are too few channels for the
 * chip a sequence is cut into parts that are worked on at the same time, in two kernels.  0 if there is nothing to gain.  With less, or NULL, the
 * call does without; the results agree up to rounding.  The memory holds nothing between calls. */
long long xl_selective_scan_workspace(const xl_scan_args *args);

/*
 * x [rows, k] -> q [rows, k] in e4m3 and scales: x is about q * scale.  A scale is max(max|x| / 448, 2^-126) over its
 * block of `block_rows` (1: activations, 128: weights) by 128 numbers; q = x / scale rounded to nearest, ties to even.
 * A block with a NaN becomes NaN; with an infinity its scale is infinite, the infinity NaN and the rest zeros.
 * scales[i, j] lies at i * scale_row + j * scale_block.  Rows of q begin at multiples of 16 bytes, and the bytes between a row's end and the
 * next multiple of 16 are set to zero.
 */
typedef struct xl_quantize_args {
    long long rows, k;
    long long block_rows;
    long long dtype;                        /* of x                                     */
    long long x_row;                        /* elements between rows                    */
    long long q_row;                        /* bytes between rows, a multiple of 16     */
    long long scale_row, scale_block;
    const void *x;
    void *q;
    float *scales;
} xl_quantize_args;
xl_status xl_quantize_blocks(const xl_quantize_args *args, void *stream);

/*
 * y[i,j] = bias[j] + sum over k-blocks b of a_scales[i,b] * b_scales[j / 128, b] * (sum over k of block b of a[i,k] * b[j,k])
 * a [m, k] and b [n, k] are e4m3 (b holds a row for each output, as a pointwise filter does), y [m, n] is of type `dtype`.
 * Rows of a and b begin at multiples of 16 bytes and can be read to the next multiple of 16 behind their k numbers; what
 * lies there does not matter.  A scale for each block is applied to the block's sum, and the blocks are summed in fp32.  Inside a block of 128 products sums are fp32 where y is.  Where y has 16
 * bits they are those of the 8-bit matrix operation, which drops, of eight neighbours, what lies more than 13 bits below the largest product: 1e-5 to 7e-5 of the result's norm, less than y's rounding,
 * but more than the last place of a single result in which much cancels.  The product of a scale of a and one of b has to be an fp32 number.  y must not overlap a or b.
 */
typedef struct xl_block_matmul_args {
    long long m, n, k;
    long long dtype;                        /* of y                                     */
    long long a_row, b_row;                 /* bytes between rows                       */
    long long a_scale_row, a_scale_block;   /* a_scales[i, b] lies at i * a_scale_row + b * a_scale_block */
    long long b_scale_row, b_scale_block;   /* b_scales[j / 128, b] likewise            */
    long long y_row;                        /* elements between rows                    */
    const void *a, *b;
    const float *a_scales, *b_scales;
    const float *bias;                      /* [n] or NULL                              */
    void *y;
} xl_block_matmul_args;
xl_status xl_block_matmul(const xl_block_matmul_args *args, void *stream);

const char *xl_seq_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* XL_SEQ_H */
