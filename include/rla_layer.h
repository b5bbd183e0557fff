/*
 * rla_layer.h -- C ABI of the operators around a sequence-mixing layer (the
 * same library as rla.h): the short causal convolution of its projections, a
 * selective state-space scan (a mixer with one decay per channel and state),
 * the residual addition with the norm before a block, and the gated norm after
 * one.
 *
 * Conventions shared by every entry point are those of rla.h: device memory
 * owned by the caller, nothing allocated or kept between calls, asynchronous
 * on `stream`, argument errors returned as an rla_status before any HIP call,
 * no call aborts or throws.  Beyond them:
 *   Tokens.  A token's row holds `channels` values next to each other.  Dense
 *     tokens are [B, T], n = b; packed tokens (cu_seqlens != NULL, B = 1) are
 *     T tokens in N sequences, read on the device as rla.h says: disjoint,
 *     possibly empty sequences, whatever the offsets hold.  Tokens outside every
 *     sequence are not read (beyond being loaded) and get zero outputs and
 *     gradients; an empty sequence's final state is its initial one.
 *   Strides.  Where a problem has a *_stride field, the rows of that input
 *     are that many elements apart (0: next to each other): slices of a wider
 *     projection are read in place.  Every other array is contiguous.
 *   Alignment.  Arrays need the alignment of their elements only; workspaces
 *     256 bytes.
 *   Types.  Activations are fp32 or bf16 (`dtype`), outputs and activation
 *     gradients of the same type (rounded once, to nearest); parameters,
 *     their gradients and the scan's states fp32.  All sums, states and
 *     statistics are held in fp32.
 *   Aliasing.  Outputs overlap neither inputs nor each other, except where an
 *     entry point says so.
 *   Determinism.  Equal calls give equal bits: sums run in an order fixed by
 *     the sizes, and no atomics add values.
 */
#ifndef RLA_MI355X_RLA_LAYER_H
#define RLA_MI355X_RLA_LAYER_H

#include "rla.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------
 * Short causal convolution, depthwise:
 *   pre_t = bias + sum_{i < taps} weight[:, i] * x_{t - taps + 1 + i}
 *   y_t   = pre_t, or pre_t sigmoid(pre_t) with `silu`
 * x before a sequence's start is its initial state, zero without one.  A
 * state holds a sequence's last taps - 1 inputs, oldest first, in x's type
 * (exact copies).
 * Sizes: calls of more than a launch can hold (some 2^38 values, 2^34 of single
 * tokens) are RLA_ERR_SHAPE.
 * ------------------------------------------------------------------------ */
typedef struct {
  int64_t batch, seq_len;    /* B, T (packed: 1, all tokens) */
  int64_t channels;          /* D >= 1 */
  int64_t num_seqs;          /* N with cu_seqlens, else ignored */
  const int32_t *cu_seqlens; /* device, N + 1 offsets, or NULL */
  int64_t x_stride;          /* elements between rows of x (0: D) */
  int64_t dy_stride;         /* ... and of dy */
  int32_t taps;              /* 2, 3 or 4 */
  int32_t silu;              /* 0 or 1 */
  int32_t dtype;             /* rla_dtype of x, y, dy, dx and the states */
} rla_conv_problem;

/* Bytes of workspace: packed sequences need it in every call, the backward
 * always (`backward` 0 or 1).  0 for an invalid problem too. */
size_t rla_conv_workspace_size(const rla_conv_problem *problem, int backward);

/* weight [D, taps], bias [D] or NULL, state_init [N, taps-1, D] or NULL
 * (zeros), state_final [N, taps-1, D] or NULL (not written). */
rla_status rla_conv_forward(const rla_conv_problem *problem, const void *x,
                            const float *weight, const float *bias, const void *state_init,
                            void *y, void *state_final,
                            void *workspace, size_t workspace_bytes, void *stream);

/* Gradients of <dy, y> + <dstate_final, state_final> (dstate_final NULL:
 * zeros).  dx [tokens, D], dweight [D, taps], dbias [D] or NULL (not written),
 * dstate_init [N, taps-1, D] or NULL (not written). */
rla_status rla_conv_backward(const rla_conv_problem *problem, const void *x,
                             const float *weight, const float *bias, const void *state_init,
                             const void *dy, const void *dstate_final,
                             void *dx, float *dweight, float *dbias, void *dstate_init,
                             void *workspace, size_t workspace_bytes, void *stream);

/* T new tokens (a few) of B sequences onto their states: state_out may be
 * state_in (in place).  state_in NULL: zeros.  No workspace; dense only
 * (RLA_ERR_UNSUPPORTED with cu_seqlens). */
rla_status rla_conv_decode(const rla_conv_problem *problem, const void *x,
                           const float *weight, const float *bias, const void *state_in,
                           void *y, void *state_out, void *stream);

/* ------------------------------------------------------------------------
 * Selective state-space scan, one decay per channel c and state n:
 *   s_t   = delta_t + delta_bias, through softplus with `softplus`
 *   h_t   = exp(s_t A) h_{t-1} + s_t u_t B_t         h [D, N]
 *   o_t   = (sum_n C_t h_t + skip u_t) z_t sigmoid(z_t)
 * B and C are shared by the channels of a group: channel c reads group
 * c / (D / groups).  skip (NULL: none), z (NULL: no gate), delta_bias (NULL:
 * none) are optional.  A is used as given (negative in a model that decays).
 * Decays below 2^-126 are zero.  Sizes: channels come in blocks (64 of up to 16
 * states, 32 of up to 32, 16 of more; a group's last one in part), and a forward or
 * backward takes fewer than 2^24 (block, sequence) pairs, rla_ssm_decode some
 * 2^25; more are RLA_ERR_SHAPE.
 * ------------------------------------------------------------------------ */
typedef struct {
  int64_t batch, seq_len;
  int64_t channels;          /* D < 2^24, a multiple of groups */
  int64_t states;            /* N_state, 1 to 64 */
  int64_t groups;            /* G >= 1 */
  int64_t num_seqs;
  const int32_t *cu_seqlens;
  int64_t u_stride, delta_stride, z_stride, do_stride;   /* 0: D; all < 2^24 */
  int64_t b_stride, c_stride;                             /* 0: G * N_state */
  int32_t softplus;          /* 0 or 1 */
  int32_t dtype;             /* rla_dtype of u, delta, B, C, z, o and their gradients */
} rla_ssm_problem;

typedef enum {
  RLA_SSM_FORWARD = 0,
  RLA_SSM_BACKWARD = 1       /* also a forward that saves for it */
} rla_ssm_op;

size_t rla_ssm_workspace_size(const rla_ssm_problem *problem, int op);

/* u, delta, z, o [tokens, D]; A [D, N_state]; B, C [tokens, G, N_state]; h_init,
 * h_final [N, D, N_state] fp32, both may be NULL (zeros / not written).  `save`:
 * the workspace, of RLA_SSM_BACKWARD's size, keeps what a backward with
 * use_saved reads instead of recomputing it. */
rla_status rla_ssm_forward(const rla_ssm_problem *problem, const void *u, const void *delta,
                           const float *A, const void *B, const void *C, const float *skip,
                           const void *z, const float *delta_bias, const float *h_init,
                           void *o, float *h_final, int save,
                           void *workspace, size_t workspace_bytes, void *stream);

/* Gradients of <dO, o> + <dh_final, h_final> (dh_final NULL: zeros).  dskip, dz,
 * ddelta_bias are written where skip, z, delta_bias are given (and required
 * then); dh_init may be NULL.  use_saved: the workspace is that of the last
 * forward with `save`, for the same problem and inputs. */
rla_status rla_ssm_backward(const rla_ssm_problem *problem, const void *u, const void *delta,
                            const float *A, const void *B, const void *C, const float *skip,
                            const void *z, const float *delta_bias, const float *h_init,
                            const void *dO, const float *dh_final,
                            void *du, void *ddelta, float *dA, void *dB, void *dC,
                            float *dskip, void *dz, float *ddelta_bias, float *dh_init,
                            int use_saved, void *workspace, size_t workspace_bytes, void *stream);

/* T new tokens (a few) of B sequences: h_out [B, D, N_state], which may be h_in
 * (in place; h_in NULL: zeros).  No workspace; dense only. */
rla_status rla_ssm_decode(const rla_ssm_problem *problem, const void *u, const void *delta,
                          const float *A, const void *B, const void *C, const float *skip,
                          const void *z, const float *delta_bias, const float *h_in,
                          void *o, float *h_out, void *stream);

/* ------------------------------------------------------------------------
 * Norms.  RMS(y) = y / sqrt(mean(y^2) + eps) over a row of `width` values.
 * ------------------------------------------------------------------------ */

/* Before a block: the residual stream takes the previous block's output, and
 * the next block's input is its norm:
 *   residual_out = residual + scale * x;   n = RMS(residual_out) * weight
 * residual NULL: 0; scale [width] NULL: 1.  n is of x's type; the norm is of the
 * sum before it is rounded to the stream's type. */
typedef struct {
  int64_t rows, width;
  int64_t x_stride;          /* elements between rows of x (0: width) */
  int64_t dn_stride;         /* ... and of dn */
  int32_t dtype;             /* rla_dtype of x, n, dn, dx */
  int32_t residual_dtype;    /* rla_dtype of the stream and its gradients */
  float eps;                 /* >= 0 */
} rla_addnorm_problem;

size_t rla_addnorm_workspace_size(const rla_addnorm_problem *problem);   /* the backward's */

/* residual_out may be residual (in place). */
rla_status rla_addnorm_forward(const rla_addnorm_problem *problem, const void *x,
                               const void *residual, const float *weight, const float *scale,
                               void *n, void *residual_out, void *stream);

/* Gradients of <dn, n> + <dresidual_out, residual_out> (dresidual_out NULL:
 * zeros) from the stream that the forward left: dx, dresidual (NULL: not
 * written), dweight [width], dscale [width] (written where scale is given; then
 * x is needed).  dresidual may be dresidual_out. */
rla_status rla_addnorm_backward(const rla_addnorm_problem *problem, const void *dn,
                                const void *dresidual_out, const void *residual_out,
                                const void *x, const float *weight, const float *scale,
                                void *dx, void *dresidual, float *dweight, float *dscale,
                                void *workspace, size_t workspace_bytes, void *stream);

/* After a block, per head: with y = x, or x silu(g) if gate_first,
 *   o = RMS(y) weight silu(g), or RMS(y) weight if gate_first.
 * weight [width], or [heads, width] with weight_per_head. */
typedef struct {
  int64_t tokens, heads, width;
  int64_t x_stride, gate_stride, do_stride;   /* elements between tokens (0: heads * width) */
  int32_t dtype;             /* rla_dtype of the gate, o, dO, dgate */
  int32_t x_dtype;           /* rla_dtype of x, dx: `dtype`, or fp32 */
  int32_t gate_first, weight_per_head;        /* 0 or 1 */
  float eps;
} rla_gatenorm_problem;

size_t rla_gatenorm_workspace_size(const rla_gatenorm_problem *problem);   /* the backward's */

rla_status rla_gatenorm_forward(const rla_gatenorm_problem *problem, const void *x,
                                const void *gate, const float *weight, void *o, void *stream);

/* dx [tokens, heads, width] in x_dtype, dgate in dtype, dweight like weight. */
rla_status rla_gatenorm_backward(const rla_gatenorm_problem *problem, const void *dO,
                                 const void *x, const void *gate, const float *weight,
                                 void *dx, void *dgate, float *dweight,
                                 void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* RLA_MI355X_RLA_LAYER_H */
