/*
 * rla_model.h -- C ABI of the operators at the ends of a language model on
 * these mixing layers (the same library as rla.h), and of a second recurrent
 * mixer: the lookup of tokens in an embedding table, the gated linear
 * recurrence (one state per channel, the decay from a gate of its own), and the
 * log probabilities of given tokens with the rows' entropy and likeliest
 * alternatives; each with its gradients.
 *
 * Conventions shared by every entry point are those of rla.h and rla_layer.h:
 * device memory owned by the caller, nothing allocated or kept between calls,
 * asynchronous on `stream`, argument errors returned as an rla_status before any
 * HIP call, no call aborts or throws; token rows contiguous, *_stride elements
 * apart (0: next to each other), every other array contiguous; arrays aligned to
 * their elements, workspaces to 256 bytes (the size for a problem is enough for one
 * of fewer tokens or rows, sequences and alternatives, everything else equal); activations fp32 or bf16, rounded
 * once; sums, states and statistics in fp32; outputs overlap neither inputs nor
 * each other, except where an entry point says so; equal calls give equal
 * bits (atomics count tokens, none adds values).
 */
#ifndef RLA_MI355X_RLA_MODEL_H
#define RLA_MI355X_RLA_MODEL_H

#include "rla.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of token ids. */
typedef enum {
  RLA_INDEX_I32 = 0,
  RLA_INDEX_I64 = 1
} rla_index;

/* ------------------------------------------------------------------------
 * Embedding: out_t = scale * table[ids_t].  An id outside [0, vocab) stands for
 * no token: a row of zeros, and no part in the gradient.
 * ------------------------------------------------------------------------ */
typedef struct {
  int64_t tokens;            /* n */
  int64_t vocab;             /* V >= 1 rows of the table; < 2^31 (gradients: < 2^22) */
  int64_t width;             /* D >= 1 values a row; <= 2^20 */
  int64_t dout_stride;       /* elements between rows of dout (0: D) */
  int32_t index;             /* rla_index of ids */
  int32_t dtype;             /* rla_dtype of out, dout */
  int32_t table_dtype;       /* rla_dtype of the table (the gradient is fp32) */
  float scale;               /* finite */
} rla_embed_problem;

size_t rla_embed_workspace_size(const rla_embed_problem *problem);   /* the backward's */

/* ids [n], table [V, D], out [n, D]. */
rla_status rla_embed_forward(const rla_embed_problem *problem, const void *ids, const void *table,
                             void *out, void *stream);

/* dtable [V, D] = base + the table's gradient of <dout, out>: row v gets scale
 * times the sum, in the order of t, of dout_t where ids_t = v.  base NULL: 0.  base
 * may be dtable (in place): then rows that no token points at are not
 * touched. */
rla_status rla_embed_backward(const rla_embed_problem *problem, const void *ids, const void *dout,
                              const float *base, float *dtable,
                              void *workspace, size_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------
 * Log probabilities.  With z = scale * logits, a row of `vocab` values:
 *   lse      = log sum_j e^z_j
 *   logprob  = z_y - lse for the row's token y; 0 for y outside [0, vocab)
 *              (a row that is left out)
 *   entropy  = lse - sum_j p_j z_j,  p_j = e^(z_j - lse)
 *   top      the `top` largest logits, equal ones by their place, as log
 *            probabilities and ids; -inf and -1 where fewer have a probability
 * -inf is a logit without a probability.  A row of nothing else has lse = -inf,
 * entropy 0, log probability -inf and a gradient of zeros.  Where scale times finite
 * logits leaves fp32, lse alone is infinite: everything else is taken from the
 * logits' differences.  NaN or +inf in a row gives that row NaN
 * (lse, log probability, entropy and those of its alternatives; which ids they
 * have is then not said).
 * ------------------------------------------------------------------------ */
typedef struct {
  int64_t rows;              /* n */
  int64_t vocab;             /* V >= 1; <= 2^30 */
  int64_t logits_stride;     /* elements between rows of the logits (0: V) */
  int32_t index;             /* rla_index of the tokens */
  int32_t dtype;             /* rla_dtype of logits, dlogits */
  int32_t top;               /* alternatives a row, 0 to 64, <= V */
  float scale;               /* inverse temperature: > 0, scale log2 e finite */
} rla_logprob_problem;

/* Bytes of the forward's workspace (0: none is needed, or an invalid problem). */
size_t rla_logprob_workspace_size(const rla_logprob_problem *problem);

/* logits [n, V], targets [n]; logprob, lse, entropy [n]; top_logprobs fp32,
 * top_ids int32 [n, top].  logprob (and targets), lse, entropy may be NULL: not
 * written. */
rla_status rla_logprob_forward(const rla_logprob_problem *problem, const void *logits,
                               const void *targets, float *logprob, float *lse, float *entropy,
                               float *top_logprobs, int32_t *top_ids,
                               void *workspace, size_t workspace_bytes, void *stream);

/* dlogits [n, V]: gradients of <dlogprob, logprob> + <dentropy, entropy> from the
 * lse and entropy that the forward wrote (fp32: what rounding lse costs p is made
 * good from the row, where it has more than 20480 logits if |lse| > 32):
 *   scale * (dlogprob (1[j = y] - p_j) - dentropy p_j (z_j - lse + entropy))
 * with a row's first part 0 where it is left out.  dlogprob (then targets) and
 * dentropy (then entropy) may be NULL: zeros.  dlogits may be logits (in place,
 * rows next to each other).  No workspace. */
rla_status rla_logprob_backward(const rla_logprob_problem *problem, const void *logits,
                                const void *targets, const float *lse, const float *entropy,
                                const float *dlogprob, const float *dentropy, void *dlogits,
                                void *stream);

/* ------------------------------------------------------------------------
 * Gated linear recurrence, one state a channel:
 *   a_t = exp(A sigmoid(r_t))                               A [D] as used: <= 0
 *   b_t = m_t sigmoid(i_t) x_t,   m_t = sqrt(1 - a_t^2) with `normalize`, else 1
 *   h_t = a_t h_{t-1} + b_t
 *   o_t = h_t, or h_t z_t sigmoid(z_t)
 * i (NULL: the factor 1) and z (NULL: no gate) are optional.  Where a_t = 1 the
 * gradient of m_t counts as 0.  Dense, packed and empty sequences as in
 * rla_layer.h.
 * ------------------------------------------------------------------------ */
typedef struct {
  int64_t batch, seq_len;    /* B, T (packed: 1, all tokens) */
  int64_t channels;          /* D, 1 to 2^23 - 1 */
  int64_t num_seqs;          /* N with cu_seqlens, else ignored */
  const int32_t *cu_seqlens; /* device, N + 1 offsets, or NULL */
  int64_t x_stride, r_stride, i_stride, z_stride, do_stride;   /* 0: D; all < 2^23 */
  int32_t normalize;         /* 0 or 1 */
  int32_t dtype;             /* rla_dtype of x, r, i, z, o and their gradients */
} rla_glr_problem;

typedef enum {
  RLA_GLR_FORWARD = 0,
  RLA_GLR_BACKWARD = 1       /* also a forward that saves for it */
} rla_glr_op;

size_t rla_glr_workspace_size(const rla_glr_problem *problem, int op);

/* x, r, i, z, o [tokens, D]; A [D]; h_init, h_final [N, D] fp32, both may be NULL
 * (zeros / not written).  `save`: the workspace, of RLA_GLR_BACKWARD's size, keeps
 * what a backward with use_saved reads instead of recomputing it. */
rla_status rla_glr_forward(const rla_glr_problem *problem, const void *x, const void *r,
                           const float *A, const void *i, const void *z, const float *h_init,
                           void *o, float *h_final, int save,
                           void *workspace, size_t workspace_bytes, void *stream);

/* Gradients of <dO, o> + <dh_final, h_final> (dh_final NULL: zeros).  di and dz are
 * written where i and z are given (and required then); dh_init may be NULL.
 * use_saved: the workspace is that of the last forward with `save`, for the same
 * problem and inputs. */
rla_status rla_glr_backward(const rla_glr_problem *problem, const void *x, const void *r,
                            const float *A, const void *i, const void *z, const float *h_init,
                            const void *dO, const float *dh_final,
                            void *dx, void *dr, float *dA, void *di, void *dz, float *dh_init,
                            int use_saved, void *workspace, size_t workspace_bytes, void *stream);

/* T new tokens (a few) of B sequences: h_out [B, D], which may be h_in (in place;
 * h_in NULL: zeros), as o may be x, r, i or z with rows next to each other.  No
 * workspace; dense only (RLA_ERR_UNSUPPORTED with cu_seqlens). */
rla_status rla_glr_decode(const rla_glr_problem *problem, const void *x, const void *r,
                          const float *A, const void *i, const void *z, const float *h_in,
                          void *o, float *h_out, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* RLA_MI355X_RLA_MODEL_H */
