/*
 * lsam_ops.h -- operators of token models for AMD MI355X (gfx950), in liblsam.so.
 *
 * The step engine of lsam.h takes gradients of any model in its raw-vector mode
 * (lsam_step_grads: [K, d] fp32 vectors).  These are the operators such a model of K replicas is
 * made of where it reads tokens.  They hold no context: every call is one pass over arrays that
 * are the caller's.
 *
 * Conventions are those of lsam.h: C linkage, 0 or a negative LSAM_E* code with a message in
 * lsam_last_error(), pointers marked [host] or [device], kernels enqueued on the caller's stream,
 * nothing allocated, the host never blocked, every call valid under HIP graph capture.  Strides are
 * counted in elements; the last index of every array is contiguous, and arrays need the
 * alignment of one element only (16-byte aligned rows are faster).  Sizes of zero are valid and
 * launch nothing that has nothing to write.  Outputs must not lie over inputs, except where that
 * is said to be allowed.  Results do not depend on the stream, on timing or on other calls: sums are
 * added in a fixed order.
 */
#ifndef LSAM_OPS_H
#define LSAM_OPS_H

#include "lsam.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LSAM_DTYPE_FP32 0
#define LSAM_DTYPE_BF16 1

/* ---- dropout --------------------------------------------------------------------------------
 * y = residual + m x / (1 - p'), m in {0, 1}, for `replicas` matrices [rows, cols].
 *
 * The mask is a function of where a value is, and never stored: Philox4x32-10 with
 *   counter = (col / 8, row, site | (first_replica + k) << 16, step),  key = seed,
 * gives eight 16-bit numbers for eight neighbouring columns (column 8 j + e takes the low (even e) or
 * high (odd e) half of word e / 2), and a value is kept where its number is at least 65536 p',
 * p' = p rounded to a multiple of 1/65536.  So both passes of a sharpness-aware step, which must see
 * the same function of the parameters, drop the same values when they name the same step, and the
 * backward pass is the same call on dy (dx = m dy / (1 - p'), residual NULL).  `site` tells the dropout
 * layers of a model apart.  A dropped value is exactly 0 whatever x holds there; p = 1 drops all.
 *   x, y [device] replicas matrices of `dtype`; residual [device] the same, or NULL
 * y may be x or residual itself (same pointer and strides). */
typedef struct {
  int32_t replicas;                          /* 0..65535                                     */
  int32_t dtype;                             /* LSAM_DTYPE_*                                 */
  int64_t rows, cols;                        /* of one replica, each below 2^31              */
  int64_t x_stride, x_replica;               /* from row to row, from replica to replica     */
  int64_t residual_stride, residual_replica;
  int64_t y_stride, y_replica;
  double p;                                  /* probability of dropping a value, 0..1        */
  uint64_t seed;
  uint32_t step;
  uint32_t site;                             /* 0..65535                                     */
  uint32_t first_replica;                    /* first_replica + replicas <= 65536            */
} lsam_dropout_desc;
int lsam_dropout(const lsam_dropout_desc* d, const void* x, const void* residual, void* y, void* stream);

/* ---- log probabilities of given tokens --------------------------------------------------------
 * For each of `rows` rows of logits z [vocab] (dtype), with sums in fp32:
 *   lse     [device] [rows, 2] floats: the largest logit m, and ln sum_j e^{z_j - m}.  The log normaliser is their sum;
 *           ln p_j = (z_j - m) - ln sum e^{z - m} keeps its digits however large the logits are
 *   entropy [device] [rows] floats: H = -sum_j p_j ln p_j, p = e^{z - lse}
 *   logp    [device] [rows] floats: ln p of tokens[row]; 0 for a token outside 0..vocab-1, which does not count.
 *           tokens [device] [rows] int32, or NULL: logp is not written
 *   top_ids, top_logp [device] [rows, top]: the `top` largest logits' indices and log probabilities, the largest first, the
 *           lowest index first among equals.  May be NULL where top = 0
 * A logit of -inf is barred: probability 0, gradient 0, never an alternative; where fewer than `top` are left the
 * rest is index -1, log probability -inf.  A row with every logit barred has lse (-inf, 0), entropy 0, logp -inf and
 * no gradient.  NaN or +inf in a row makes its lse, entropy and log probabilities NaN.
 * workspace [device, 16-byte aligned], lsam_logprobs_workspace_bytes(d) bytes (0 where rows fill the chip; also 0, with a
 * message, for a descriptor that is refused); nothing in it has to survive the call. */
#define LSAM_TOP_MAX 32
typedef struct {
  int64_t rows;
  int64_t vocab;                             /* 1..2^31-1                                    */
  int64_t stride;                            /* of the logits, from row to row               */
  int32_t dtype;                             /* LSAM_DTYPE_*                                 */
  int32_t top;                               /* 0..LSAM_TOP_MAX, at most vocab               */
} lsam_logprobs_desc;
size_t lsam_logprobs_workspace_bytes(const lsam_logprobs_desc* d);
int lsam_logprobs(const lsam_logprobs_desc* d, const void* logits, const int32_t* tokens, float* logp, float* lse,
                  float* entropy, int32_t* top_ids, float* top_logp, void* workspace, size_t workspace_bytes, void* stream);

/* Gradient of sum_rows g_logp logp + g_entropy entropy with respect to the logits:
 *   dlogits_j = g_logp (1[j = token] - p_j) - g_entropy p_j (ln p_j + H)
 * g_logp, g_entropy [device] [rows] floats, either may be NULL (0); lse and entropy as the forward call left them.
 * dlogits has the logits' type and may be the logits themselves. `top` is not looked at beyond its range. */
int lsam_logprobs_backward(const lsam_logprobs_desc* d, const void* logits, const int32_t* tokens, const float* lse,
                           const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits,
                           int64_t dlogits_stride, void* stream);

/* ---- gated linear recurrence -------------------------------------------------------------------
 * For every sequence and channel:  h_t = a_t h_{t-1} + (1 - a_t) x_t,  a_t = 1 / (1 + e^{-f_t}),  t = 0, 1, ...,
 * from h_{-1} = h0.  States and sums are fp32; h, df and dx are rounded once, where they are stored.
 *
 * Sequences of equal length (packed = 0): f, x, h are `seqs` matrices [rows, dim]; rows = 1 is a step of generation.
 * Packed sequences of any lengths (packed = 1): f, x, h are one matrix [rows, dim], and sequence i is rows offsets[i] to
 * offsets[i + 1] - 1 of it (offsets [device] [seqs + 1] int64, not decreasing, within 0..rows: values outside are
 * taken as the nearest inside).  Rows of no sequence are neither read nor written.  A sequence of no rows leaves its
 * state as it is.
 *   h0     [device] [seqs, dim] floats, or NULL: 0
 *   last   [device] [seqs, dim] floats that receive the states after the last row, or NULL
 *   states [device] [lsam_recurrence_states(d), dim] floats that receive what the backward pass needs, or NULL
 * workspace [device, 16-byte aligned], lsam_recurrence_workspace_bytes(d) bytes (0 where sequences and channels fill the
 * chip; also 0, with a message, for a descriptor that is refused); nothing in it has to survive a call. */
typedef struct {
  int64_t stride;                            /* from row to row, at least dim                */
  int64_t seq;                               /* from sequence to sequence; packed: not used  */
} lsam_rows;
typedef struct {
  int64_t seqs;
  int64_t rows;                              /* of each sequence; packed: of all             */
  int64_t dim;
  int32_t dtype;                             /* LSAM_DTYPE_* of f, x, h, dh, df, dx          */
  int32_t packed;
  lsam_rows f, x, h;                         /* h: not looked at by the backward pass        */
  lsam_rows dh, df, dx;                      /* not looked at by the forward pass            */
} lsam_recurrence_desc;
size_t lsam_recurrence_workspace_bytes(const lsam_recurrence_desc* d);
int64_t lsam_recurrence_states(const lsam_recurrence_desc* d);
int lsam_recurrence(const lsam_recurrence_desc* d, const int64_t* offsets, const void* f, const void* x, const float* h0,
                    void* h, float* last, float* states, void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of sum dh h + dlast last with respect to f, x and h0:
 *   e_t = a_t (dh_t + e_{t+1}) from e = dlast behind the last row,  d_t = dh_t + e_{t+1},
 *   dx_t = (1 - a_t) d_t,  df_t = a_t (1 - a_t) d_t (h_{t-1} - x_t),  dh0 = e_0.
 * seqs, rows, dim, dtype, packed, offsets, h0 and states are those of the forward call; dlast [device] [seqs, dim] floats or
 * NULL (0); dh0 [device] [seqs, dim] floats or NULL (not wanted). */
int lsam_recurrence_backward(const lsam_recurrence_desc* d, const int64_t* offsets, const void* f, const void* x,
                             const float* h0, const float* states, const void* dh, const float* dlast, void* df, void* dx,
                             float* dh0, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LSAM_OPS_H */
