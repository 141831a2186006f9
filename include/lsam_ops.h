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
 * launch nothing that has nothing to write.  Outputs and workspaces must not lie over inputs or each
 * other, except where that is said to be allowed: such calls are refused.  Results do not depend on the stream, on timing or on other calls: sums are
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
 * A logit of -inf is barred: probability 0, never an alternative, gradient 0 unless it is the row's own token (whose logp is
 * -inf, and whose logit receives g_logp as the formula below has it).  Where fewer than `top` are left the rest is index -1,
 * log probability -inf.  A row with every logit barred has lse (-inf, 0), entropy 0, logp -inf and no gradient.  NaN or +inf in
 * a row makes its lse, entropy and log probabilities NaN.
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
 * from h_{-1} = h0.  States and sums are fp32; h, df and dx are rounded once, where they are stored.  A gate below 2^-126 is 0.  An
 * infinite state stays infinite while the gates are positive, and is NaN behind a gate of 0, as step by step.
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

/* ---- low-rank adapters beside a shared projection ------------------------------------------------
 * For `rows` rows x [in]:  y = x W^T + bias + scale (x A_a^T) B_a^T, with W [out, in] and bias shared by all rows and a the adapter
 * of the row.  The rows of a request, or of a replica, are one segment: segment s is rows seg_begin[s] .. seg_begin[s + 1] - 1
 * (seg_begin [device] [segs + 1] int32, not decreasing; values outside 0..rows are taken as the nearest inside) with adapter
 * seg_adapter[s] ([device] [segs] int32).  Rows of no segment, and of segments whose adapter is outside 0..adapters-1 (-1, say),
 * have none: y = x W^T + bias.  Several segments may share an adapter; segments may be empty.
 *   x, W, y    [device] of dtype; bias [device] [out] floats, or NULL
 *   A, B       [device] of adapter_dtype: adapters matrices [rank, in] and [out, rank], as far apart as a_adapter and b_adapter
 *              say (for replicas whose parameters are rows of a [K, d] array: d)
 *   u          [device] [rows, rank] floats that receive x A_a^T (0 without an adapter), for the backward pass
 * Products are summed in fp32; operands in fp32, u among them, are not rounded to fewer bits.  No value of another row, and none
 * of another adapter, takes part in a row's result; the order in which its sums are added goes by the sizes of the call.
 * What is not finite in x, W, A_a or B_a makes the results it takes part in infinite or NaN.
 * workspace [device, 256-byte aligned], lsam_adapter_workspace_bytes(d, 0) bytes for this call, (d, 1) for the backward one (0, with
 * a message, for a descriptor that is refused); nothing in it has to survive a call.  Parts of it are used only where rows are
 * not aligned to 16 bytes, or fp32. */
#define LSAM_ADAPTER_MAX_RANK 64
typedef struct {
  int64_t rows;                              /* below 2^28                                   */
  int32_t in, out;                           /* 1..2^21; rows in, rows out, in out <= 2^35   */
  int32_t rank;                              /* 1..LSAM_ADAPTER_MAX_RANK                     */
  int32_t adapters, segs;                    /* adapters up to 65535                         */
  int32_t dtype, adapter_dtype;              /* LSAM_DTYPE_*                                 */
  float scale;
  int64_t x_stride, w_stride, y_stride;      /* from row to row                              */
  int64_t a_adapter, a_stride;               /* from adapter to adapter, from rank to rank   */
  int64_t b_adapter, b_stride;               /* from adapter to adapter, from output to output */
  int64_t dy_stride, dx_stride;              /* backward pass only, as what follows          */
  int64_t da_adapter, da_stride, db_adapter, db_stride;
} lsam_adapter_desc;
size_t lsam_adapter_workspace_bytes(const lsam_adapter_desc* d, int32_t backward);
int lsam_adapter(const lsam_adapter_desc* d, const void* x, const void* W, const float* bias, const void* A, const void* B,
                 const int32_t* seg_begin, const int32_t* seg_adapter, float* u, void* y, void* workspace,
                 size_t workspace_bytes, void* stream);

/* Gradients with respect to x, A and B (W and bias are frozen), for the dy of y:
 *   du = scale dy B_a,  dx = dy W + du A_a,  dA_a = sum du^T x,  dB_a = scale sum dy^T u over the rows of adapter a.
 *   u      as the forward call left it
 *   dx     [device] of dtype, or NULL: not wanted
 *   dA, dB [device] floats laid out as A and B are, strides of their own, or both NULL.  Written whole (0 for an adapter
 *          of no row), not added to.  They may be parts of one [adapters, d] array */
int lsam_adapter_backward(const lsam_adapter_desc* d, const void* x, const void* W, const void* A, const void* B,
                          const int32_t* seg_begin, const int32_t* seg_adapter, const float* u, const void* dy, void* dx,
                          float* dA, float* dB, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LSAM_OPS_H */
