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

/* ---- embedding ---------------------------------------------------------------------------------
 * y = scale E_k[token] for `rows` tokens of each of `replicas` replicas: rows of the replica's table E_k [vocab, dim], or of one table
 * that all share (table_replica = 0).  A token outside 0..vocab-1 holds nothing (padding): its row of y is 0.
 *   tokens [device] replicas times [rows] int32, token_replica apart
 *   table  [device] of table_dtype;  y [device] of dtype, rounded once */
#define LSAM_EMBEDDING_MAX_VOCAB (1 << 22)
typedef struct {
  int32_t replicas;                          /* 0..65535                                     */
  int32_t dtype, table_dtype;                /* LSAM_DTYPE_* of y and dy, of the table       */
  float scale;
  int64_t rows;                              /* of one replica, below 2^31                   */
  int64_t vocab;                             /* 1..LSAM_EMBEDDING_MAX_VOCAB                  */
  int64_t dim;                               /* 1..2^24                                      */
  int64_t token_replica;                     /* from replica to replica                      */
  int64_t table_stride, table_replica;       /* from row to row, from replica to replica     */
  int64_t y_stride, y_replica;
  int64_t dy_stride, dy_replica;             /* backward pass only, as what follows          */
  int64_t dtable_stride, dtable_replica;
} lsam_embedding_desc;
int lsam_embedding(const lsam_embedding_desc* d, const int32_t* tokens, const void* table, void* y, void* stream);

/* Gradient with respect to the tables:  dE_k[v] = scale sum of the replica's rows of dy whose token is v, in fp32, in the order of the rows.
 *   dtable [device] replicas times [vocab, dim] floats, apart from each other; written whole (0 where a token does not occur), not
 *          added to.  They may be parts of one [replicas, d] array.  The gradient of a table that replicas share is that of one
 *          replica with all their rows
 * workspace [device, 16-byte aligned], lsam_embedding_workspace_bytes(d) bytes (0, with a message, for a descriptor that is refused);
 * nothing in it has to survive the call. */
size_t lsam_embedding_workspace_bytes(const lsam_embedding_desc* d);
int lsam_embedding_backward(const lsam_embedding_desc* d, const int32_t* tokens, const void* dy, float* dtable, void* workspace,
                            size_t workspace_bytes, void* stream);

/* ---- between two blocks --------------------------------------------------------------------------
 * With n(x) = x / sqrt(mean x^2 + eps) over the `dim` numbers of a row, for `rows` rows of each of `replicas` replicas:
 *   r' = alpha r + beta sigmoid(gate) w_post n(y)     what a block made of the stream joins it
 *   h  = w_pre n(r')                                  what the next block reads; the norm is that of r' as it is stored
 *   r, y, gate [device] of dtype; gate NULL: 1
 *   w_post     [device] replicas times [dim] floats, or NULL: y itself in place of w_post n(y)
 *   w_pre      [device] replicas times [dim] floats, or NULL: no h
 *   r_out, h   [device] of dtype.  r_out may be r itself (same pointer and strides)
 * y NULL (before the first block): r' is r, nothing is joined, and r_out, gate and w_post are not looked at.
 * Sums are fp32: a row whose squares pass its range, or whose mean x^2 + eps is below its normal numbers (2^-126), has n(x) = 0, and no gradient through
 * it.  What is not finite in a row reaches no other row. */
#define LSAM_RESIDUAL_MAX_DIM 16384
typedef struct {
  int32_t replicas;                          /* 0..65535                                     */
  int32_t dtype;                             /* LSAM_DTYPE_*                                 */
  int64_t rows;                              /* of one replica, below 2^31                   */
  int64_t dim;                               /* 1..LSAM_RESIDUAL_MAX_DIM                     */
  float alpha, beta, eps;                    /* eps >= 0                                     */
  int64_t w_pre_replica, w_post_replica;     /* from replica to replica; 0: all share one    */
  int64_t r_stride, r_replica;               /* from row to row, from replica to replica     */
  int64_t y_stride, y_replica, gate_stride, gate_replica;
  int64_t r_out_stride, r_out_replica, h_stride, h_replica;
  int64_t dr_stride, dr_replica, dh_stride, dh_replica;              /* backward pass only, as what follows */
  int64_t dr_out_stride, dr_out_replica, dy_stride, dy_replica, dgate_stride, dgate_replica;
  int64_t dw_pre_replica, dw_post_replica;
} lsam_residual_desc;
int lsam_residual(const lsam_residual_desc* d, const void* r, const void* y, const void* gate, const float* w_pre, const float* w_post,
                  void* r_out, void* h, void* stream);

/* Gradients of sum dr r' + dh h, where r is r' as the forward call left it (the stream before it where y is NULL):
 *   D = dr + through(r', w_pre dh),  dr_out = alpha D (D where y is NULL),  o = w_post n(y),  dgate = beta D o s (1 - s),  s = sigmoid(gate),
 *   dy = through(y, beta D s w_post),  dw_pre = sum dh n(r'),  dw_post = sum beta D s n(y) over the rows of a replica,
 *   through(x, g) = (g - n(x) mean(g n(x))) / sqrt(mean x^2 + eps), g itself where there is no norm
 *   dr      [device] of dtype, or NULL: 0.  dr_out may be dr itself (same pointer and strides)
 *   dh      [device] of dtype; not looked at where w_pre is NULL
 *   dr_out, dy, dgate [device] of dtype, dw_pre, dw_post [device] replicas times [dim] floats; each may be NULL: not wanted.  Weights
 *           are written whole, not added to, lie apart from each other, and may be parts of one [replicas, d] array
 * The gradient of weights that replicas share is that of one replica with all their rows.
 * workspace [device, 16-byte aligned], lsam_residual_workspace_bytes(d) bytes (0, with a message, for a descriptor that is refused);
 * needed where a gradient of weights is wanted; nothing in it has to survive the call. */
size_t lsam_residual_workspace_bytes(const lsam_residual_desc* d);
int lsam_residual_backward(const lsam_residual_desc* d, const void* r, const void* y, const void* gate, const float* w_pre,
                           const float* w_post, const void* dr, const void* dh, void* dr_out, void* dy, void* dgate, float* dw_pre,
                           float* dw_post, void* workspace, size_t workspace_bytes, void* stream);

/* ---- attention -----------------------------------------------------------------------------------
 * For sequences packed one after the other, causal, with `heads` query heads in kv_heads groups of neighbours that share keys and values:
 *   o_i = sum_j p_ij v_j,  p_ij = e^{scale q_i k_j - lse_i},  lse_i = ln sum_j e^{scale q_i k_j},  j over the rows of i's sequence up to i itself
 * Sequence s is rows offsets[s] .. offsets[s + 1] - 1 (offsets [device] [seqs + 1] int64, not decreasing, within 0..rows: values outside are
 * taken as the nearest inside).  What rows of no sequence hold reaches nothing, and outputs are not written there.
 *   q, o   [device] [rows, heads, dim], k, v [rows, kv_heads, dim], of dtype; strides from row to row and from head to head are free, so q, k and
 *          v may be parts of one array
 *   lse    [device] [heads, rows] floats that receive lse, for the backward pass, or NULL
 * Scores, sums and lse are fp32.  Products of fp32 operands are those of three bf16 pieces of each, six products in fp32: 2^-22 of |a| |b| at most is
 * left out.  bf16 operands meet probabilities rounded to bf16 (2^-8 of themselves, once, before the sum over j).  A p below 2^-126 is 0, and
 * that of a score of -inf.  What is not finite in a row that i does not see does not reach o_i. */
#define LSAM_ATTENTION_MAX_DIM 128
#define LSAM_ATTENTION_MAX_SCALE 0x1p100f
typedef struct {
  int64_t stride, head;                      /* from row to row, from head to head           */
} lsam_heads;
typedef struct {
  int64_t rows;                              /* rows heads below 2^30                        */
  int64_t seqs;                              /* below 2^31                                   */
  int32_t heads, kv_heads;                   /* heads a multiple of kv_heads, at most 65536  */
  int32_t dim;                               /* 1..LSAM_ATTENTION_MAX_DIM                    */
  int32_t dtype;                             /* LSAM_DTYPE_*                                 */
  float scale;                               /* 0..LSAM_ATTENTION_MAX_SCALE                  */
  lsam_heads q, k, v, o;
  lsam_heads d_o, dq, dk, dv;                /* not looked at by the forward pass            */
} lsam_attention_desc;
int lsam_attention(const lsam_attention_desc* d, const int64_t* offsets, const void* q, const void* k, const void* v, void* o, float* lse,
                   void* stream);

/* Gradients of sum d_o o with respect to q, k and v:
 *   ds_ij = p_ij (d_o_i v_j - d_o_i o_i),  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij d_o_i,
 * those of k and v summed over the heads of their group.  o and lse as the forward call left them; d_o, dq, dk, dv [device] of dtype, laid out
 * as o, q, k and v, strides of their own.  bf16 operands meet p and ds rounded to bf16, and d_o_i o_i is that of o as
 * it was stored, with those roundings: dq and dk are off by about 2.5e-3 of their norm where sequences have a thousand rows, by 3.1e-3 at 16 and 4.4e-3 at 2,
 * where d_o_i v_j - d_o_i o_i cancels most; dv by 2.3e-3 at most.  1.7e-3 of each is their own rounding.
 * workspace [device, 16-byte aligned], lsam_attention_workspace_bytes(d) bytes (0, with a message, for a descriptor that is refused); nothing in
 * it has to survive the call. */
size_t lsam_attention_workspace_bytes(const lsam_attention_desc* d);
int lsam_attention_backward(const lsam_attention_desc* d, const int64_t* offsets, const void* q, const void* k, const void* v, const void* o,
                            const float* lse, const void* d_o, void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                            void* stream);

/* ---- attention of one token -----------------------------------------------------------------------
 * The step of generation: one query of each of `seqs` sequences attends to `prefix` keys and values that all sequences share (an instruction, or one
 * prompt of many answers), and then to the first lengths[s] of its own:  o = softmax(scale q k) v over both.  The prefix is read once for
 * all sequences.  With nothing to attend to, or with scores that are all -inf, o is 0.
 *   q, o               [device] [seqs, heads, dim] of dtype
 *   k, v               [device] caches [seqs, capacity, kv_heads, dim] of dtype; places from lengths[s] on reach nothing
 *   lengths            [device] [seqs] int32; values outside 0..capacity are taken as the nearest inside
 *   prefix_k, prefix_v [device] [prefix, kv_heads, dim] of dtype; may be NULL where prefix is 0
 * Numerics are those of lsam_attention.  All strides of k, v and the prefix may be anything not negative.
 * workspace [device, 16-byte aligned], lsam_attention_step_workspace_bytes(d) bytes (0 where sequences and heads fill the chip; also 0, with a
 * message, for a descriptor that is refused); nothing in it has to survive the call. */
typedef struct {
  int64_t seqs;                              /* seqs heads below 2^23                        */
  int64_t capacity, prefix;                  /* below 2^30                                   */
  int32_t heads, kv_heads;                   /* heads a multiple of kv_heads, at most 65536  */
  int32_t dim;                               /* 1..LSAM_ATTENTION_MAX_DIM                    */
  int32_t dtype;                             /* LSAM_DTYPE_*                                 */
  float scale;                               /* 0..LSAM_ATTENTION_MAX_SCALE                  */
  lsam_heads q, o;                           /* stride: from sequence to sequence            */
  lsam_heads k, v;                           /* stride: from place to place                  */
  int64_t k_seq, v_seq;                      /* from sequence to sequence                    */
  lsam_heads prefix_k, prefix_v;
} lsam_attention_step_desc;
size_t lsam_attention_step_workspace_bytes(const lsam_attention_step_desc* d);
int lsam_attention_step(const lsam_attention_step_desc* d, const int32_t* lengths, const void* q, const void* k, const void* v,
                        const void* prefix_k, const void* prefix_v, void* o, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LSAM_OPS_H */
