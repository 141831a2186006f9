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

#ifdef __cplusplus
}
#endif
#endif /* LSAM_OPS_H */
