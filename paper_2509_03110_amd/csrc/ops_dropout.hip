// lsam_dropout: y = residual + m x / (1 - p'), the mask m a function of a Philox4x32-10 counter.
#include <math.h>

#include "ops.h"
#include "langevin.h"

namespace lsam {
namespace {

constexpr int kThreads = 256;

struct DropoutParams {
  const void* x; const void* residual; void* y;
  int64_t x_stride, x_replica, r_stride, r_replica, y_stride, y_replica;
  uint32_t row0, rows, cols, groups;       // rows of this launch; groups = pieces of 8 columns in a row
  uint32_t key0, key1, step, code;         // code: site | first replica << 16
  uint32_t drop;                           // 65536 p'
  float scale;                             // 1 / (1 - p')
};

// One piece of eight columns per lane: the 128 bits of one counter decide them, so that neither the mask nor a state of a
// generator goes through memory, and the backward call forms the same mask again.  Bound by memory: 8 x 4096 x 4096 bf16 with
// a residual, 805 MB, take 137 us (5.9 TB/s; a copy reaches 6.6); 2 x 32 x 784 fp32 3.2 us, the launch.
template <int DTYPE>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutParams p) {
  typedef Value<DTYPE> V;
  typedef typename V::T T;
  const uint32_t at = blockIdx.x * (uint32_t)kThreads + threadIdx.x;      // rows * groups < 2^31
  const uint32_t r = at / p.groups;
  if (r >= p.rows) return;
  const uint32_t group = at - r * p.groups, row = p.row0 + r, k = blockIdx.y;
  const int64_t col = (int64_t)group * 8;
  const T* x = static_cast<const T*>(p.x) + k * p.x_replica + row * p.x_stride + col;
  const T* res = static_cast<const T*>(p.residual) + k * p.r_replica + row * p.r_stride + col;
  T* y = static_cast<T*>(p.y) + k * p.y_replica + row * p.y_stride + col;
  const int n = p.cols - col < 8 ? (int)(p.cols - col) : 8;
  float v[8], b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (n == 8) {
    V::load8(x, v);
    if (p.residual) V::load8(res, b);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = e < n ? V::get(x + e) : 0.f;
      if (p.residual && e < n) b[e] = V::get(res + e);
    }
  }
  uint32_t w[4];
  philox4x32_10(group, row, p.code + (k << 16), p.step, p.key0, p.key1, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t half = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu;
    v[e] = half >= p.drop ? __builtin_fmaf(v[e], p.scale, b[e]) : b[e];
  }
  if (n == 8) {
    V::store8(y, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) V::put(y + e, v[e]);
  }
}

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" int lsam_dropout(const lsam_dropout_desc* d, const void* x, const void* residual, void* y, void* stream) {
  if (!d) return refuse(LSAM_EINVAL, "dropout: the descriptor is NULL");
  if (!known_dtype(d->dtype)) return refuse(LSAM_EINVAL, "dropout: dtype %d is none of LSAM_DTYPE_*", d->dtype);
  if (d->replicas < 0 || d->replicas > 65535) return refuse(LSAM_EINVAL, "dropout: replicas outside 0..65535");
  if (d->rows < 0 || d->rows >= 1ll << 31 || d->cols < 0 || d->cols >= 1ll << 31)
    return refuse(LSAM_EINVAL, "dropout: rows and cols must be in 0..2^31-1");
  if (!(d->p >= 0.0 && d->p <= 1.0)) return refuse(LSAM_EINVAL, "dropout: p outside 0..1");
  if (d->site > 65535 || (uint64_t)d->first_replica + (uint64_t)d->replicas > 65536)
    return refuse(LSAM_EINVAL, "dropout: site and replicas must be below 65536");
  if (d->replicas == 0 || d->rows == 0 || d->cols == 0) return LSAM_OK;
  const int bytes = dtype_bytes(d->dtype);
  const bool many = d->replicas > 1, tall = d->rows > 1;
  const Arg args[] = {matrices("x", x, d->replicas, d->x_replica, d->rows, d->x_stride, d->cols, bytes, false),
                      matrices("y", y, d->replicas, d->y_replica, d->rows, d->y_stride, d->cols, bytes, true),
                      matrices("the residual", residual, residual ? d->replicas : 0, d->residual_replica, d->rows, d->residual_stride,
                               d->cols, bytes, false)};
  const int rc = check_values(args, 3, "dropout");
  if (rc != LSAM_OK) return rc;
  if (!apart(d->replicas, d->y_replica, d->rows, d->y_stride, d->cols))
    return refuse(LSAM_EINVAL, "dropout: the replicas of y lie over each other");
  if (meet(args[0], args[1]) && !(x == y && (!tall || d->x_stride == d->y_stride) && (!many || d->x_replica == d->y_replica)))
    return refuse(LSAM_EINVAL, "dropout: y lies over x without being x");
  if (meet(args[2], args[1]) &&
      !(residual == y && (!tall || d->residual_stride == d->y_stride) && (!many || d->residual_replica == d->y_replica)))
    return refuse(LSAM_EINVAL, "dropout: y lies over the residual without being it");

  DropoutParams p;
  p.x = x; p.residual = residual; p.y = y;
  p.x_stride = d->x_stride; p.x_replica = d->x_replica;
  p.r_stride = d->residual_stride; p.r_replica = d->residual_replica;
  p.y_stride = d->y_stride; p.y_replica = d->y_replica;
  p.cols = (uint32_t)d->cols;
  p.groups = (uint32_t)((d->cols + 7) / 8);
  p.key0 = (uint32_t)d->seed; p.key1 = (uint32_t)(d->seed >> 32);
  p.step = d->step;
  p.code = d->site | d->first_replica << 16;
  p.drop = (uint32_t)nearbyint(d->p * 65536.0);
  p.scale = p.drop < 65536 ? (float)(65536.0 / (65536 - (int)p.drop)) : 0.f;
  // pieces of a launch are counted in 31 bits: more rows take further launches
  const int64_t most = ((1ll << 31) - kThreads) / p.groups;
  for (int64_t row0 = 0; row0 < d->rows; row0 += most) {
    p.row0 = (uint32_t)row0;
    p.rows = (uint32_t)(d->rows - row0 < most ? d->rows - row0 : most);
    const dim3 grid((unsigned)(((int64_t)p.rows * p.groups + kThreads - 1) / kThreads), (unsigned)d->replicas);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->dtype == LSAM_DTYPE_BF16) dropout_kernel<LSAM_DTYPE_BF16><<<grid, kThreads, 0, s>>>(p);
    else dropout_kernel<LSAM_DTYPE_FP32><<<grid, kThreads, 0, s>>>(p);
  }
  return launched();
}
