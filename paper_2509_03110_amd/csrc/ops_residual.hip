// lsam_residual, lsam_residual_backward: r' = alpha r + beta sigmoid(gate) w_post n(y), h = w_pre n(r'), and its gradient.
//
// A workgroup holds whole rows in registers, so that every array is read once and written once: eight numbers of a row a
// lane, or sixteen, and as many wavefronts as that takes.  The sums over a row go through a wavefront's lanes and LDS.  The
// backward pass forms both norms again from r' and y, of which it needs every number anyway; its sums over rows stay in
// registers while a workgroup walks over some of a replica's rows, and a second launch adds those of the workgroups.
// Bound by memory.  3 x 5001 x 1001 fp32 (240 MB, which the last-level cache holds in part): 39 us, 6.2 TB/s; the gradient of 8 x 2048 x 4096 bf16 with gate and
// both weights (1.07 GB): 228 us, 4.7 TB/s, 8 of them for the workgroups' sums.  Registers do not hold what the gradient keeps of rows of more than 8192 numbers, nor of more
// than 4096 of fp32: 540 MB of 8192 numbers a row take 149 us in bf16 and 182 in fp32, of 16384 639 and 604 (540 and 768 bytes a lane in memory).
#include "ops.h"

namespace lsam {
namespace {

struct Tensor { void* p; int64_t stride, replica; };

struct ResidualParams {
  Tensor r, y, gate, r_out, h, dr, dh, dr_out, dy, dgate;
  const float* w_pre; const float* w_post;
  int64_t w_pre_replica, w_post_replica;
  int64_t rows, row0, dim;
  float alpha, beta, eps;
  int32_t replica0;
  int groups;                            // backward: workgroups of a replica, each takes every groups-th row
  float* sums;                           // [replicas][groups][2][dim]: of w_pre, of w_post
  bool want_pre, want_post;
};
struct SumsParams { const float* sums; float* out[2]; int64_t stride[2], dim; int groups; int32_t replica0; };

// Eight numbers as they are stored.
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <int DTYPE> struct Raw;
template <> struct Raw<LSAM_DTYPE_BF16> {
  typedef u16x8 T;
  static __device__ __forceinline__ T load(const unsigned short* p) { return *reinterpret_cast<const u16x8_any*>(p); }
  static __device__ __forceinline__ float wide(unsigned short v) { return widen(v); }
};
template <> struct Raw<LSAM_DTYPE_FP32> {
  typedef f32x8 T;
  static __device__ __forceinline__ T load(const float* p) {
    const f32x4 a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  static __device__ __forceinline__ float wide(float v) { return v; }
};

// Sum over all lanes of the workgroup, the same in each; `shared`: a number for each wavefront, not in use.
template <int WAVES>
__device__ __forceinline__ float sum_over_row(float v, float* shared) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += shared[w];
  }
  return v;
}

// The same for N sums at once.
template <int WAVES, int N>
__device__ __forceinline__ void sums_over_row(float (&v)[N], float (*shared)[WAVES]) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) shared[i][threadIdx.x >> 6] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v[i] += shared[i][w];
    }
  }
}

// A lane's numbers of a row: CH runs of eight, neighbouring lanes side by side.
template <int WAVES, int CH>
struct Columns {
  int64_t dim;
  __device__ __forceinline__ int64_t col(int c) const { return (int64_t)(c * WAVES * 64 + threadIdx.x % (WAVES * 64)) * 8; }
  __device__ __forceinline__ int count(int c) const {
    const int64_t n = dim - col(c);
    return n < 0 ? 0 : n < 8 ? (int)n : 8;
  }
  template <int DTYPE>
  __device__ __forceinline__ void load(const typename Value<DTYPE>::T* p, float (&v)[CH][8]) const {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int n = count(c);
      if (n == 8) {
        Value<DTYPE>::load8(p + col(c), v[c]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = e < n ? Value<DTYPE>::get(p + col(c) + e) : 0.f;
      }
    }
  }
  // As they are stored, for a row ahead; zeros behind the row's end.
  template <int DTYPE>
  __device__ __forceinline__ void ask(const typename Value<DTYPE>::T* p, typename Raw<DTYPE>::T (&v)[CH]) const {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int n = count(c);
      if (n == 8) {
        v[c] = Raw<DTYPE>::load(p + col(c));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[c][e] = 0;
          if (e < n) v[c][e] = p[col(c) + e];
        }
      }
    }
  }
  template <int DTYPE>
  __device__ __forceinline__ void store(typename Value<DTYPE>::T* p, const float (&v)[CH][8]) const {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int n = count(c);
      if (n == 8) {
        Value<DTYPE>::store8(p + col(c), v[c]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n) Value<DTYPE>::put(p + col(c) + e, v[c][e]);
      }
    }
  }
};

template <int DTYPE, int CH>
__device__ __forceinline__ void widen_row(const typename Raw<DTYPE>::T (&r)[CH], float (&v)[CH][8]) {
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) v[c][e] = Raw<DTYPE>::wide(r[c][e]);
}

template <int DTYPE>
__device__ __forceinline__ typename Value<DTYPE>::T* row_of(const Tensor& t, int64_t replica, int64_t row) {
  return static_cast<typename Value<DTYPE>::T*>(t.p) + replica * t.replica + row * t.stride;
}

// 1 / (1 + e^-x), and what is missing to 1, neither from the other: both keep their digits where they are small.
__device__ __forceinline__ void sigmoid(float x, float& s, float& rest) {
  const float e = __expf(-__builtin_fabsf(x)), r = __builtin_amdgcn_rcpf(1.f + e), small = e * r;
  s = x >= 0.f ? r : small;
  rest = x >= 0.f ? small : r;
}
template <int CH>
__device__ __forceinline__ float squares(const float (&v)[CH][8]) {
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[c][e] * v[c][e];
  return s;
}
// 1 / sqrt(mean x^2 + eps); 0 where that mean is below the normal numbers, as 1 / inf is where it is above: squares lose digits there, down to 1 / 0.  (From
// 2^-126 on what underflow takes from dim squares, half a step of 2^-149 each, is at most 2^-24 of their sum.)
__device__ __forceinline__ float inverse(float squares, const ResidualParams& p) {
  const float mean = squares / (float)p.dim + p.eps;
  return mean < 0x1p-126f ? 0.f : 1.f / __builtin_sqrtf(mean);
}

// Rows of a workgroup of the forward pass: where a wavefront holds one, four.
template <int WAVES> constexpr int kRowsOf = WAVES == 1 ? 4 : 1;

template <int DTYPE, int WAVES, int CH>
__global__ __launch_bounds__(WAVES * 64 * kRowsOf<WAVES>) void residual_kernel(ResidualParams p) {
  __shared__ float shared[2][WAVES];
  const Columns<WAVES, CH> at{p.dim};
  const int64_t replica = p.replica0 + blockIdx.y, row = p.row0 + (int64_t)blockIdx.x * kRowsOf<WAVES> + (kRowsOf<WAVES> > 1 ? threadIdx.x >> 6 : 0);
  if (row >= p.rows) return;
  float r[CH][8];
  at.template load<DTYPE>(row_of<DTYPE>(p.r, replica, row), r);
  if (p.y.p) {
    float y[CH][8], g[CH][8], w[CH][8];
    at.template load<DTYPE>(row_of<DTYPE>(p.y, replica, row), y);
    if (p.gate.p) at.template load<DTYPE>(row_of<DTYPE>(p.gate, replica, row), g);
    float inv = 1.f;
    if (p.w_post) {
      at.template load<LSAM_DTYPE_FP32>(p.w_post + replica * p.w_post_replica, w);
      inv = inverse(sum_over_row<WAVES>(squares(y), shared[0]), p);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float o = y[c][e];
        if (p.w_post) o = o * inv * w[c][e];
        if (p.gate.p) {
          float s, rest;
          sigmoid(g[c][e], s, rest);
          o *= s;
        }
        r[c][e] = p.alpha * r[c][e] + p.beta * o;
        if constexpr (DTYPE == LSAM_DTYPE_BF16) r[c][e] = widen(narrow(r[c][e]));       // as it is stored
      }
    at.template store<DTYPE>(row_of<DTYPE>(p.r_out, replica, row), r);
  }
  if (p.w_pre) {
    float w[CH][8];
    at.template load<LSAM_DTYPE_FP32>(p.w_pre + replica * p.w_pre_replica, w);
    const float inv = inverse(sum_over_row<WAVES>(squares(r), shared[1]), p);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) r[c][e] = r[c][e] * inv * w[c][e];
    at.template store<DTYPE>(row_of<DTYPE>(p.h, replica, row), r);
  }
}

// A row's sums are two rounds: the squares of r' and y; then, of m = n(r'), g = w_pre dh, and what is multiplied by c = beta s w_post n(y),
//   sum g m,  sum c (dr + i g),  sum c m    (i = 1 / sqrt(mean r'^2 + eps)),
// of which sum c D = sum c (dr + i g) - i mean(g m) sum c m needs no third.  The next row is on its way meanwhile.
template <int DTYPE, int WAVES, int CH>
__global__ __launch_bounds__(WAVES * 64) void residual_grad_kernel(ResidualParams p) {
  typedef typename Raw<DTYPE>::T Eight;
  __shared__ float shared[2][5][WAVES];
  const Columns<WAVES, CH> at{p.dim};
  const int64_t replica = p.replica0 + blockIdx.y;
  const bool join = p.y.p != nullptr, post = p.w_post != nullptr, gated = p.gate.p != nullptr, pre = p.w_pre != nullptr;
  const float per = 1.f / (float)p.dim;
  float w_pre[CH][8], w_post[CH][8], sum_pre[CH][8], sum_post[CH][8];
  Eight next_r[CH], next_h[CH], next_d[CH], next_y[CH], next_g[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w_pre[c][e] = w_post[c][e] = 1.f;
      sum_pre[c][e] = sum_post[c][e] = 0.f;
      next_r[c][e] = next_h[c][e] = next_d[c][e] = next_y[c][e] = next_g[c][e] = 0;
    }
  }
  if (pre) at.template load<LSAM_DTYPE_FP32>(p.w_pre + replica * p.w_pre_replica, w_pre);
  if (post) at.template load<LSAM_DTYPE_FP32>(p.w_post + replica * p.w_post_replica, w_post);
  const auto ask = [&](int64_t row) {
    if (row >= p.rows) return;
    if (pre) {
      at.template ask<DTYPE>(row_of<DTYPE>(p.r, replica, row), next_r);
      at.template ask<DTYPE>(row_of<DTYPE>(p.dh, replica, row), next_h);
    }
    if (p.dr.p) at.template ask<DTYPE>(row_of<DTYPE>(p.dr, replica, row), next_d);
    if (join) at.template ask<DTYPE>(row_of<DTYPE>(p.y, replica, row), next_y);
    if (join && gated) at.template ask<DTYPE>(row_of<DTYPE>(p.gate, replica, row), next_g);
  };
  ask(blockIdx.x);
  int b = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += p.groups, b ^= 1) {
    float r[CH][8], h[CH][8], d[CH][8], y[CH][8], g[CH][8];
    widen_row<DTYPE>(next_r, r);
    widen_row<DTYPE>(next_h, h);
    widen_row<DTYPE>(next_d, d);
    widen_row<DTYPE>(next_y, y);
    widen_row<DTYPE>(next_g, g);
    ask(row + p.groups);
    float two[2] = {squares(r), squares(y)};
    sums_over_row<WAVES>(two, &shared[b][0]);
    const float ir = pre ? inverse(two[0], p) : 0.f, iy = post ? inverse(two[1], p) : 1.f;
    float three[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float s = 1.f, rest = 0.f;
        if (gated) sigmoid(g[c][e], s, rest);
        r[c][e] *= ir;
        sum_pre[c][e] += h[c][e] * r[c][e];
        h[c][e] *= w_pre[c][e];
        d[c][e] += ir * h[c][e];
        y[c][e] *= iy;
        const float by = p.beta * s * w_post[c][e] * y[c][e];
        three[0] += h[c][e] * r[c][e];
        three[1] += by * d[c][e];
        three[2] += by * r[c][e];
      }
    sums_over_row<WAVES>(three, &shared[b][2]);
    const float dot = ir * three[0] * per, post_dot = (three[1] - dot * three[2]) * per;
    float out[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        d[c][e] -= dot * r[c][e];
        out[c][e] = join ? p.alpha * d[c][e] : d[c][e];
      }
    if (p.dr_out.p) at.template store<DTYPE>(row_of<DTYPE>(p.dr_out, replica, row), out);
    if (!join) continue;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float s = 1.f, rest = 0.f;
        if (gated) sigmoid(g[c][e], s, rest);
        const float whole = p.beta * d[c][e], part = whole * s;
        g[c][e] = whole * (y[c][e] * w_post[c][e]) * (s * rest);
        sum_post[c][e] += part * y[c][e];
        out[c][e] = part * w_post[c][e];
        if (post) out[c][e] = iy * (out[c][e] - y[c][e] * post_dot);
      }
    if (gated && p.dgate.p) at.template store<DTYPE>(row_of<DTYPE>(p.dgate, replica, row), g);
    if (p.dy.p) at.template store<DTYPE>(row_of<DTYPE>(p.dy, replica, row), out);
  }
  float* sums = p.sums + (replica * p.groups + blockIdx.x) * 2 * p.dim;
  if (p.want_pre) at.template store<LSAM_DTYPE_FP32>(sums, sum_pre);
  if (p.want_post) at.template store<LSAM_DTYPE_FP32>(sums + p.dim, sum_post);
}

// Adds the workgroups' sums of a replica, in their order: 64 columns a workgroup, a run of workgroups a wavefront.
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(kSumWaves * 64) void residual_sums_kernel(SumsParams p) {
  __shared__ float part[kSumWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, side = blockIdx.y;
  const int64_t replica = p.replica0 + blockIdx.z, col = (int64_t)blockIdx.x * 64 + lane;
  if (!p.out[side]) return;
  const int each = (p.groups + kSumWaves - 1) / kSumWaves, first = wave * each, end = first + each < p.groups ? first + each : p.groups;
  const float* from = p.sums + (replica * p.groups * 2 + side) * p.dim + (col < p.dim ? col : 0);
  float sum = 0.f;
#pragma unroll 8
  for (int i = first; i < end; ++i) sum += from[i * 2 * p.dim];
  part[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || col >= p.dim) return;
#pragma unroll
  for (int w = 1; w < kSumWaves; ++w) sum += part[w][lane];
  p.out[side][replica * p.stride[side] + col] = sum;
}

// Workgroups of a replica in the backward pass: four a unit for all replicas, and no more sums to add than that.
int groups_of(const lsam_residual_desc* d) {
  const int64_t replicas = d->replicas > 0 ? d->replicas : 1;
  int64_t g = (1024 + replicas - 1) / replicas;
  g = g < d->rows ? g : d->rows;
  return (int)(g > 0 ? g : 1);
}

int check(const lsam_residual_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype)) return refuse(LSAM_EINVAL, "%s: dtype %d is none of LSAM_DTYPE_*", who, d->dtype);
  if (d->replicas < 0 || d->replicas > 65535) return refuse(LSAM_EINVAL, "%s: replicas must be in 0..65535", who);
  if (d->rows < 0 || d->rows >= 1ll << 31) return refuse(LSAM_EINVAL, "%s: rows must be in 0..2^31-1", who);
  if (d->dim < 1 || d->dim > LSAM_RESIDUAL_MAX_DIM) return refuse(LSAM_EINVAL, "%s: dim must be in 1..%d", who, LSAM_RESIDUAL_MAX_DIM);
  if (!(d->eps >= 0.f) || d->eps > 3e38f) return refuse(LSAM_EINVAL, "%s: eps must be finite and not negative", who);
  if ((__int128)d->replicas * d->rows * d->dim >= (__int128)1 << 44) return refuse(LSAM_EINVAL, "%s: the arrays are too large", who);
  return LSAM_OK;
}

// The rows of all replicas, where `there`; replicas of an output have to lie apart.
Arg arg(const lsam_residual_desc* d, const char* name, const void* p, int64_t stride, int64_t replica, bool there, bool output) {
  Arg a = matrices(name, p, there ? d->replicas : 0, replica, d->rows, stride, d->dim, dtype_bytes(d->dtype), output);
  if (output && there && !apart(d->replicas, replica, d->rows, stride, d->dim)) a.bytes = -1;
  return a;
}
Arg weights(const lsam_residual_desc* d, const char* name, const float* p, int64_t replica, bool output) {
  Arg a = matrices(name, p, p ? d->replicas : 0, replica, 1, 0, d->dim, 4, output);
  if (output && p && !apart(d->replicas, replica, 1, 0, d->dim)) a.bytes = -1;
  return a;
}
// That outputs lie apart; where `same`, an output lies on args[in] itself.
int check_apart_but(const Arg* args, int n, int in, bool same, const char* who) {
  Arg rest[16];
  int m = 0;
  for (int i = 0; i < n; ++i)
    if (!same || i != in) rest[m++] = args[i];
  return check_apart(rest, m, who);
}

template <int DTYPE, int WAVES, int CH>
void launch(const ResidualParams& p, bool grad, dim3 grid, hipStream_t s) {
  if (grad) {
    residual_grad_kernel<DTYPE, WAVES, CH><<<grid, WAVES * 64, 0, s>>>(p);
  } else {
    grid.x = (grid.x + kRowsOf<WAVES> - 1) / kRowsOf<WAVES>;
    residual_kernel<DTYPE, WAVES, CH><<<grid, WAVES * 64 * kRowsOf<WAVES>, 0, s>>>(p);
  }
}
template <int DTYPE>
void launch_wide(const ResidualParams& p, bool grad, dim3 grid, hipStream_t s) {
  if (p.dim <= 512) launch<DTYPE, 1, 1>(p, grad, grid, s);
  else if (p.dim <= 1024) launch<DTYPE, 1, 2>(p, grad, grid, s);
  else if (p.dim <= 2048) launch<DTYPE, 4, 1>(p, grad, grid, s);
  else if (p.dim <= 4096) launch<DTYPE, 4, 2>(p, grad, grid, s);
  else if (p.dim <= 8192) launch<DTYPE, 8, 2>(p, grad, grid, s);
  else launch<DTYPE, 16, 2>(p, grad, grid, s);
}
void launch_any(const ResidualParams& p, int dtype, bool grad, dim3 grid, hipStream_t s) {
  if (dtype == LSAM_DTYPE_BF16) launch_wide<LSAM_DTYPE_BF16>(p, grad, grid, s);
  else launch_wide<LSAM_DTYPE_FP32>(p, grad, grid, s);
}

ResidualParams params(const lsam_residual_desc* d, const float* w_pre, const float* w_post) {
  ResidualParams p{};
  p.w_pre = w_pre; p.w_post = w_post;
  p.w_pre_replica = d->w_pre_replica; p.w_post_replica = d->w_post_replica;
  p.rows = d->rows; p.dim = d->dim;
  p.alpha = d->alpha; p.beta = d->beta; p.eps = d->eps;
  return p;
}
Tensor tensor(const void* p, int64_t stride, int64_t replica) { return Tensor{const_cast<void*>(p), stride, replica}; }

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" int lsam_residual(const lsam_residual_desc* d, const void* r, const void* y, const void* gate, const float* w_pre, const float* w_post,
                             void* r_out, void* h, void* stream) {
  const char* who = "residual";
  int rc = check(d, who);
  if (rc != LSAM_OK) return rc;
  if (d->replicas == 0 || d->rows == 0) return LSAM_OK;
  if (!y && !w_pre) return refuse(LSAM_EINVAL, "%s: neither y nor w_pre is there: nothing to do", who);
  const bool join = y != nullptr;
  if (!join) { gate = nullptr; w_post = nullptr; r_out = nullptr; }
  if (!w_pre) h = nullptr;
  const Arg args[] = {arg(d, "r", r, d->r_stride, d->r_replica, true, false),
                      arg(d, "y", y, d->y_stride, d->y_replica, join, false),
                      arg(d, "gate", gate, d->gate_stride, d->gate_replica, gate != nullptr, false),
                      weights(d, "w_pre", w_pre, d->w_pre_replica, false), weights(d, "w_post", w_post, d->w_post_replica, false),
                      arg(d, "r_out", r_out, d->r_out_stride, d->r_out_replica, join, true),
                      arg(d, "h", h, d->h_stride, d->h_replica, w_pre != nullptr, true)};
  constexpr int n = sizeof args / sizeof args[0];
  const bool same = join && r_out == r && d->r_out_stride == d->r_stride && d->r_out_replica == d->r_replica;
  rc = check_values(args, n, who);
  if (rc == LSAM_OK) rc = check_apart_but(args, n, 0, same, who);
  if (rc != LSAM_OK) return rc;
  ResidualParams p = params(d, w_pre, w_post);
  p.r = tensor(r, d->r_stride, d->r_replica); p.y = tensor(y, d->y_stride, d->y_replica); p.gate = tensor(gate, d->gate_stride, d->gate_replica);
  p.r_out = tensor(r_out, d->r_out_stride, d->r_out_replica); p.h = tensor(h, d->h_stride, d->h_replica);
  // launches of less than 2^32 lanes
  const int64_t most = 1 << 21;
  for (p.row0 = 0; p.row0 < d->rows; p.row0 += most) {
    const unsigned rows = (unsigned)(d->rows - p.row0 < most ? d->rows - p.row0 : most), together = (1u << 21) / rows < 65535 ? (1u << 21) / rows : 65535;
    for (unsigned k = 0, K = (unsigned)d->replicas; k < K; k += together) {
      p.replica0 = (int32_t)k;
      launch_any(p, d->dtype, false, dim3(rows, K - k < together ? K - k : together), static_cast<hipStream_t>(stream));
    }
  }
  return launched();
}

extern "C" size_t lsam_residual_workspace_bytes(const lsam_residual_desc* d) {
  if (check(d, "residual") != LSAM_OK) return 0;
  return (size_t)d->replicas * groups_of(d) * 2 * (size_t)d->dim * 4;
}

extern "C" int lsam_residual_backward(const lsam_residual_desc* d, const void* r, const void* y, const void* gate, const float* w_pre,
                                      const float* w_post, const void* dr, const void* dh, void* dr_out, void* dy, void* dgate, float* dw_pre,
                                      float* dw_post, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "residual_backward";
  int rc = check(d, who);
  if (rc != LSAM_OK) return rc;
  if (d->replicas == 0) return LSAM_OK;
  const bool join = y || d->rows == 0;         // an array of no rows may have no address
  if (!join && !w_pre) return refuse(LSAM_EINVAL, "%s: neither y nor w_pre is there: nothing to do", who);
  if (!join) { gate = nullptr; w_post = nullptr; dy = nullptr; }
  if (!w_pre) { r = nullptr; dh = nullptr; dw_pre = nullptr; }
  if (!w_post) dw_post = nullptr;
  if (!gate) dgate = nullptr;
  const Arg args[] = {arg(d, "r", r, d->r_stride, d->r_replica, w_pre != nullptr, false),
                      arg(d, "y", y, d->y_stride, d->y_replica, join, false),
                      arg(d, "gate", gate, d->gate_stride, d->gate_replica, gate != nullptr, false),
                      weights(d, "w_pre", w_pre, d->w_pre_replica, false), weights(d, "w_post", w_post, d->w_post_replica, false),
                      arg(d, "dr", dr, d->dr_stride, d->dr_replica, dr != nullptr, false),
                      arg(d, "dh", dh, d->dh_stride, d->dh_replica, w_pre != nullptr, false),
                      arg(d, "dr_out", dr_out, d->dr_out_stride, d->dr_out_replica, dr_out != nullptr, true),
                      arg(d, "dy", dy, d->dy_stride, d->dy_replica, dy != nullptr, true),
                      arg(d, "dgate", dgate, d->dgate_stride, d->dgate_replica, dgate != nullptr, true),
                      weights(d, "dw_pre", dw_pre, d->dw_pre_replica, true), weights(d, "dw_post", dw_post, d->dw_post_replica, true)};
  constexpr int n = sizeof args / sizeof args[0];
  const bool same = dr && dr_out == dr && d->dr_out_stride == d->dr_stride && d->dr_out_replica == d->dr_replica;
  const int groups = groups_of(d);
  rc = check_values(args, n, who);
  if (rc == LSAM_OK) rc = check_apart_but(args, n, 5, same, who);
  if (rc == LSAM_OK && (dw_pre || dw_post)) rc = check_workspace(args, n, workspace, workspace_bytes, lsam_residual_workspace_bytes(d), 16, who);
  if (rc != LSAM_OK) return rc;
  ResidualParams p = params(d, w_pre, w_post);
  p.r = tensor(r, d->r_stride, d->r_replica); p.y = tensor(y, d->y_stride, d->y_replica); p.gate = tensor(gate, d->gate_stride, d->gate_replica);
  p.dr = tensor(dr, d->dr_stride, d->dr_replica); p.dh = tensor(dh, d->dh_stride, d->dh_replica);
  p.dr_out = tensor(dr_out, d->dr_out_stride, d->dr_out_replica); p.dy = tensor(dy, d->dy_stride, d->dy_replica);
  p.dgate = tensor(dgate, d->dgate_stride, d->dgate_replica);
  p.groups = groups; p.sums = static_cast<float*>(workspace);
  p.want_pre = dw_pre != nullptr; p.want_post = dw_post != nullptr;
  hipStream_t s = static_cast<hipStream_t>(stream);
  // launches of less than 2^32 lanes
  const unsigned K = (unsigned)d->replicas, together = (1u << 21) / groups;
  for (unsigned k = 0; k < K; k += together) {
    p.replica0 = (int32_t)k;
    launch_any(p, d->dtype, true, dim3((unsigned)groups, K - k < together ? K - k : together), s);
  }
  if (dw_pre || dw_post) {
    const unsigned slabs = (unsigned)((d->dim + 63) / 64), apiece = (1u << 20) / slabs;
    for (unsigned k = 0; k < K; k += apiece) {
      const SumsParams q{p.sums, {dw_pre, dw_post}, {d->dw_pre_replica, d->dw_post_replica}, d->dim, groups, (int32_t)k};
      residual_sums_kernel<<<dim3(slabs, 2, K - k < apiece ? K - k : apiece), kSumWaves * 64, 0, s>>>(q);
    }
  }
  return launched();
}
