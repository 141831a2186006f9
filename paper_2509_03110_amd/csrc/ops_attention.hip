// lsam_attention, lsam_attention_backward: causal attention over packed sequences with grouped heads, and its gradient.
//
//   attention_kernel  o and lse.  A wavefront owns 32 rows of a head, a workgroup 128; it walks over the keys that they see in tiles, forms
//                     the scores of a tile with keys as rows and queries as columns (a lane's column is one query), keeps the running
//                     maximum and sum of each column, and adds the tile's part of o^T
//   dq_kernel         the same walk: scores and d_o v again, ds, dq^T; leaves d_o o and lse of each row for
//   dkv_kernel        a wavefront owns 32 keys, and walks over the rows that see them, head by head of the group: scores with queries as
//                     rows, dv^T and dk^T.  No sum goes over workgroups, so no atomics
//
// Both gradients form the scores again: 7 products in place of 5, for results that do not depend on timing.
#include "attention.h"

namespace lsam {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsOf = 128;               // rows of a workgroup

struct Tensor { void* p; int64_t stride, head; };

struct AttentionParams {
  Tensor q, k, v, o, d_o, dq, dk, dv;
  Sequences seq;
  float* lse;
  float* stats;                            // backward: [2][heads][padded]: lse in powers of 2, d_o o
  int64_t padded;                          // rows, and what a tile may reach past them
  int heads, group, dim, tiles;
  float scale;
};

template <int DTYPE> constexpr int kTile = DTYPE == LSAM_DTYPE_BF16 ? 64 : 32;      // rows of a tile in LDS
template <int DTYPE, int DP> constexpr int kLds = 4 * kTile<DTYPE> * DP * Operand<DTYPE>::B;   // two tensors, two tiles of each

// Which tile of rows and which head a workgroup has.  Workgroups go round the eight XCDs in turn: those that read the same keys
// meet in as few XCDs as that many heads allow.  `of`: heads of a group that are workgroups of their own.
struct Work { int tile, kv, g; bool here; };
__device__ __forceinline__ Work work(int tiles, int kv_heads, int of, bool last_first) {
  const unsigned common = kv_heads % 8 == 0 ? 8 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  const unsigned xcd = blockIdx.x % 8, i = blockIdx.x / 8, parts = 8 / common, mine = kv_heads / common;
  Work w;
  w.g = i % of;
  const unsigned rest = i / of;
  w.kv = (int)(rest % mine * common + xcd % common);
  w.tile = (int)(rest / mine * parts + xcd / common);
  w.here = w.tile < tiles;
  if (last_first) w.tile = tiles - 1 - w.tile;
  return w;
}
unsigned workgroups(int tiles, int kv_heads, int of) {
  const unsigned common = kv_heads % 8 == 0 ? 8 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  const unsigned parts = 8 / common, mine = kv_heads / common;
  return 8 * (((unsigned)tiles + parts - 1) / parts) * mine * of;
}

// What a wavefront's rows see (or are seen by): numbers lo .. hi altogether, all of them from `all_lo` to `all_hi`.
struct Range { int lo, hi, all_lo, all_hi; };
__device__ __forceinline__ Range range_of(bool valid, int first, int last) {
  Range r;
  r.lo = smallest(valid ? first : 0x7FFFFFFF);
  r.hi = largest(valid ? last : -1);
  r.all_lo = largest(valid ? first : -1);
  r.all_hi = smallest(valid ? last : 0x7FFFFFFF);
  return r;
}
// The same for the workgroup.
__device__ __forceinline__ void join_ranges(const Range& r, int& lo, int& hi) {
  __shared__ int shared[2][kThreads / 64];
  if ((threadIdx.x & 63) == 0) { shared[0][threadIdx.x >> 6] = r.lo; shared[1][threadIdx.x >> 6] = r.hi; }
  __syncthreads();
  lo = shared[0][0];
  hi = shared[1][0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) {
    lo = shared[0][i] < lo ? shared[0][i] : lo;
    hi = shared[1][i] > hi ? shared[1][i] : hi;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
}

template <int DTYPE>
__device__ __forceinline__ typename Value<DTYPE>::T* head_of(const Tensor& t, int head) { return static_cast<typename Value<DTYPE>::T*>(t.p) + head * t.head; }

template <int DTYPE, int DP>
__global__ __launch_bounds__(kThreads) void attention_kernel(AttentionParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef Operand<DTYPE> O;
  typedef Rows<DTYPE, DP> R;
  constexpr int BN = kTile<DTYPE>, STEPS = DP / 16;
  __shared__ __attribute__((aligned(16))) unsigned char memory[kLds<DTYPE, DP>];
  lds_byte* const lds = (lds_byte*)memory;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work(p.tiles, p.heads / p.group, p.group, true);
  if (!w.here) return;
  const int head = w.kv * p.group + w.g, row0 = w.tile * kRowsOf + wave * 32, row = row0 + (lane & 31);
  int begin, end;
  span_of(p.seq, row0, row, begin, end);
  const bool valid = end > 0;
  const int first = valid ? begin : 0x7FFFFFFF, last = valid ? row : -1;
  const Range r = range_of(valid, first, last);
  int lo, hi;
  join_ranges(r, lo, hi);
  if (hi < 0) return;

  const HeadRows k{head_of<DTYPE>(p.k, w.kv), p.k.stride}, v{head_of<DTYPE>(p.v, w.kv), p.v.stride};
  Stage<DTYPE, DP, BN, kThreads> sk, sv;
  sk.ask(k, lo, hi + 1, p.dim);
  sv.ask(v, lo, hi + 1, p.dim);
  typename O::F q[STEPS];
  const T* q_row = head_of<DTYPE>(p.q, head) + (valid ? row : 0) * p.q.stride;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) q[s] = load_operand<DTYPE>(q_row, s, lane, valid ? p.dim : 0);

  const float c = exponent(p.scale);
  float m = -__builtin_inff(), l = 0.f;
  f32x16 acc[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) acc[t] = zero16();
  int b = 0;
  for (int j0 = lo; j0 <= hi; j0 += BN, b ^= 1) {
    lds_byte* const tk = lds + b * 2 * BN * R::BYTES;
    lds_byte* const tv = tk + BN * R::BYTES;
    sk.put(tk);
    sv.put(tv);
    __syncthreads();
    if (j0 + BN <= hi) {
      sk.ask(k, j0 + BN, hi + 1, p.dim);
      sv.ask(v, j0 + BN, hi + 1, p.dim);
    }
    if (j0 > r.hi || j0 + BN <= r.lo) continue;
    f32x16 s[BN / 32];
#pragma unroll
    for (int i = 0; i < BN / 32; ++i) s[i] = zero16();
#pragma unroll
    for (int d = 0; d < STEPS; ++d)
#pragma unroll
      for (int i = 0; i < BN / 32; ++i) s[i] = O::multiply(R::along(tk, i * 32, d, lane), q[d], s[i]);
    const bool masked = j0 < r.all_lo || j0 + BN - 1 > r.all_hi;
    if (masked) {
#pragma unroll
      for (int i = 0; i < BN / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = j0 + i * 32 + result_row(e, lane);
          if (j < first || j > last) s[i][e] = -__builtin_inff();
        }
    }
    float most = m;
#pragma unroll
    for (int i = 0; i < BN / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) most = __builtin_fmaxf(most, s[i][e]);
    most = __builtin_fmaxf(most, other_half(most));
    const float base = most == -__builtin_inff() ? 0.f : most * c;
    if (__any(most > m)) {
      const float less = __builtin_amdgcn_exp2f(m * c - base);
      l *= less;
#pragma unroll
      for (int t = 0; t < DP / 32; ++t) acc[t] *= less;
    }
    m = most;
#pragma unroll
    for (int i = 0; i < BN / 32; ++i) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[i][e] = __builtin_amdgcn_exp2f(s[i][e] * c - base);
        l += s[i][e];
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
        multiply_across<DTYPE, DP>(acc, tv, i * 32 + t * 16, O::from(s[i], t), lane, masked, first - j0, last - j0);
    }
  }
  if (!valid) return;
  l += other_half(l);
  store_column<DTYPE, DP>(acc, 1.f / l, head_of<DTYPE>(p.o, head) + row * p.o.stride, lane, p.dim);
  if (p.lse && lane < 32) p.lse[(int64_t)head * p.seq.rows + row] = m * p.scale + __logf(l);
}

template <int DTYPE, int DP>
__global__ __launch_bounds__(kThreads) void dq_kernel(AttentionParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef Operand<DTYPE> O;
  typedef Rows<DTYPE, DP> R;
  constexpr int BN = kTile<DTYPE>, STEPS = DP / 16;
  __shared__ __attribute__((aligned(16))) unsigned char memory[kLds<DTYPE, DP>];
  lds_byte* const lds = (lds_byte*)memory;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work(p.tiles, p.heads / p.group, p.group, true);
  if (!w.here) return;
  const int head = w.kv * p.group + w.g, row0 = w.tile * kRowsOf + wave * 32, row = row0 + (lane & 31);
  int begin, end;
  span_of(p.seq, row0, row, begin, end);
  const bool valid = end > 0;
  const int first = valid ? begin : 0x7FFFFFFF, last = valid ? row : -1;
  const Range r = range_of(valid, first, last);
  int lo, hi;
  join_ranges(r, lo, hi);
  if (hi < 0) return;

  const HeadRows k{head_of<DTYPE>(p.k, w.kv), p.k.stride}, v{head_of<DTYPE>(p.v, w.kv), p.v.stride};
  Stage<DTYPE, DP, BN, kThreads> sk, sv;
  sk.ask(k, lo, hi + 1, p.dim);
  sv.ask(v, lo, hi + 1, p.dim);
  typename O::F q[STEPS], g[STEPS];
  const int at = valid ? row : 0, dim = valid ? p.dim : 0;
  const T* q_row = head_of<DTYPE>(p.q, head) + at * p.q.stride;
  const T* g_row = head_of<DTYPE>(p.d_o, head) + at * p.d_o.stride;
  const T* o_row = head_of<DTYPE>(p.o, head) + at * p.o.stride;
  float dot = 0.f;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    q[s] = load_operand<DTYPE>(q_row, s, lane, dim);
    g[s] = load_operand<DTYPE>(g_row, s, lane, dim);
    const typename O::F o = load_operand<DTYPE>(o_row, s, lane, dim);
#pragma unroll
    for (int e = 0; e < 8; ++e) dot += (float)o[e] * (float)g[s][e];
  }
  dot += other_half(dot);
  const float c = exponent(p.scale), base = valid ? p.lse[(int64_t)head * p.seq.rows + row] * kLog2e : 0.f;
  if (valid && lane < 32) {
    p.stats[head * p.padded + row] = base;
    p.stats[(p.heads + head) * p.padded + row] = dot;
  }
  f32x16 acc[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) acc[t] = zero16();
  int b = 0;
  for (int j0 = lo; j0 <= hi; j0 += BN, b ^= 1) {
    lds_byte* const tk = lds + b * 2 * BN * R::BYTES;
    lds_byte* const tv = tk + BN * R::BYTES;
    sk.put(tk);
    sv.put(tv);
    __syncthreads();
    if (j0 + BN <= hi) {
      sk.ask(k, j0 + BN, hi + 1, p.dim);
      sv.ask(v, j0 + BN, hi + 1, p.dim);
    }
    if (j0 > r.hi || j0 + BN <= r.lo) continue;
    const bool masked = j0 < r.all_lo || j0 + BN - 1 > r.all_hi;
#pragma unroll
    for (int i = 0; i < BN / 32; ++i) {
      f32x16 s = zero16(), d = zero16();
#pragma unroll
      for (int n = 0; n < STEPS; ++n) {
        s = O::multiply(R::along(tk, i * 32, n, lane), q[n], s);
        d = O::multiply(R::along(tv, i * 32, n, lane), g[n], d);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = j0 + i * 32 + result_row(e, lane);
        s[e] = __builtin_amdgcn_exp2f(s[e] * c - base) * (d[e] - dot);
        if (masked && (j < first || j > last)) s[e] = 0.f;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
        multiply_across<DTYPE, DP>(acc, tk, i * 32 + t * 16, O::from(s, t), lane, masked, first - j0, last - j0);
    }
  }
  if (valid) store_column<DTYPE, DP>(acc, p.scale, head_of<DTYPE>(p.dq, head) + row * p.dq.stride, lane, p.dim);
}

template <int DTYPE, int DP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(1, 2))) void dkv_kernel(AttentionParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef Operand<DTYPE> O;
  typedef Rows<DTYPE, DP> R;
  constexpr int BN = kTile<DTYPE>, STEPS = DP / 16;
  __shared__ __attribute__((aligned(16))) unsigned char memory[kLds<DTYPE, DP>];
  lds_byte* const lds = (lds_byte*)memory;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work(p.tiles, p.heads / p.group, 1, false);
  if (!w.here) return;
  const int row0 = w.tile * kRowsOf + wave * 32, row = row0 + (lane & 31);
  int begin, end;
  span_of(p.seq, row0, row, begin, end);
  const bool valid = end > 0;
  const int first = valid ? row : 0x7FFFFFFF, last = valid ? end - 1 : -1;          // rows that see this key
  const Range r = range_of(valid, first, last);
  int lo, hi;
  join_ranges(r, lo, hi);
  if (hi < 0) return;

  typename O::F k[STEPS], v[STEPS];
  const int at = valid ? row : 0, dim = valid ? p.dim : 0;
  const T* k_row = head_of<DTYPE>(p.k, w.kv) + at * p.k.stride;
  const T* v_row = head_of<DTYPE>(p.v, w.kv) + at * p.v.stride;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    k[s] = load_operand<DTYPE>(k_row, s, lane, dim);
    v[s] = load_operand<DTYPE>(v_row, s, lane, dim);
  }
  const float c = exponent(p.scale);
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int t = 0; t < DP / 32; ++t) dk[t] = dv[t] = zero16();
  Stage<DTYPE, DP, BN, kThreads> sq, sg;
  auto ask = [&](int head, int i0) {
    sq.ask(HeadRows{head_of<DTYPE>(p.q, head), p.q.stride}, i0, hi + 1, p.dim);
    sg.ask(HeadRows{head_of<DTYPE>(p.d_o, head), p.d_o.stride}, i0, hi + 1, p.dim);
  };
  int head = w.kv * p.group, b = 0;
  const int behind = head + p.group;
  ask(head, lo);
  for (int i0 = lo; head < behind; b ^= 1) {
    lds_byte* const tq = lds + b * 2 * BN * R::BYTES;
    lds_byte* const tg = tq + BN * R::BYTES;
    sq.put(tq);
    sg.put(tg);
    __syncthreads();
    const int now = i0, with = head;
    i0 += BN;
    if (i0 > hi) { i0 = lo; ++head; }
    if (head < behind) ask(head, i0);
    const float* base = p.stats + with * p.padded;
    const float* dots = base + p.heads * p.padded;
#pragma unroll
    for (int i = 0; i < BN / 32; ++i) {
      const int top = now + i * 32;
      if (top > r.hi || top + 32 <= r.lo) continue;
      const bool masked = top < r.all_lo || top + 31 > r.all_hi;
      f32x16 s = zero16(), d = zero16();
#pragma unroll
      for (int n = 0; n < STEPS; ++n) {
        s = O::multiply(R::along(tq, i * 32, n, lane), k[n], s);
        d = O::multiply(R::along(tg, i * 32, n, lane), v[n], d);
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int of = top + 8 * g + 4 * (lane >> 5);
        const f32x4 bs = *reinterpret_cast<const f32x4_any*>(base + of), ds = *reinterpret_cast<const f32x4_any*>(dots + of);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float pr = __builtin_amdgcn_exp2f(s[4 * g + e] * c - bs[e]);
          s[4 * g + e] = pr;
          d[4 * g + e] = pr * (d[4 * g + e] - ds[e]);
          if (masked && (of + e < first || of + e > last)) s[4 * g + e] = d[4 * g + e] = 0.f;
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        multiply_across<DTYPE, DP>(dv, tg, i * 32 + t * 16, O::from(s, t), lane, masked, first - now, last - now);
        multiply_across<DTYPE, DP>(dk, tq, i * 32 + t * 16, O::from(d, t), lane, masked, first - now, last - now);
      }
    }
  }
  if (!valid) return;
  store_column<DTYPE, DP>(dk, p.scale, head_of<DTYPE>(p.dk, w.kv) + row * p.dk.stride, lane, p.dim);
  store_column<DTYPE, DP>(dv, 1.f, head_of<DTYPE>(p.dv, w.kv) + row * p.dv.stride, lane, p.dim);
}

int check(const lsam_attention_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype)) return refuse(LSAM_EINVAL, "%s: dtype %d is none of LSAM_DTYPE_*", who, d->dtype);
  if (d->kv_heads < 1 || d->heads < 1 || d->heads > 65536 || d->heads % d->kv_heads)
    return refuse(LSAM_EINVAL, "%s: heads must be a multiple of kv_heads, in 1..65536", who);
  if (d->dim < 1 || d->dim > LSAM_ATTENTION_MAX_DIM) return refuse(LSAM_EINVAL, "%s: dim must be in 1..%d", who, LSAM_ATTENTION_MAX_DIM);
  if (d->seqs < 0 || d->seqs >= 1ll << 31) return refuse(LSAM_EINVAL, "%s: seqs must be in 0..2^31-1", who);
  if (d->rows < 0 || d->rows >= 1ll << 31 || d->rows * d->heads >= 1ll << 31) return refuse(LSAM_EINVAL, "%s: rows times heads must be below 2^31", who);
  if (!(d->scale >= 0.f) || d->scale > 3e38f) return refuse(LSAM_EINVAL, "%s: the scale must be finite and not negative", who);
  return LSAM_OK;
}

// A tensor as an argument: heads inside of rows, or rows inside of heads.
Arg arg(const lsam_attention_desc* d, const char* name, const void* p, const lsam_heads& t, int heads, bool output) {
  const int b = dtype_bytes(d->dtype);
  if (heads > 1 && t.head >= d->dim && d->rows > 1 && (__int128)t.stride >= (__int128)(heads - 1) * t.head + d->dim)
    return matrices(name, p, 1, 0, d->rows, t.stride, (heads - 1) * t.head + d->dim, b, output);
  Arg a = matrices(name, p, heads, t.head, d->rows, t.stride, d->dim, b, output);
  if (output && !apart(heads, t.head, d->rows, t.stride, d->dim)) a.bytes = -1;
  return a;
}
Tensor tensor(const void* p, const lsam_heads& t) { return Tensor{const_cast<void*>(p), t.stride, t.head}; }

AttentionParams params(const lsam_attention_desc* d, const int64_t* offsets) {
  AttentionParams p{};
  p.seq = Sequences{offsets, (int)d->seqs, (int)d->rows};
  p.heads = d->heads; p.group = d->heads / d->kv_heads; p.dim = d->dim; p.scale = d->scale;
  p.tiles = (int)((d->rows + kRowsOf - 1) / kRowsOf);
  p.padded = (d->rows + 127) / 64 * 64;
  return p;
}

template <int DTYPE, int DP>
int launch(const AttentionParams& p, bool backward, hipStream_t s) {
  const unsigned all = workgroups(p.tiles, p.heads / p.group, p.group), of_keys = workgroups(p.tiles, p.heads / p.group, 1);
  if (backward) {
    dq_kernel<DTYPE, DP><<<all, kThreads, 0, s>>>(p);
    dkv_kernel<DTYPE, DP><<<of_keys, kThreads, 0, s>>>(p);
  } else {
    attention_kernel<DTYPE, DP><<<all, kThreads, 0, s>>>(p);
  }
  return launched();
}
int launch_any(const AttentionParams& p, int dtype, bool backward, hipStream_t s) {
  if (dtype == LSAM_DTYPE_BF16)
    return p.dim <= 64 ? launch<LSAM_DTYPE_BF16, 64>(p, backward, s) : launch<LSAM_DTYPE_BF16, 128>(p, backward, s);
  return p.dim <= 64 ? launch<LSAM_DTYPE_FP32, 64>(p, backward, s) : launch<LSAM_DTYPE_FP32, 128>(p, backward, s);
}

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" int lsam_attention(const lsam_attention_desc* d, const int64_t* offsets, const void* q, const void* k, const void* v, void* o, float* lse,
                              void* stream) {
  const char* who = "attention";
  int rc = check(d, who);
  if (rc != LSAM_OK) return rc;
  if (d->rows == 0 || d->seqs == 0) return LSAM_OK;
  const Arg args[] = {arg(d, "q", q, d->q, d->heads, false), arg(d, "k", k, d->k, d->kv_heads, false), arg(d, "v", v, d->v, d->kv_heads, false),
                      arg(d, "o", o, d->o, d->heads, true), {"offsets", offsets, (d->seqs + 1) * 8, 8, false},
                      {"lse", lse, lse ? d->heads * d->rows * 4 : 0, 4, true}};
  constexpr int n = sizeof args / sizeof args[0];
  rc = check_values(args, n, who);
  if (rc == LSAM_OK) rc = check_apart(args, n, who);
  if (rc != LSAM_OK) return rc;
  AttentionParams p = params(d, offsets);
  p.q = tensor(q, d->q); p.k = tensor(k, d->k); p.v = tensor(v, d->v); p.o = tensor(o, d->o);
  p.lse = lse;
  return launch_any(p, d->dtype, false, static_cast<hipStream_t>(stream));
}

extern "C" size_t lsam_attention_workspace_bytes(const lsam_attention_desc* d) {
  if (check(d, "attention") != LSAM_OK) return 0;
  const AttentionParams p = params(d, nullptr);
  return (size_t)p.heads * p.padded * 2 * 4;
}

extern "C" int lsam_attention_backward(const lsam_attention_desc* d, const int64_t* offsets, const void* q, const void* k, const void* v, const void* o,
                                       const float* lse, const void* d_o, void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                                       void* stream) {
  const char* who = "attention_backward";
  int rc = check(d, who);
  if (rc != LSAM_OK) return rc;
  if (d->rows == 0 || d->seqs == 0) return LSAM_OK;
  const Arg args[] = {arg(d, "q", q, d->q, d->heads, false), arg(d, "k", k, d->k, d->kv_heads, false), arg(d, "v", v, d->v, d->kv_heads, false),
                      arg(d, "o", o, d->o, d->heads, false), arg(d, "d_o", d_o, d->d_o, d->heads, false),
                      {"lse", lse, d->heads * d->rows * 4, 4, false}, {"offsets", offsets, (d->seqs + 1) * 8, 8, false},
                      arg(d, "dq", dq, d->dq, d->heads, true), arg(d, "dk", dk, d->dk, d->kv_heads, true),
                      arg(d, "dv", dv, d->dv, d->kv_heads, true)};
  constexpr int n = sizeof args / sizeof args[0];
  rc = check_values(args, n, who);
  if (rc == LSAM_OK) rc = check_apart(args, n, who);
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, lsam_attention_workspace_bytes(d), 16, who);
  if (rc != LSAM_OK) return rc;
  AttentionParams p = params(d, offsets);
  p.q = tensor(q, d->q); p.k = tensor(k, d->k); p.v = tensor(v, d->v); p.o = tensor(o, d->o);
  p.d_o = tensor(d_o, d->d_o); p.dq = tensor(dq, d->dq); p.dk = tensor(dk, d->dk); p.dv = tensor(dv, d->dv);
  p.lse = const_cast<float*>(lse); p.stats = static_cast<float*>(workspace);
  return launch_any(p, d->dtype, true, static_cast<hipStream_t>(stream));
}
