// lsam_logprobs, lsam_logprobs_backward: log probabilities of given tokens, entropy and the best alternatives of
// rows of logits, and the gradient.
//
// One pass over the logits.  With m the largest logit seen so far a lane keeps s = sum e^{z-m} and
// t = sum e^{z-m} (z-m); where m grows by D, s becomes s e^{-D} and t becomes (t - s D) e^{-D}.  Then
//   ln sum e^z = m + ln s,    entropy = ln s - t / s.
// Sums are fp32, joined in a fixed order over lanes, wavefronts and pieces of a row.  m and ln s stay apart: in their
// sum, ln s drowns where the logits are large (rows masked with the type's lowest value), and with it the difference
// between certainty and an even choice.
#include "ops.h"

namespace lsam {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxSplits = 64;         // pieces of a row: what one wavefront joins
constexpr int kCandidates = 1024;

typedef unsigned long long u64;

struct LogprobParams {
  const void* z; int64_t stride;
  int64_t row0, rows; int64_t V;       // rows of this launch
  const int32_t* tokens;
  float* logp; float* lse; float* entropy;
  int32_t* ids; float* best;
  int top, splits;
  int64_t piece;                       // logits of a row that one workgroup reads
  float* part;                         // [rows][splits][4]: m, s, t of a piece
  u64* part_keys;                      // [rows][splits][top]
};

// Order of alternatives: larger logits first, lower indices first among equals.  The key of a logit grows with it (NaN
// above all); 0 stands for none, which a logit of -inf is too.
__device__ __forceinline__ unsigned key_of(float z) {
  if (z == -__builtin_inff()) return 0u;
  const unsigned u = __builtin_bit_cast(unsigned, z + 0.f);           // -0 ranks as 0
  if (z != z) return 0xFFFFFFFFu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(unsigned key) {
  if (key == 0xFFFFFFFFu) return __builtin_nanf("");
  return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ u64 ranked(unsigned key, unsigned index) { return (u64)key << 32 | (0xFFFFFFFFu - index); }

struct TopShared {
  u64 list[2][LSAM_TOP_MAX];           // the best so far, best first, and the next such list
  u64 cand[kCandidates + 8];
  u64 wave_max[kWaves];
  unsigned bound[kWaves];
  int count, hits;
};

// Puts the `top` best of the list (`have` entries, in list[cur]) and of the N logits that each lane holds into
// list[cur ^ 1] and returns how many there are.  `later`: all indices are above those in the list, so that equals of its
// last entry rank behind it.
//
// A wavefront's top-th largest of its 64 lane maxima is no larger than the block's top-th largest logit: what lies
// below that bound (found bit by bit, with ballots) cannot be among the best.  Little more than `top` candidates are
// left as a rule, the list among them; each counts the candidates above it, which is its rank.  Where many equals leave too many
// of them, the best are found one after the other instead.
template <int N>
__device__ __forceinline__ int join_top(TopShared& sh, int cur, int have, int top, const unsigned (&key)[N],
                                        const unsigned (&index)[N], bool later) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const u64* list = sh.list[cur];
  u64* next = sh.list[cur ^ 1];
  const unsigned last = have == top && later ? (unsigned)(list[top - 1] >> 32) : 0u;
  unsigned most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) most = key[i] > most ? key[i] : most;
  if (tid == 0) { sh.count = have; sh.hits = 0; }
  if (tid < have) sh.cand[tid] = list[tid];
  __syncthreads();
  if (__ballot(most > last) != 0 && lane == 0) sh.hits = 1;
  // 18 bits tell bfloat16 logits apart and fp32 ones to 2^-9: a bound that is a little low lets a few more candidates through
  unsigned bound = 0;
#pragma unroll
  for (int bit = 31; bit >= 14; --bit) {
    const unsigned trial = bound | 1u << bit;
    if (__popcll(__ballot(most >= trial)) >= top) bound = trial;
  }
  if (lane == 0) sh.bound[wave] = bound;
  __syncthreads();
  if (!sh.hits) {                       // the same for all: nothing of these is better
    if (tid < have) next[tid] = list[tid];
    __syncthreads();
    return have;
  }
#pragma unroll
  for (int w = 0; w < kWaves; ++w) bound = sh.bound[w] > bound ? sh.bound[w] : bound;
  if (most > last && most >= bound) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (key[i] > last && key[i] >= bound) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kCandidates) sh.cand[at] = ranked(key[i], index[i]);
      }
  }
  __syncthreads();
  const int n = sh.count;
  int got = n < top ? n : top;
  if (n <= kCandidates) {
    // nothing behind the last candidate is above any, so that they can be read eight at a time
    if (tid < 8) sh.cand[n + tid] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += kThreads) {
      const u64 mine = sh.cand[j];
      int above = 0;
      for (int i = 0; i < n; i += 8) {
        u64 c[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = sh.cand[i + e];
#pragma unroll
        for (int e = 0; e < 8; ++e) above += c[e] > mine;
      }
      if (above < top) next[above] = mine;
    }
  } else {
    u64 below = ~0ull;
    got = 0;
    for (int r = 0; r < top; ++r) {
      u64 m = tid < have && list[tid] < below ? list[tid] : 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const u64 c = key[i] ? ranked(key[i], index[i]) : 0;
        if (c < below && c > m) m = c;
      }
      for (int off = 32; off > 0; off >>= 1) {
        const u64 o = __shfl_xor(m, off, 64);
        m = o > m ? o : m;
      }
      if (lane == 0) sh.wave_max[wave] = m;
      __syncthreads();
      m = sh.wave_max[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) m = sh.wave_max[w] > m ? sh.wave_max[w] : m;
      __syncthreads();
      if (m == 0) break;                // the same for all
      if (tid == 0) next[r] = m;
      below = m;
      ++got;
    }
  }
  __syncthreads();
  return got;
}

struct Sums { float m, s, t; };

__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
  const float m = __builtin_fmaxf(a.m, b.m);
  Sums r{m, 0.f, 0.f};
  const float inf = __builtin_inff();
  if (a.m != -inf || a.s != 0.f) {
    const float d = a.m - m, e = __expf(d);
    r.s += a.s * e;
    r.t += e != 0.f ? (a.t + a.s * d) * e : 0.f;
  }
  if (b.m != -inf || b.s != 0.f) {
    const float d = b.m - m, e = __expf(d);
    r.s += b.s * e;
    r.t += e != 0.f ? (b.t + b.s * d) * e : 0.f;
  }
  return r;
}

__device__ __forceinline__ Sums join_wave(Sums v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const Sums o{__shfl_xor(v.m, off, 64), __shfl_xor(v.s, off, 64), __shfl_xor(v.t, off, 64)};
    // the lower lane's part comes first on both sides, so that both get the same sum
    v = threadIdx.x & off ? join(o, v) : join(v, o);
  }
  return v;
}

// The row's token and its logit, asked for before the row is read.
struct Wanted { int64_t token; float z; };
template <int DTYPE>
__device__ __forceinline__ Wanted wanted(const LogprobParams& p, int64_t row) {
  typedef typename Value<DTYPE>::T T;
  Wanted w{-1, 0.f};
  if (p.tokens) w.token = p.tokens[row];
  if (w.token >= p.V) w.token = -1;
  if (w.token >= 0) w.z = Value<DTYPE>::get(static_cast<const T*>(p.z) + row * p.stride + w.token);
  return w;
}

// The row's results from its sums; one lane.
__device__ __forceinline__ void finish_row(const LogprobParams& p, int64_t row, const Sums& v, const Wanted& w, float (&lse)[2]) {
  const float inf = __builtin_inff();
  const bool empty = v.m == -inf && v.s == 0.f;                       // every logit is -inf
  const float ln_s = empty ? 0.f : logf(v.s);
  lse[0] = v.s != v.s ? v.s : v.m;                                    // NaN or +inf in the row: NaN
  lse[1] = ln_s;
  p.entropy[row] = empty ? 0.f : ln_s - v.t / v.s;
  p.lse[2 * row] = lse[0];
  p.lse[2 * row + 1] = lse[1];
  if (p.tokens) p.logp[row] = w.token < 0 ? 0.f : empty ? -inf : w.z - lse[0] - ln_s;
}

__device__ __forceinline__ void write_top(const LogprobParams& p, int64_t row, const u64* list, int have, const float* lse) {
  const int j = threadIdx.x;
  if (j >= p.top) return;
  p.ids[row * p.top + j] = j < have ? (int32_t)(0xFFFFFFFFu - (unsigned)list[j]) : -1;
  p.best[row * p.top + j] = j < have ? logit_of((unsigned)(list[j] >> 32)) - lse[0] - lse[1] : -__builtin_inff();
}

// One workgroup per piece of a row; NV words of eight logits in flight for each lane: four, or one in pieces that are read in one
// go (with the best 8 of 700 rows of 50257 49 us against 61, of 64 rows of 32000, in pieces of 2000, 23 against 18).
// Reads every logit once.  8192 x 49999 bf16, 819 MB, rows not aligned: 203-225 us (3.6-4.0 TB/s), bound by the vector units
// (a power, two fused products and the maximum for each logit) and the reading alike; 1 x 131072 with the best 20: 9 us and 6 us
// to join the pieces, 1024 x 1000 fp32 with the best 5: 9 us, bound by the steps of the ranking that wait for each other.
template <int DTYPE, int NV, bool TOP>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobParams p) {
  typedef Value<DTYPE> V;
  typedef typename V::T T;
  constexpr int N = NV * 8;
  constexpr int kStep = kThreads * N;
  __shared__ Sums wave_sums[kWaves];
  __shared__ float row_lse[2];
  __shared__ TopShared top_shared[1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned local = blockIdx.x / (unsigned)p.splits;
  const int64_t row = p.row0 + local;
  const int split = (int)(blockIdx.x - local * (unsigned)p.splits);
  const int64_t begin = split * p.piece, end = begin + p.piece < p.V ? begin + p.piece : p.V;
  const T* z = static_cast<const T*>(p.z) + row * p.stride;
  const float inf = __builtin_inff();
  Sums v{-inf, 0.f, 0.f};
  int have = 0, cur = 0;
  Wanted w{-1, 0.f};
  if (p.splits == 1 && tid == 0) w = wanted<DTYPE>(p, row);
  for (int64_t at = begin; at < end; at += kStep) {
    float x[N];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = at + (j * kThreads + tid) * 8;
      float eight[8];
      if (c + 8 <= end) {
        V::load8(z + c, eight);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) eight[e] = c + e < end ? V::get(z + c + e) : -inf;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * j + e] = eight[e];
    }
    float m = v.m;
#pragma unroll
    for (int e = 0; e < N; ++e) m = __builtin_fmaxf(m, x[e]);
    if (m > v.m) {
      if (v.m != -inf) {
        const float d = v.m - m, e = __expf(d);
        v.t = e != 0.f ? (v.t + v.s * d) * e : 0.f;
        v.s *= e;
      }
      v.m = m;
    }
    const float base = m == -inf ? 0.f : m;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      // a logit so far below that its power is 0 must add 0 to t as well, -inf among them
      const float d = x[e] - base, q = __expf(d);
      v.s += q;
      v.t = __builtin_fmaf(q, __builtin_fmaxf(d, -200.f), v.t);
    }
    if constexpr (TOP) {
      unsigned key[N], index[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        key[e] = key_of(x[e]);
        index[e] = (unsigned)(at + ((e >> 3) * kThreads + tid) * 8 + (e & 7));
      }
      have = join_top<N>(top_shared[0], cur, have, p.top, key, index, true);
      cur ^= 1;
    }
  }
  v = join_wave(v);
  if (lane == 0) wave_sums[wave] = v;
  __syncthreads();
  v = wave_sums[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) v = join(v, wave_sums[w]);
  if (p.splits == 1) {
    if (tid == 0) {
      float lse[2];
      finish_row(p, row, v, w, lse);
      row_lse[0] = lse[0];
      row_lse[1] = lse[1];
    }
    if constexpr (TOP) {
      __syncthreads();
      write_top(p, row, top_shared[0].list[cur], have, row_lse);
    }
  } else {
    const int64_t slot = row * p.splits + split;
    if (tid == 0) *reinterpret_cast<f32x4*>(p.part + 4 * slot) = f32x4{v.m, v.s, v.t, 0.f};
    if constexpr (TOP)
      if (tid < p.top) p.part_keys[slot * p.top + tid] = tid < have ? top_shared[0].list[cur][tid] : 0;
  }
}

// Joins the pieces of a row; one workgroup per row.
template <int DTYPE, bool TOP>
__global__ __launch_bounds__(kThreads) void logprobs_join_kernel(LogprobParams p) {
  constexpr int N = kMaxSplits * LSAM_TOP_MAX / kThreads;
  __shared__ float row_lse[2];
  __shared__ TopShared top_shared[1];
  const int tid = threadIdx.x;
  const int64_t row = p.row0 + blockIdx.x;
  if (tid < 64) {
    Sums v{-__builtin_inff(), 0.f, 0.f};
    Wanted w{-1, 0.f};
    if (tid == 0) w = wanted<DTYPE>(p, row);
    if (tid < p.splits) {
      const f32x4 q = *reinterpret_cast<const f32x4*>(p.part + 4 * (row * p.splits + tid));
      v = Sums{q[0], q[1], q[2]};
    }
    v = join_wave(v);
    if (tid == 0) {
      float lse[2];
      finish_row(p, row, v, w, lse);
      row_lse[0] = lse[0];
      row_lse[1] = lse[1];
    }
  }
  if constexpr (TOP) {
    unsigned key[N], index[N];
    const int n = p.splits * p.top;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = i * kThreads + tid;
      const u64 k = j < n ? p.part_keys[row * n + j] : 0;
      key[i] = (unsigned)(k >> 32);
      index[i] = 0xFFFFFFFFu - (unsigned)k;
    }
    const int have = join_top<N>(top_shared[0], 0, 0, p.top, key, index, false);
    write_top(p, row, top_shared[0].list[1], have, row_lse);
  }
}

// e^x, denormal results included (the instruction has none: it is asked 64 powers of two higher for those).
__device__ __forceinline__ float power(float x) {
  const float y = x * 1.44269504f;
  const bool low = y < -126.f;
  const float e = __builtin_amdgcn_exp2f(low ? y + 64.f : y);
  return low ? e * 0x1p-64f : e;
}

struct GradParams {
  const void* z; int64_t stride;
  void* dz; int64_t dstride;
  int64_t V, row0;
  unsigned pieces;
  const int32_t* tokens; const float* lse; const float* entropy; const float* g_logp; const float* g_entropy;
};

// dz_j = g_logp (1[j = token] - p_j) - g_entropy p_j (ln p_j + H): reads and writes every logit once, nothing else of that size.
// Bound by memory: 8192 x 49999 bf16, 1.64 GB, 253-265 us (6.2-6.5 TB/s; a copy reaches 6.6), 290-326 where every power is
// looked at by itself.
constexpr int kGradWords = 2;
constexpr int kGradStep = kThreads * 8 * kGradWords;
template <int DTYPE>
__global__ __launch_bounds__(kThreads) void logprobs_grad_kernel(GradParams p) {
  typedef Value<DTYPE> V;
  typedef typename V::T T;
  const int tid = threadIdx.x;
  const unsigned local = blockIdx.x / p.pieces;
  const int64_t row = p.row0 + local;
  const int64_t begin = (int64_t)(blockIdx.x - local * p.pieces) * kGradStep;
  const T* z = static_cast<const T*>(p.z) + row * p.stride;
  T* dz = static_cast<T*>(p.dz) + row * p.dstride;
  const float inf = __builtin_inff(), lo = p.lse[2 * row + 1], H = p.entropy[row];
  float hi = p.lse[2 * row];
  const bool empty = hi == -inf;
  if (empty) hi = inf;                         // every power is 0 then
  int64_t tok = p.tokens && p.g_logp ? p.tokens[row] : -1;
  if (tok >= p.V) tok = -1;
  const float g = tok >= 0 ? p.g_logp[row] : 0.f;
  const float h = p.g_entropy ? p.g_entropy[row] : 0.f;
  float x[kGradWords][8];
#pragma unroll
  for (int j = 0; j < kGradWords; ++j) {
    const int64_t c = begin + (j * kThreads + tid) * 8;
    if (c + 8 <= p.V) {
      V::load8(z + c, x[j]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[j][e] = c + e < p.V ? V::get(z + c + e) : 0.f;
    }
  }
  // p = e^{z - m} / sum: the quotient once a row.  Powers below the smallest normal number, and those of barred logits, take longer.
  const float share = __expf(-lo), flat = __builtin_fmaf(h, H - lo, g) * share, steep = h * share;
#pragma unroll
  for (int j = 0; j < kGradWords; ++j) {
    const int64_t c = begin + (j * kThreads + tid) * 8;
    float least = inf;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[j][e] -= hi;
      least = __builtin_fminf(least, x[j][e]);
    }
    const int own = tok >= c && tok < c + 8 && !empty ? (int)(tok - c) : 8;
    if (__any(!(least > -87.f))) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float ln = x[j][e] - lo, q = power(ln);
        x[j][e] = q == 0.f ? 0.f : -q * __builtin_fmaf(h, ln + H, g);      // nothing for a barred logit or a row of them
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[j][e] = -__builtin_amdgcn_exp2f(x[j][e] * 1.44269504f) * __builtin_fmaf(steep, x[j][e], flat);
    }
    if (own < 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e == own) x[j][e] += g;
    }
    if (c + 8 <= p.V) {
      V::store8(dz + c, x[j]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (c + e < p.V) V::put(dz + c + e, x[j][e]);
    }
  }
}

// Pieces of a row: one where there are rows enough for four workgroups on every unit, otherwise as many as make that
// many workgroups, of at least 2048 logits each.  For two, four and eight workgroups on a unit 700 rows of 50257 take 21, 21
// and 27 us, with the best 8 48, 49 and 62; 256 rows of 32000 with the best 8 22, 24 and 33.
struct Cut { int splits; int64_t piece; };
Cut cut_rows(int64_t rows, int64_t V) {
  constexpr int64_t kWanted = 1024, kLeast = kThreads * 8;
  int64_t splits = rows > 0 ? kWanted / rows : 1;
  if (splits > kMaxSplits) splits = kMaxSplits;
  if (splits > (V + kLeast - 1) / kLeast) splits = (V + kLeast - 1) / kLeast;
  if (splits < 1) splits = 1;
  int64_t piece = (V + splits - 1) / splits;
  piece = (piece + kLeast - 1) / kLeast * kLeast;
  return {(int)((V + piece - 1) / piece), piece};
}

int check(const lsam_logprobs_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype)) return refuse(LSAM_EINVAL, "%s: dtype %d is none of LSAM_DTYPE_*", who, d->dtype);
  if (d->rows < 0 || d->vocab < 1 || d->vocab >= 1ll << 31) return refuse(LSAM_EINVAL, "%s: rows must be at least 0 and vocab in 1..2^31-1", who);
  if (d->top < 0 || d->top > LSAM_TOP_MAX || d->top > d->vocab)
    return refuse(LSAM_EINVAL, "%s: top outside 0..LSAM_TOP_MAX, or above vocab", who);
  if (extent(1, 0, d->rows, d->stride, d->vocab, dtype_bytes(d->dtype)) < 0)
    return refuse(LSAM_EINVAL, "%s: the row stride is below vocab, or the array is too large", who);
  return LSAM_OK;
}

// A launch has less than 2^32 lanes: more rows take further launches.
constexpr int64_t kMostGroups = 1ll << 23;

template <int DTYPE, bool TOP>
void launch(LogprobParams p, int64_t row0, hipStream_t s) {
  const int64_t most = kMostGroups / p.splits;
  p.row0 = row0;
  p.rows = p.rows - row0 < most ? p.rows - row0 : most;
  const unsigned grid = (unsigned)(p.rows * p.splits);
  if (p.piece <= kThreads * 8) logprobs_kernel<DTYPE, 1, TOP><<<grid, kThreads, 0, s>>>(p);
  else logprobs_kernel<DTYPE, 4, TOP><<<grid, kThreads, 0, s>>>(p);
  if (p.splits > 1) logprobs_join_kernel<DTYPE, TOP><<<(unsigned)p.rows, kThreads, 0, s>>>(p);
}

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" size_t lsam_logprobs_workspace_bytes(const lsam_logprobs_desc* d) {
  if (check(d, "logprobs") != LSAM_OK) return 0;
  const Cut c = cut_rows(d->rows, d->vocab);
  return c.splits > 1 ? (size_t)d->rows * c.splits * (16 + 8 * (size_t)d->top) : 0;
}

extern "C" int lsam_logprobs(const lsam_logprobs_desc* d, const void* logits, const int32_t* tokens, float* logp, float* lse,
                             float* entropy, int32_t* top_ids, float* top_logp, void* workspace, size_t workspace_bytes,
                             void* stream) {
  int rc = check(d, "logprobs");
  if (rc != LSAM_OK) return rc;
  if (d->rows == 0) return LSAM_OK;
  const int bytes = dtype_bytes(d->dtype);
  const int64_t column = d->rows * 4;
  const Arg args[] = {matrices("logits", logits, 1, 0, d->rows, d->stride, d->vocab, bytes, false),
                      {"tokens", tokens, tokens ? column : 0, 4, false}, {"logp", logp, tokens ? column : 0, 4, true},
                      {"lse", lse, 2 * column, 4, true}, {"entropy", entropy, column, 4, true},
                      {"top_ids", top_ids, column * d->top, 4, true}, {"top_logp", top_logp, column * d->top, 4, true}};
  constexpr int n = sizeof args / sizeof args[0];
  rc = check_values(args, n, "logprobs");
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, lsam_logprobs_workspace_bytes(d), 16, "logprobs");
  if (rc == LSAM_OK) rc = check_apart(args, n, "logprobs");
  if (rc != LSAM_OK) return rc;
  const Cut c = cut_rows(d->rows, d->vocab);
  LogprobParams p;
  p.z = logits; p.stride = d->stride; p.rows = d->rows; p.V = d->vocab;
  p.tokens = tokens; p.logp = logp; p.lse = lse; p.entropy = entropy; p.ids = top_ids; p.best = top_logp;
  p.top = d->top; p.splits = c.splits; p.piece = c.piece;
  p.part = static_cast<float*>(workspace);
  p.part_keys = reinterpret_cast<u64*>(static_cast<char*>(workspace) + (size_t)d->rows * c.splits * 16);
  hipStream_t s = static_cast<hipStream_t>(stream);
  for (int64_t row0 = 0; row0 < d->rows; row0 += kMostGroups / c.splits) {
    if (d->dtype == LSAM_DTYPE_BF16) {
      if (d->top) launch<LSAM_DTYPE_BF16, true>(p, row0, s); else launch<LSAM_DTYPE_BF16, false>(p, row0, s);
    } else {
      if (d->top) launch<LSAM_DTYPE_FP32, true>(p, row0, s); else launch<LSAM_DTYPE_FP32, false>(p, row0, s);
    }
  }
  return launched();
}

extern "C" int lsam_logprobs_backward(const lsam_logprobs_desc* d, const void* logits, const int32_t* tokens, const float* lse,
                                      const float* entropy, const float* g_logp, const float* g_entropy, void* dlogits,
                                      int64_t dlogits_stride, void* stream) {
  int rc = check(d, "logprobs_backward");
  if (rc != LSAM_OK) return rc;
  if (d->rows == 0) return LSAM_OK;
  if (g_logp && !tokens) return refuse(LSAM_EINVAL, "logprobs_backward: g_logp without tokens");
  const int bytes = dtype_bytes(d->dtype);
  const int64_t column = d->rows * 4;
  const bool in_place = logits == dlogits && (d->rows == 1 || d->stride == dlogits_stride);
  const Arg args[] = {matrices("dlogits", dlogits, 1, 0, d->rows, dlogits_stride, d->vocab, bytes, true),
                      {"tokens", tokens, tokens ? column : 0, 4, false}, {"lse", lse, 2 * column, 4, false},
                      {"entropy", entropy, column, 4, false}, {"g_logp", g_logp, g_logp ? column : 0, 4, false},
                      {"g_entropy", g_entropy, g_entropy ? column : 0, 4, false},
                      matrices("logits", logits, 1, 0, d->rows, d->stride, d->vocab, bytes, false)};
  constexpr int n = sizeof args / sizeof args[0];
  rc = check_values(args, n, "logprobs_backward");
  if (rc == LSAM_OK) rc = check_apart(args, in_place ? n - 1 : n, "logprobs_backward");      // dlogits may be the logits themselves
  if (rc != LSAM_OK) return rc;
  GradParams p;
  p.z = logits; p.stride = d->stride; p.dz = dlogits; p.dstride = dlogits_stride; p.V = d->vocab;
  p.pieces = (unsigned)((d->vocab + kGradStep - 1) / kGradStep);
  p.tokens = tokens; p.lse = lse; p.entropy = entropy; p.g_logp = g_logp; p.g_entropy = g_entropy;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t most = kMostGroups / p.pieces;
  for (p.row0 = 0; p.row0 < d->rows; p.row0 += most) {
    const int64_t n = d->rows - p.row0 < most ? d->rows - p.row0 : most;
    const unsigned grid = (unsigned)(n * p.pieces);
    if (d->dtype == LSAM_DTYPE_BF16) logprobs_grad_kernel<LSAM_DTYPE_BF16><<<grid, kThreads, 0, s>>>(p);
    else logprobs_grad_kernel<LSAM_DTYPE_FP32><<<grid, kThreads, 0, s>>>(p);
  }
  return launched();
}
