// lsam_attention_step: one token of each sequence attends to a prefix that all share and to its own cache.
//
//   step_kernel  keys are cut into parts.  Queries are columns, 32 a wavefront: of the prefix those of all sequences and of a group's heads,
//                of a cache those of its sequence's group alone.  Where there are more than 32 a workgroup's wavefronts take columns of
//                their own and share the keys, tile by tile; where there are not they share the columns, and take 32 keys of a tile
//                each.  A part leaves the maximum, the sum and the weighted values of each column
//   join_kernel  weighs the parts against each other
//
// Bound by memory once keys are many: eight sequences of up to 100000, 2 heads of 64 bf16 numbers: 53 us, 5.6 TB/s.  64 sequences, 32 heads of 128 over 8: a prefix
// of 16001 alone 48 us (each of its keys meets 256 queries: 2.9 times as long as its products take at the rate of large ones), caches of 768 alone 40 (5.0 TB/s), both 64
// in one launch.  One sequence: 8 us and 5 for joining, two launches that follow each other.
#include "attention.h"

namespace lsam {
namespace {

constexpr int kKeys = 128;                 // parts are cut between so many
constexpr int kMaxParts = 64;              // of the prefix, and of a cache

struct Cache { const void* k; const void* v; int64_t k_stride, k_head, k_seq, v_stride, v_head, v_seq; };

struct StepParams {
  Cache prefix, own;
  const void* q; void* o;
  int64_t q_stride, q_head, o_stride, o_head;
  const int32_t* lengths;
  int seqs, heads, group, kv_heads, dim, capacity, prefix_keys;
  float scale;
  int parts[2];                            // of the prefix, of a cache
  int columns[2];                          // workgroups that the columns of a part take
  unsigned prefix_blocks;                  // workgroups of the prefix, a multiple of eight
  bool spread;                             // of the prefix: a wavefront has columns of its own
  bool whole;                              // there is one part: o is written at once
  float* sums; float* values;              // [parts][seqs heads][2], [parts][seqs heads][dim]
};

// (64 numbers of fp32: two wavefronts a SIMD, 43 us in place of 64 for eight sequences of 20000, 2 heads; the second pass would take that room.)
template <int DTYPE, int DP, bool DIRECT>
__global__ __launch_bounds__(kThreads, DP == 64 ? 2 : kWavesOf<DTYPE>) void step_kernel(StepParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef Operand<DTYPE> O;
  constexpr int STEPS = DP / 16, BN = kTile<DTYPE>;
  static_assert(kKeys % (2 * BN) == 0, "whole tiles");
  __shared__ __attribute__((aligned(1024))) unsigned char even[kLds<DTYPE, DP>], odd[kLds<DTYPE, DP>];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // what this workgroup does: a part of the prefix for some columns, or a part of a cache
  // (products and memory side by side: groups of eight workgroups of the one and of the other in turn, while there are both)
  const unsigned own_blocks = gridDim.x - p.prefix_blocks, pairs = (p.prefix_blocks < own_blocks ? p.prefix_blocks : own_blocks) / 8;
  const unsigned eight = blockIdx.x / 8;
  unsigned block = blockIdx.x;
  bool shared;
  if (eight < 2 * pairs) {
    shared = eight % 2 == 0;
    block = eight / 2 * 8 + blockIdx.x % 8;
  } else {
    block -= pairs * 8;                                      // behind the pairs: what is left of the one, then of the other
    shared = block < p.prefix_blocks;
    if (!shared) block = blockIdx.x - p.prefix_blocks;
  }
  unsigned unit;
  int seq = 0, kv, part, first_column, keys;
  if (shared) {
    // those that read the same keys meet in an XCD
    const unsigned i = block / 8;
    unit = i / p.columns[0] * 8 + block % 8;
    if (unit >= (unsigned)(p.kv_heads * p.parts[0])) return;
    part = unit / p.kv_heads;
    kv = unit % p.kv_heads;
    first_column = (int)(i % p.columns[0]) * (p.spread ? kThreads / 2 : 32) + (p.spread ? wave * 32 : 0);
    keys = p.prefix_keys;
  } else {
    unit = block;
    first_column = (int)(unit % p.columns[1]) * 32;
    unit /= p.columns[1];
    kv = unit % p.kv_heads;
    unit /= p.kv_heads;
    seq = unit % p.seqs;
    part = unit / p.seqs;
    keys = p.lengths[seq];
    keys = keys < 0 ? 0 : keys > p.capacity ? p.capacity : keys;
  }
  const bool spread = shared && p.spread;
  const int all = shared ? p.seqs * p.group : p.group, column = first_column + (lane & 31);
  const bool valid = column < all;
  if (shared && valid) seq = column / p.group;
  const int head = kv * p.group + (shared ? column % p.group : column);
  const int64_t place = ((int64_t)(shared ? part : p.parts[0] + part) * p.seqs + seq) * p.heads + head;

  const int64_t tiles = ((int64_t)keys + kKeys - 1) / kKeys, run = (tiles + p.parts[!shared] - 1) / p.parts[!shared] * kKeys;
  const int from = (int)(part * run < keys ? part * run : keys), to = (int)(from + run < keys ? from + run : keys);
  const Cache& c = shared ? p.prefix : p.own;
  const int64_t of = shared ? 0 : seq;
  const HeadRows k{static_cast<const T*>(c.k) + of * c.k_seq + kv * c.k_head, c.k_stride};
  const HeadRows v{static_cast<const T*>(c.v) + of * c.v_seq + kv * c.v_head, c.v_stride};
  typename O::F q[STEPS];
  const T* q_row = static_cast<const T*>(p.q) + (valid ? seq * p.q_stride + head * p.q_head : 0);
#pragma unroll
  for (int s = 0; s < STEPS; ++s) q[s] = operand(load_part<DTYPE>(q_row, s, lane, valid ? p.dim : 0));
  const Reader<DTYPE, DP> read(lane);
  const float scale = exponent(p.scale);
  unsigned found = 0;                                        // keys that are not there are zeros: nothing has to be told apart in a first pass
  bool lost = false;
  Running<DP> a;
  const auto pass = [&](auto clean) {
    constexpr bool CLEAN = decltype(clean)::value;
    const auto again = [&](int j0) { return Scores<DTYPE, CLEAN>{k, j0, HeadRows{q_row, 0}, 0, 0, to - 1, lane, p.dim, lost}; };
    a = Running<DP>();
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) a.acc[t] = zero16();
    if (spread) {
      walk<DTYPE, DP, DIRECT>((lds_byte*)even, (lds_byte*)odd, k, v, from, to - 1, p.dim, [&](const lds_byte* tk, const lds_byte* tv, int j0) {
        attend<DTYPE, DP, BN / 32, CLEAN>(a, read, q, tk, tv, scale, lane, j0 + BN > to, 0, to - 1 - j0, found, again(j0), Quiet());
      });
      a.l += other_half(a.l);
    } else {
      walk_shared<DTYPE, DP, DIRECT>(even, odd, k, v, from, to - 1, p.dim, [&](const lds_byte* tk, const lds_byte* tv, int j0, const auto& bring) {
        attend<DTYPE, DP, 1, CLEAN>(a, read, q, tk, tv, scale, lane, j0 + 32 > to, 0, to - 1 - j0, found, again(j0), bring);
      });
      join_running<DTYPE, DP>(a, scale, wave, lane, even, odd);
    }
  };
  pass(No());
  const bool mine = valid && (spread || wave == 0);          // this wavefront has results
  if constexpr (O::PLANES > 1) {                             // pieces of what is not finite: again, with such numbers told apart
    if (any_of_workgroup(mine && not_finite(a.acc))) {
      pass(Yes());
      if (any_of_workgroup(found != 0)) add_what_is_seen<DTYPE, DP>(a.acc, v, from, to, 0, to - 1, lane, p.dim);
    }
  }
  if (!mine) return;
  const float l = a.l;
  if (p.whole) {
    store_column<DTYPE, DP>(a.acc, l == 0.f ? 0.f : 1.f / l, static_cast<T*>(p.o) + seq * p.o_stride + head * p.o_head, lane, p.dim);
  } else {
    if (lane < 32) *reinterpret_cast<f32x2*>(p.sums + place * 2) = f32x2{l == 0.f ? -__builtin_inff() : a.base, l};
    if (l != 0.f) store_column<LSAM_DTYPE_FP32, DP>(a.acc, 1.f, p.values + place * p.dim, lane, p.dim);
  }
}

// A workgroup for each sequence and head: a part's maximum and sum in each lane, found once; then its eight groups of 32 lanes, four columns a lane,
// weigh every eighth part.
template <int DTYPE>
__global__ __launch_bounds__(256) void join_kernel(StepParams p) {
  static_assert(2 * kMaxParts <= 128, "two parts a lane");
  __shared__ float weights[2 * kMaxParts], values[8][32][4];
  const int lane = threadIdx.x & 63, group = threadIdx.x >> 5, parts = p.parts[0] + p.parts[1];
  const int64_t at = blockIdx.x, all = (int64_t)p.seqs * p.heads;
  float m[2], sum[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int part = i * 64 + lane;
    const f32x2 v = part < parts ? *reinterpret_cast<const f32x2*>(p.sums + (part * all + at) * 2) : f32x2{-__builtin_inff(), 0.f};
    m[i] = v[0];
    sum[i] = v[1];
  }
  float most = __builtin_fmaxf(m[0], m[1]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) most = __builtin_fmaxf(most, __shfl_xor(most, d));
  const float base = most == -__builtin_inff() ? 0.f : most;
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float weight = sum[i] == 0.f ? 0.f : __builtin_amdgcn_exp2f(m[i] - base);      // no keys: its values were not written
    l += sum[i] * weight;
    if (threadIdx.x < 64) weights[i * 64 + lane] = sum[i] == 0.f ? -1.f : weight;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
  __syncthreads();
  const int col = (threadIdx.x & 31) * 4, n = p.dim - col < 4 ? p.dim - col : 4;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (n > 0) {
#pragma unroll 4
    for (int i = group; i < parts; i += 8) {
      const float weight = weights[i];
      const float* from = p.values + (i * all + at) * p.dim + col;
      if (weight == -1.f) continue;
      if (n == 4) {
        const f32x4 w = *reinterpret_cast<const f32x4_any*>(from);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += w[e] * weight;
      } else {
        for (int e = 0; e < n; ++e) v[e] += from[e] * weight;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) values[group][threadIdx.x & 31][e] = v[e];
  __syncthreads();
  if (threadIdx.x >= 32 || n <= 0) return;
#pragma unroll
  for (int g = 1; g < 8; ++g)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += values[g][threadIdx.x][e];
  typename Value<DTYPE>::T* o = static_cast<typename Value<DTYPE>::T*>(p.o) + at / p.heads * p.o_stride + at % p.heads * p.o_head + col;
  for (int e = 0; e < n; ++e) Value<DTYPE>::put(o + e, l == 0.f ? 0.f : v[e] / l);
}

// How keys are cut: about as many workgroups as two for each unit, of a tile of keys at least.
constexpr int kGroups = 512;
struct Plan { int parts[2], columns[2]; bool spread; unsigned prefix_blocks, blocks; size_t values_at, bytes; };
Plan plan(const lsam_attention_step_desc* d) {
  Plan c{};
  const int group = d->heads / d->kv_heads;
  const int64_t together = d->seqs * group;
  c.spread = together > 32;
  c.columns[0] = (int)(c.spread ? (together + kThreads / 2 - 1) / (kThreads / 2) : 1);
  c.columns[1] = (group + 31) / 32;
  const int64_t keys[2] = {d->prefix, d->capacity}, base[2] = {(int64_t)d->kv_heads * c.columns[0], d->seqs * d->kv_heads * c.columns[1]};
  for (int i = 0; i < 2; ++i) {
    int64_t parts = (kGroups + base[i] - 1) / base[i];
    const int64_t tiles = (keys[i] + kKeys - 1) / kKeys;
    parts = parts < tiles ? parts : tiles;
    c.parts[i] = (int)(parts < kMaxParts ? parts : kMaxParts);
  }
  c.prefix_blocks = (unsigned)(((int64_t)d->kv_heads * c.parts[0] + 7) / 8 * 8 * c.columns[0]);
  c.blocks = c.prefix_blocks + (unsigned)(base[1] * c.parts[1]);
  const int parts = c.parts[0] + c.parts[1];
  const size_t places = (size_t)parts * d->seqs * d->heads;
  if (parts > 1) {
    c.values_at = (places * 8 + 255) / 256 * 256;
    c.bytes = c.values_at + places * d->dim * 4;
  }
  return c;
}

int check(const lsam_attention_step_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype)) return refuse(LSAM_EINVAL, "%s: dtype %d is none of LSAM_DTYPE_*", who, d->dtype);
  if (d->kv_heads < 1 || d->heads < 1 || d->heads > 65536 || d->heads % d->kv_heads)
    return refuse(LSAM_EINVAL, "%s: heads must be a multiple of kv_heads, in 1..65536", who);
  if (d->dim < 1 || d->dim > LSAM_ATTENTION_MAX_DIM) return refuse(LSAM_EINVAL, "%s: dim must be in 1..%d", who, LSAM_ATTENTION_MAX_DIM);
  if (d->seqs < 0 || d->seqs >= 1 << 23 || d->seqs * d->heads >= 1 << 23) return refuse(LSAM_EINVAL, "%s: seqs times heads must be below 2^23", who);
  if (d->capacity < 0 || d->capacity >= 1 << 30 || d->prefix < 0 || d->prefix >= 1 << 30)
    return refuse(LSAM_EINVAL, "%s: capacity and prefix must be in 0..2^30-1", who);
  if (!(d->scale >= 0.f) || d->scale > LSAM_ATTENTION_MAX_SCALE) return refuse(LSAM_EINVAL, "%s: the scale must be in 0..2^100", who);
  return LSAM_OK;
}

// Rows that are only read, of any strides that are not negative.
Arg read_only(const lsam_attention_step_desc* d, const char* name, const void* p, int64_t seqs, int64_t seq, int64_t rows, const lsam_heads& t, int heads) {
  const int b = dtype_bytes(d->dtype);
  if (seqs == 0 || rows == 0) return Arg{name, p, 0, b, false};
  if (t.stride < 0 || t.head < 0 || (seqs > 1 && seq < 0)) return Arg{name, p, -1, b, false};
  const __int128 n = ((__int128)(seqs - 1) * (seqs > 1 ? seq : 0) + (__int128)(rows - 1) * t.stride + (__int128)(heads - 1) * t.head + d->dim) * b;
  return Arg{name, p, n < ((__int128)1 << 46) ? (int64_t)n : -1, b, false};
}

template <int DTYPE, int DP, bool DIRECT>
void launch(const StepParams& p, unsigned blocks, hipStream_t s) {
  if (blocks) step_kernel<DTYPE, DP, DIRECT><<<blocks, kThreads, 0, s>>>(p);
  if (!p.whole) join_kernel<DTYPE><<<(unsigned)(p.seqs * p.heads), 256, 0, s>>>(p);
}
template <int DTYPE, bool DIRECT>
void launch_wide(const StepParams& p, unsigned blocks, hipStream_t s) {
  if (p.dim <= 64) launch<DTYPE, 64, DIRECT>(p, blocks, s);
  else launch<DTYPE, 128, DIRECT>(p, blocks, s);
}

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" size_t lsam_attention_step_workspace_bytes(const lsam_attention_step_desc* d) {
  if (check(d, "attention_step") != LSAM_OK) return 0;
  return d->seqs ? plan(d).bytes : 0;
}

extern "C" int lsam_attention_step(const lsam_attention_step_desc* d, const int32_t* lengths, const void* q, const void* k, const void* v,
                                   const void* prefix_k, const void* prefix_v, void* o, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "attention_step";
  int rc = check(d, who);
  if (rc != LSAM_OK) return rc;
  if (d->seqs == 0) return LSAM_OK;
  const Plan c = plan(d);
  const int b = dtype_bytes(d->dtype);
  const Arg args[] = {read_only(d, "q", q, 1, 0, d->seqs, d->q, d->heads), read_only(d, "k", k, d->seqs, d->k_seq, d->capacity, d->k, d->kv_heads),
                      read_only(d, "v", v, d->seqs, d->v_seq, d->capacity, d->v, d->kv_heads),
                      read_only(d, "prefix_k", prefix_k, 1, 0, d->prefix, d->prefix_k, d->kv_heads),
                      read_only(d, "prefix_v", prefix_v, 1, 0, d->prefix, d->prefix_v, d->kv_heads),
                      {"lengths", lengths, d->seqs * 4, 4, false},
                      [&] {
                        if (d->heads > 1 && d->o.head >= d->dim && d->seqs > 1 && (__int128)d->o.stride >= (__int128)(d->heads - 1) * d->o.head + d->dim)
                          return matrices("o", o, 1, 0, d->seqs, d->o.stride, (d->heads - 1) * d->o.head + d->dim, b, true);
                        Arg a = matrices("o", o, d->heads, d->o.head, d->seqs, d->o.stride, d->dim, b, true);
                        if (!apart(d->heads, d->o.head, d->seqs, d->o.stride, d->dim)) a.bytes = -1;
                        return a;
                      }()};
  constexpr int n = sizeof args / sizeof args[0];
  rc = check_values(args, n, who);
  if (rc == LSAM_OK) rc = check_apart(args, n, who);
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, c.bytes, 16, who);
  if (rc != LSAM_OK) return rc;
  StepParams p{};
  p.prefix = Cache{prefix_k, prefix_v, d->prefix_k.stride, d->prefix_k.head, 0, d->prefix_v.stride, d->prefix_v.head, 0};
  p.own = Cache{k, v, d->k.stride, d->k.head, d->k_seq, d->v.stride, d->v.head, d->v_seq};
  p.q = q; p.o = o;
  p.q_stride = d->q.stride; p.q_head = d->q.head; p.o_stride = d->o.stride; p.o_head = d->o.head;
  p.lengths = lengths;
  p.seqs = (int)d->seqs; p.heads = d->heads; p.kv_heads = d->kv_heads; p.group = d->heads / d->kv_heads; p.dim = d->dim;
  p.capacity = (int)d->capacity; p.prefix_keys = (int)d->prefix; p.scale = d->scale;
  for (int i = 0; i < 2; ++i) { p.parts[i] = c.parts[i]; p.columns[i] = c.columns[i]; }
  p.prefix_blocks = c.prefix_blocks; p.spread = c.spread;
  p.whole = c.parts[0] + c.parts[1] == 1;
  p.sums = static_cast<float*>(workspace);
  p.values = reinterpret_cast<float*>(static_cast<char*>(workspace) + c.values_at);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto fits = [&](const void* t, const lsam_heads& h, int64_t seq) { return direct(t, h.stride, h.head, seq, d->dim, d->dtype); };
  const bool fast = (c.parts[0] == 0 || (fits(prefix_k, d->prefix_k, 0) && fits(prefix_v, d->prefix_v, 0))) &&
                    (c.parts[1] == 0 || (fits(k, d->k, d->k_seq) && fits(v, d->v, d->v_seq)));
  if (d->dtype == LSAM_DTYPE_FP32 && fast) launch_wide<LSAM_DTYPE_FP32, true>(p, c.blocks, s);
  else if (d->dtype == LSAM_DTYPE_FP32) launch_wide<LSAM_DTYPE_FP32, false>(p, c.blocks, s);
  else if (fast) launch_wide<LSAM_DTYPE_BF16, true>(p, c.blocks, s);
  else launch_wide<LSAM_DTYPE_BF16, false>(p, c.blocks, s);
  return launched();
}
