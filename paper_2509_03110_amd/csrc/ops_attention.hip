// lsam_attention, lsam_attention_backward: causal attention over packed sequences with grouped heads, and its gradient.
//
//   attention_kernel  o and lse.  A wavefront owns 32 rows of a head, a workgroup 128; it walks over the keys that they see in tiles, forms
//                     the scores of a tile with keys as rows and queries as columns (a lane's column is one query), keeps the running
//                     maximum and sum of each column, and adds the tile's part of o^T
//   dq_kernel         the same walk: scores and d_o v again, ds, dq^T; leaves d_o o and lse of each row for
//   dkv_kernel        a wavefront owns 32 keys, and walks over the rows that see them, head by head of the group: scores with queries as
//                     rows, dv^T and dk^T.  Where keys are few workgroups share a group's heads, and
//   join_kernel       adds their sums in their order: no atomics
//
// Both gradients form the scores again: 7 products in place of 5, for results that do not depend on timing.
//
// Rounded to bf16, for products of bf16 operands: p (o, dv) and ds (dq, dk), each by half a step at most and once.  Held in two pieces they would cost
// half the products again.  d_o o is that of o as it was stored: exact ones, sums of p d_o v, would cost dq_kernel a second walk.  Off from the definition in 64 bits,
// of the norm, at 2048, 256, 16 and 2 rows a sequence: o 2.1e-3, 1.9e-3, 1.7e-3, 1.1e-3; dq and dk 2.5e-3, 2.6e-3, 3.1e-3, 4.4e-3; dv 2.3e-3, 2.3e-3, 2.2e-3, 1.9e-3.  The
// rounding of what is stored is 1.7e-3 by itself.
//
// Bound by the vector unit beside the matrix unit, which is busy for 43 to 49 % of the time: exponentials, maxima and roundings of a tile take as long as
// its products, and the two of a wavefront do not overlap.  Four sequences of 4096, 16 heads of 128 over 4: 302 us forward (0.91 PFLOP/s), dq 428 us
// (0.96), dk and dv 648 us (0.85); together 1378 with a profiler attached, 1348 without.
#include "attention.h"

namespace lsam {
namespace {

// Rows of a workgroup: 32 a wavefront, or 32 that its wavefronts share.
template <bool SHARED> constexpr int kRowsOf = SHARED ? 32 : 32 * kThreads / 64;

struct Tensor { void* p; int64_t stride, head; };

struct AttentionParams {
  Tensor q, k, v, o, d_o, dq, dk, dv;
  Sequences seq;
  float* lse;
  f32x2* stats;                            // backward: [heads][padded]: lse as a power of 2, d_o o
  int64_t padded;                          // rows, and what a tile may reach past them
  int heads, group, dim, tiles;
  int parts, apiece;                       // dkv: workgroups that share the heads of a group, heads of one
  float* sums;                             // dkv of more than one: [dk, dv][parts][kv_heads][rows][dim]
  float scale;
};

// Which tile of rows and which head a workgroup has.  Workgroups go round the eight XCDs in turn: those that read the same keys
// meet in as few XCDs as that many heads allow.  `of`: heads of a group that are workgroups of their own.  The last tiles of a sequence see most
// keys and come first (last_first); the first keys are seen by most rows and come first, but every second round of an XCD's 32 units
// goes backwards: all workgroups are there at once, two to a unit, and a unit with a long one gets a short one.
struct Work { int tile, kv, g; bool here; };
__device__ __forceinline__ Work work(int tiles, int kv_heads, int of, bool last_first) {
  const unsigned common = kv_heads % 8 == 0 ? 8 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  const unsigned xcd = blockIdx.x % 8, i = blockIdx.x / 8, parts = 8 / common, mine = kv_heads / common;
  Work w;
  w.g = i % of;
  const unsigned rest = i / of;
  unsigned at = rest / mine;
  if (!last_first) {
    const unsigned all = (tiles + parts - 1) / parts, units = mine * of, round = units < 32 ? 32 / units : 1, from = at / round * round;
    if (at / round % 2) at = from + (from + round <= all ? round : all - from) - 1 - (at - from);
  }
  w.kv = (int)(rest % mine * common + xcd % common);
  w.tile = (int)(at * parts + xcd / common);
  w.here = w.tile < tiles;
  if (last_first) w.tile = tiles - 1 - w.tile;
  return w;
}
unsigned workgroups(int tiles, int kv_heads, int of) {
  const unsigned common = kv_heads % 8 == 0 ? 8 : kv_heads % 4 == 0 ? 4 : kv_heads % 2 == 0 ? 2 : 1;
  const unsigned parts = 8 / common, mine = kv_heads / common;
  return 8 * (((unsigned)tiles + parts - 1) / parts) * mine * of;
}

// What a wavefront's rows see (or are seen by): numbers lo .. hi altogether, all of them from all_lo to all_hi.  Both ends grow with the
// row, so the first and the last row that has a sequence tell.  Without any: lo behind everything, hi before it.
struct Range { int lo, hi, all_lo, all_hi; };
__device__ __forceinline__ Range range_of(bool valid, int first, int last) {
  const unsigned long long rows = __ballot(valid);
  if (!rows) return Range{0x7FFFFFFF, -1, 0x7FFFFFFF, -1};
  const int a = __builtin_ctzll(rows), b = 63 - __builtin_clzll(rows);      // (the upper half of the lanes has the same rows)
  const int low = a < 32 ? a : a - 32, high = b >= 32 ? b - 32 : b;
  return Range{__builtin_amdgcn_readlane(first, low), __builtin_amdgcn_readlane(last, high), __builtin_amdgcn_readlane(first, high),
               __builtin_amdgcn_readlane(last, low)};
}

template <int DTYPE>
__device__ __forceinline__ typename Value<DTYPE>::T* head_of(const Tensor& t, int head) { return static_cast<typename Value<DTYPE>::T*>(t.p) + head * t.head; }

// (64 numbers of fp32: two wavefronts a SIMD where rows are shared; the second pass would take that room, which the first does not need.)
template <int DTYPE, int DP, bool DIRECT, bool SHARED>
__global__ __launch_bounds__(kThreads, SHARED && DP == 64 ? 2 : kWavesOf<DTYPE>) void attention_kernel(AttentionParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef Operand<DTYPE> O;
  constexpr int BN = kTile<DTYPE>, STEPS = DP / 16;
  __shared__ __attribute__((aligned(1024))) unsigned char even[kLds<DTYPE, DP>], odd[kLds<DTYPE, DP>];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work(p.tiles, p.heads / p.group, p.group, true);
  if (!w.here) return;
  const int head = w.kv * p.group + w.g, row = w.tile * kRowsOf<SHARED> + (SHARED ? 0 : wave * 32) + (lane & 31);
  const int top = w.tile * kRowsOf<SHARED>, bottom = top + kRowsOf<SHARED> <= p.seq.rows ? top + kRowsOf<SHARED> - 1 : p.seq.rows - 1;
  typename O::F q[STEPS];                                    // on its way while sequences are looked for
  const T* q_row = head_of<DTYPE>(p.q, head) + (row <= bottom ? row : bottom) * p.q.stride;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) q[s] = operand(load_part<DTYPE>(q_row, s, lane, p.dim));
  const Span span = span_of(p.seq, row, top, bottom);
  const bool valid = span.end > 0;
  const int first = valid ? span.begin : 0x7FFFFFFF, last = valid ? row : -1;
  const Range r = range_of(valid, first, last);
  const int lo = span.top_begin, hi = bottom;
  const Reader<DTYPE, DP> read(lane);
  const float c = exponent(p.scale);
  const HeadRows k{head_of<DTYPE>(p.k, w.kv), p.k.stride}, v{head_of<DTYPE>(p.v, w.kv), p.v.stride};
  Running<DP> a;
  unsigned found = 0;
  bool lost = false;
  const auto pass = [&](auto clean) {
    constexpr bool CLEAN = decltype(clean)::value;
    const auto again = [&](int j0) { return Scores<DTYPE, CLEAN>{k, j0, HeadRows{head_of<DTYPE>(p.q, head), p.q.stride}, row, first, last, lane, p.dim, lost}; };
    a = Running<DP>();
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) a.acc[t] = zero16();
    if constexpr (SHARED) {
      walk_shared<DTYPE, DP, DIRECT>(even, odd, k, v, lo, hi, p.dim, [&](const lds_byte* tk, const lds_byte* tv, int j0, const auto& bring) {
        if (j0 > r.hi || j0 + 32 <= r.lo) return bring.neither();
        attend<DTYPE, DP, 1, CLEAN>(a, read, q, tk, tv, c, lane, j0 < r.all_lo || j0 + 31 > r.all_hi, first - j0, last - j0, found, again(j0), bring);
      });
      join_running<DTYPE, DP>(a, c, wave, lane, even, odd);
    } else {
      walk<DTYPE, DP, DIRECT>((lds_byte*)even, (lds_byte*)odd, k, v, lo, hi, p.dim, [&](const lds_byte* tk, const lds_byte* tv, int j0) {
        if (j0 > r.hi || j0 + BN <= r.lo) return;
        attend<DTYPE, DP, BN / 32, CLEAN>(a, read, q, tk, tv, c, lane, j0 < r.all_lo || j0 + BN - 1 > r.all_hi, first - j0, last - j0, found, again(j0), Quiet());
      });
      a.l += other_half(a.l);
    }
  };
  pass(No());
  const bool mine = valid && (!SHARED || wave == 0);         // this wavefront has results
  if (any_of_workgroup(mine && not_finite(a.acc))) {         // by a value that is seen, or by one that is not: again, telling them apart
    pass(Yes());
    if (any_of_workgroup(found != 0)) add_what_is_seen<DTYPE, DP>(a.acc, v, r.lo, r.hi + 1, first, last, lane, p.dim);
  }
  if (!mine) return;
  store_column<DTYPE, DP>(a.acc, 1.f / a.l, head_of<DTYPE>(p.o, head) + row * p.o.stride, lane, p.dim);
  if (p.lse && lane < 32) p.lse[(int64_t)head * p.seq.rows + row] = a.m * p.scale + __logf(a.l);
}

template <int DTYPE, int DP, int TILES, bool CLEAN>
__device__ __forceinline__ void dq_tile(f32x16 (&acc)[DP / 32], const Reader<DTYPE, DP>& read, const typename Operand<DTYPE>::F (&q)[DP / 16],
                                        const typename Operand<DTYPE>::F (&g)[DP / 16], const lds_byte* tk, const lds_byte* tv, float c, float base,
                                        float dot, int lane, bool masked, int first, int last, unsigned& found,
                                        const Scores<DTYPE, CLEAN>& again) {
  typedef Operand<DTYPE> O;
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    f32x16 s = zero16(), d = zero16();
    products<DP / 16, 2>([&](int n) { return Few<DTYPE, 2>{read.along(tk, i * 32, n), read.along(tv, i * 32, n)}; },
                         [&](int n, const Few<DTYPE, 2>& a) {
                           multiply_few<DTYPE, 2>(a, [&](int j) -> const typename O::F& { return j ? g[n] : q[n]; }, [&](int j) -> f32x16& { return j ? d : s; });
                         });
    again(s, i);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_exp2f(s[e] * c - base) * (d[e] - dot);
    if (masked) {
      const Seen seen(first, last, lane);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = seen(i, e) ? s[e] : 0.f;
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) multiply_across<DTYPE, DP, CLEAN>(acc, read, tk, i * 32 + t * 16, O::from(s, t, false), found);
  }
}

template <int DTYPE, int DP, bool DIRECT, bool SHARED>
__global__ __launch_bounds__(kThreads, kWavesOf<DTYPE>) void dq_kernel(AttentionParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef Operand<DTYPE> O;
  constexpr int BN = kTile<DTYPE>, STEPS = DP / 16;
  __shared__ __attribute__((aligned(1024))) unsigned char even[kLds<DTYPE, DP>], odd[kLds<DTYPE, DP>];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work(p.tiles, p.heads / p.group, p.group, true);
  if (!w.here) return;
  const int head = w.kv * p.group + w.g, row = w.tile * kRowsOf<SHARED> + (SHARED ? 0 : wave * 32) + (lane & 31);
  const int top = w.tile * kRowsOf<SHARED>, bottom = top + kRowsOf<SHARED> <= p.seq.rows ? top + kRowsOf<SHARED> - 1 : p.seq.rows - 1;
  typename O::F q[STEPS], g[STEPS];                          // on their way while sequences are looked for
  const int at = row <= bottom ? row : bottom;
  const T* q_row = head_of<DTYPE>(p.q, head) + at * p.q.stride;
  const T* g_row = head_of<DTYPE>(p.d_o, head) + at * p.d_o.stride;
  const T* o_row = head_of<DTYPE>(p.o, head) + at * p.o.stride;
  float dot = 0.f;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    q[s] = operand(load_part<DTYPE>(q_row, s, lane, p.dim));
    const typename Unit<DTYPE>::T d_o = load_part<DTYPE>(g_row, s, lane, p.dim), o = load_part<DTYPE>(o_row, s, lane, p.dim);
    g[s] = operand(d_o);
#pragma unroll
    for (int e = 0; e < 8; ++e) dot += number(o[e]) * number(d_o[e]);
  }
  dot += other_half(dot);
  const float base = p.lse[(int64_t)head * p.seq.rows + at] * kLog2e;
  const Span span = span_of(p.seq, row, top, bottom);
  const bool valid = span.end > 0;
  const int first = valid ? span.begin : 0x7FFFFFFF, last = valid ? row : -1;
  const Range r = range_of(valid, first, last);
  const int lo = span.top_begin, hi = bottom;
  const Reader<DTYPE, DP> read(lane);
  const float c = exponent(p.scale);
  if (valid && lane < 32 && (!SHARED || wave == 0)) p.stats[head * p.padded + row] = f32x2{base, dot};
  const HeadRows k{head_of<DTYPE>(p.k, w.kv), p.k.stride}, v{head_of<DTYPE>(p.v, w.kv), p.v.stride};
  unsigned found = 0;
  bool lost = false;
  f32x16 acc[DP / 32];
  const auto pass = [&](auto clean) {
    constexpr bool CLEAN = decltype(clean)::value;
    const auto again = [&](int j0) { return Scores<DTYPE, CLEAN>{k, j0, HeadRows{head_of<DTYPE>(p.q, head), p.q.stride}, row, first, last, lane, p.dim, lost}; };
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) acc[t] = zero16();
    if constexpr (SHARED) {
      walk_shared<DTYPE, DP, DIRECT>(even, odd, k, v, lo, hi, p.dim, [&](const lds_byte* tk, const lds_byte* tv, int j0, const auto& bring) {
        if (j0 > r.hi || j0 + 32 <= r.lo) return bring.neither();
        bring.both_next();
        dq_tile<DTYPE, DP, 1, CLEAN>(acc, read, q, g, tk, tv, c, base, dot, lane, j0 < r.all_lo || j0 + 31 > r.all_hi, first - j0, last - j0,
                                                      found, again(j0));
        bring.keys_read();
      });
      join_sums<DTYPE, DP>(acc, wave, lane, even, odd);
    } else {
      walk<DTYPE, DP, DIRECT>((lds_byte*)even, (lds_byte*)odd, k, v, lo, hi, p.dim, [&](const lds_byte* tk, const lds_byte* tv, int j0) {
        if (j0 > r.hi || j0 + BN <= r.lo) return;
        dq_tile<DTYPE, DP, BN / 32, CLEAN>(acc, read, q, g, tk, tv, c, base, dot, lane, j0 < r.all_lo || j0 + BN - 1 > r.all_hi, first - j0,
                                                            last - j0, found, again(j0));
      });
    }
  };
  pass(No());
  const bool mine = valid && (!SHARED || wave == 0);
  if (any_of_workgroup(mine && not_finite(acc))) {
    pass(Yes());
    if (any_of_workgroup(found != 0)) add_what_is_seen<DTYPE, DP>(acc, k, r.lo, r.hi + 1, first, last, lane, p.dim);
  }
  if (mine) store_column<DTYPE, DP>(acc, p.scale, head_of<DTYPE>(p.dq, head) + row * p.dq.stride, lane, p.dim);
}

// Rows of a tile of dkv_kernel, and its LDS: such tiles of q and d_o with lse and d_o o of their rows.
template <int DTYPE, bool SHARED> constexpr int kSeenRows = SHARED ? 32 * kSharing<DTYPE> : 32;
template <int DTYPE, int DP, bool SHARED> constexpr int kSeenLds = kSeenRows<DTYPE, SHARED> * (2 * Rows<DTYPE, DP>::BYTES + 8);

// What a wavefront of dkv_kernel has: its keys or where they are, its values, and the sums for them.
template <int DTYPE, int DP, bool IN_LDS> struct Keys {
  static constexpr bool LDS = IN_LDS;
  const lds_byte* at;
  typename Operand<DTYPE>::F k[LDS ? 1 : DP / 16];
  typename Operand<DTYPE>::F v[DP / 16];
  f32x16 dk[DP / 32], dv[DP / 32];
};

// A tile of rows: scores and d_o v; p and ds of them; dv and dk.
template <int DTYPE, int DP, bool CLEAN, bool IN_LDS>
__device__ __forceinline__ void dkv_tile(Keys<DTYPE, DP, IN_LDS>& w, const Reader<DTYPE, DP>& read, const lds_byte* tq, const lds_byte* tg,
                                         const lds_byte* stats, float c, int lane, bool masked, int first, int last, unsigned& found,
                                        const Scores<DTYPE, CLEAN>& again) {
  typedef Operand<DTYPE> O;
  typedef typename O::F F;
  typedef const __attribute__((address_space(3))) f32x4* quad_ptr;
  constexpr int T = DP / 32;
  f32x16 s = zero16(), d = zero16();
  if constexpr (IN_LDS)
    products<DP / 16, 2>([&](int n) { return Few<DTYPE, 3>{read.along(tq, 0, n), read.along(tg, 0, n), read.along(w.at, 0, n)}; },
                         [&](int n, const Few<DTYPE, 3>& a) {
                           s = O::multiply(0, a.f[0], a.f[2], s);
                           d = O::multiply(0, a.f[1], w.v[n], d);
                         });
  else
    products<DP / 16, 2>([&](int n) { return Few<DTYPE, 2>{read.along(tq, 0, n), read.along(tg, 0, n)}; },
                         [&](int n, const Few<DTYPE, 2>& a) {
                           multiply_few<DTYPE, 2>(a, [&](int j) -> const F& { return j ? w.v[n] : w.k[n]; }, [&](int j) -> f32x16& { return j ? d : s; });
                         });
  again(s, 0);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const lds_byte* const at = stats + (8 * g + 4 * (lane >> 5)) * 8;
    const f32x4 two[2] = {*reinterpret_cast<quad_ptr>(at), *reinterpret_cast<quad_ptr>(at + 16)};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[4 * g + e] = __builtin_amdgcn_exp2f(s[4 * g + e] * c - two[e / 2][e % 2 * 2]);
      d[4 * g + e] = s[4 * g + e] * (d[4 * g + e] - two[e / 2][e % 2 * 2 + 1]);
    }
  }
  if (masked) {
    const Seen seen(first, last, lane);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[e] = seen(0, e) ? s[e] : 0.f;
      d[e] = seen(0, e) ? d[e] : 0.f;
    }
  }
  F weight[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) weight[i] = O::from(i & 1 ? d : s, i / 2, !(i & 1));
  // dv then dk of rows 0 .. 15, dv then dk of rows 16 .. 31
  if constexpr (O::PRODUCTS == 1) {
    products<4 * T, kAhead>([&](int n) { return read.across(n / T & 1 ? tq : tg, n / (2 * T) * 16, n % T); },
                            [&](int n, const F& f) {
                              f32x16& to = n / T & 1 ? w.dk[n % T] : w.dv[n % T];
                              to = O::multiply(0, CLEAN ? O::clean(f, found) : f, weight[n / T], to);
                            });
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) multiply_across<DTYPE, DP, CLEAN>(i & 1 ? w.dk : w.dv, read, i & 1 ? tq : tg, i / 2 * 16, weight[i], found);
  }
}

// ROWS rows' lse and d_o o to LDS, 32 rows a wavefront.
template <int ROWS>
__device__ __forceinline__ void ask_stats(lds_byte* to, const AttentionParams& p, int head, int row0, int wave) {
  if (wave >= ROWS / 32) return;
  const __amdgpu_buffer_rsrc_t from = resource(p.stats + head * p.padded + row0 + wave * 32, 256);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(to + wave * 256), 4, (threadIdx.x & 63) * 4, 0, 0, 0);
}

// A tile of q, d_o and what goes with their rows.
template <int DTYPE, int DP, bool DIRECT, int ROWS> struct SeenStage {
  static constexpr int BYTES = ROWS * Rows<DTYPE, DP>::BYTES;
  Stage<DTYPE, DP, ROWS, kThreads, DIRECT> q, g;
  __device__ __forceinline__ void ask(lds_byte* to, const AttentionParams& p, int head, int row0, int limit, int wave) {
    q.p = head_of<DTYPE>(p.q, head);
    g.p = head_of<DTYPE>(p.d_o, head);
    q.ask(to, row0, limit);
    g.ask(to + BYTES, row0, limit);
    ask_stats<ROWS>(to + 2 * BYTES, p, head, row0, wave);
  }
  __device__ __forceinline__ void put(lds_byte* to) const {
    q.put(to);
    g.put(to + BYTES);
  }
};

// PARTS: the heads of a group may be shared by workgroups.  (Without it the wide kernel of 128 bf16 numbers takes 5 % less time: no other stores to find
// registers for.)
template <int DTYPE, int DP, bool DIRECT, bool SHARED, bool PARTS>
__device__ __forceinline__ void dkv(const AttentionParams& p) {
  typedef typename Value<DTYPE>::T T;
  // keys in LDS where registers are short; three pieces of 128 have no room there, but one wavefront a SIMD has registers
  constexpr bool IN_LDS = DTYPE == LSAM_DTYPE_BF16 && !SHARED;
  constexpr int BN = kSeenRows<DTYPE, SHARED>, STEPS = DP / 16, BYTES = BN * Rows<DTYPE, DP>::BYTES, EACH = 32 * Rows<DTYPE, DP>::BYTES;
  constexpr int LDS = kSeenLds<DTYPE, DP, SHARED>;
  __shared__ __attribute__((aligned(1024))) unsigned char even[LDS], odd[SHARED ? 16 : LDS], own[IN_LDS ? kRowsOf<SHARED> * Rows<DTYPE, DP>::BYTES : 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Work w = work(p.tiles, p.heads / p.group, PARTS ? p.parts : 1, false);
  if (!w.here) return;
  const int row = w.tile * kRowsOf<SHARED> + (SHARED ? 0 : wave * 32) + (lane & 31);
  const int top = w.tile * kRowsOf<SHARED>, bottom = top + kRowsOf<SHARED> <= p.seq.rows ? top + kRowsOf<SHARED> - 1 : p.seq.rows - 1;
  Keys<DTYPE, DP, IN_LDS> keys;
  if constexpr (IN_LDS) {
    Stage<DTYPE, DP, kRowsOf<SHARED>, kThreads, DIRECT> sk;
    sk.init(HeadRows{head_of<DTYPE>(p.k, w.kv), p.k.stride}, p.dim);
    sk.ask((lds_byte*)own, top, p.seq.rows);
    sk.put((lds_byte*)own);
    keys.at = (lds_byte*)own + wave * EACH;
  } else {
    const T* k_row = head_of<DTYPE>(p.k, w.kv) + (row <= bottom ? row : bottom) * p.k.stride;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) keys.k[s] = operand(load_part<DTYPE>(k_row, s, lane, p.dim));
  }
  const T* v_row = head_of<DTYPE>(p.v, w.kv) + (row <= bottom ? row : bottom) * p.v.stride;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) keys.v[s] = operand(load_part<DTYPE>(v_row, s, lane, p.dim));
  const Span span = span_of(p.seq, row, top, bottom);
  const bool valid = span.end > 0;
  const int first = valid ? row : 0x7FFFFFFF, last = valid ? span.end - 1 : -1;     // rows that see this key
  const Range r = range_of(valid, first, last);
  const int lo = top, hi = span.bottom_end - 1;
  const Reader<DTYPE, DP> read(lane);
  const float c = exponent(p.scale);
  SeenStage<DTYPE, DP, DIRECT, BN> stage;
  const int head0 = w.kv * p.group + (PARTS ? w.g * p.apiece : 0), behind = PARTS && (w.g + 1) * p.apiece < p.group ? head0 + p.apiece : (w.kv + 1) * p.group;
  stage.q.init(HeadRows{head_of<DTYPE>(p.q, head0), p.q.stride}, p.dim);
  stage.g.init(HeadRows{head_of<DTYPE>(p.d_o, head0), p.d_o.stride}, p.dim);
  unsigned found = 0;
  bool lost = false;
  const auto pass = [&](auto clean) {
    constexpr bool CLEAN = decltype(clean)::value;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) keys.dk[t] = keys.dv[t] = zero16();
    int head = head0;
    if constexpr (!SHARED) stage.ask((lds_byte*)even, p, head, lo, hi + 1, wave);
    for (int i0 = lo; head < behind;) {
#pragma unroll
      for (int b = 0; b < (SHARED ? 1 : 2); ++b) {
        lds_byte* const tq = (lds_byte*)(b ? odd : even);
        if constexpr (SHARED) stage.ask(tq, p, head, i0, hi + 1, wave);
        stage.put(tq);
        arrived();
        const int mine = SHARED ? wave : 0, now = i0 + mine * 32, of = head;
        i0 += BN;
        if (i0 > hi) { i0 = lo; ++head; }
        if (!SHARED && head < behind) stage.ask((lds_byte*)(b ? even : odd), p, head, i0, hi + 1, wave);
        if (mine < BN / 32 && now <= r.hi && now + 32 > r.lo)
          dkv_tile<DTYPE, DP, CLEAN, IN_LDS>(keys, read, tq + mine * EACH, tq + BYTES + mine * EACH, tq + 2 * BYTES + mine * 256, c, lane,
                                             now < r.all_lo || now + 31 > r.all_hi, first - now, last - now, found,
                                             Scores<DTYPE, CLEAN>{HeadRows{head_of<DTYPE>(p.q, of), p.q.stride}, now,
                                                                  HeadRows{head_of<DTYPE>(p.k, w.kv), p.k.stride}, row, first, last, lane, p.dim, lost});
        if constexpr (SHARED) __syncthreads();               // one tile at a time
        if (head == behind) break;
      }
    }
    if constexpr (SHARED) {
      static_assert(LDS >= 3 * DP * 32 * 4 || kSharing<DTYPE> == 2, "sums of three wavefronts");
      join_sums<DTYPE, DP>(keys.dv, wave, lane, even, even + 2 * DP * 32 * 4);
      __syncthreads();
      join_sums<DTYPE, DP>(keys.dk, wave, lane, even, even + 2 * DP * 32 * 4);
      __syncthreads();
    }
  };
  pass(No());
  const bool mine = valid && (!SHARED || wave == 0);
  if (any_of_workgroup(mine && (not_finite(keys.dk) || not_finite(keys.dv)))) {
    pass(Yes());
    if (any_of_workgroup(found != 0)) {
      for (int head = head0; head < behind; ++head) {
        add_what_is_seen<DTYPE, DP>(keys.dk, HeadRows{head_of<DTYPE>(p.q, head), p.q.stride}, r.lo, r.hi + 1, first, last, lane, p.dim);
        add_what_is_seen<DTYPE, DP>(keys.dv, HeadRows{head_of<DTYPE>(p.d_o, head), p.d_o.stride}, r.lo, r.hi + 1, first, last, lane, p.dim);
      }
    }
  }
  if (!mine) return;
  if (PARTS && p.parts > 1) {
    const int64_t kv_heads = p.heads / p.group, all = kv_heads * p.seq.rows, at = w.g * all + (int64_t)w.kv * p.seq.rows + row;
    store_column<LSAM_DTYPE_FP32, DP>(keys.dk, p.scale, p.sums + at * p.dim, lane, p.dim);
    store_column<LSAM_DTYPE_FP32, DP>(keys.dv, 1.f, p.sums + (p.parts * all + at) * p.dim, lane, p.dim);
  } else {
    store_column<DTYPE, DP>(keys.dk, p.scale, head_of<DTYPE>(p.dk, w.kv) + row * p.dk.stride, lane, p.dim);
    store_column<DTYPE, DP>(keys.dv, 1.f, head_of<DTYPE>(p.dv, w.kv) + row * p.dv.stride, lane, p.dim);
  }
}

template <int DTYPE, int DP, bool DIRECT, bool SHARED, bool PARTS>
__global__ __launch_bounds__(kThreads, SHARED ? 1 : kWavesOf<DTYPE>) void dkv_kernel(AttentionParams p) { dkv<DTYPE, DP, DIRECT, SHARED, PARTS>(p); }

// The sums of the workgroups that share a group's heads, in their order: a few rows of a head of keys a workgroup, four columns a lane.
constexpr int kJoinRows = 8;
template <int DTYPE>
__global__ __launch_bounds__(256) void join_kernel(AttentionParams p) {
  typedef typename Value<DTYPE>::T T;
  const unsigned kv_heads = p.heads / p.group;
  const int kv = blockIdx.x % kv_heads, top = blockIdx.x / kv_heads * kJoinRows, lane = threadIdx.x & 63;
  const int bottom = top + kJoinRows <= p.seq.rows ? top + kJoinRows - 1 : p.seq.rows - 1;
  const int row = top + lane % kJoinRows;
  const Span span = span_of(p.seq, row, top, bottom);        // by all lanes
  const unsigned long long valid = __ballot(row <= bottom && span.end > 0);
  const unsigned pieces = (p.dim + 3) / 4;
  const int64_t all = (int64_t)kv_heads * p.seq.rows * p.dim;
  for (unsigned i = threadIdx.x; i < 2 * kJoinRows * pieces; i += 256) {
    const unsigned line = i / pieces, local = line % kJoinRows;
    const int col = (int)(i - line * pieces) * 4, n = p.dim - col < 4 ? p.dim - col : 4;
    if (!(valid >> local & 1)) continue;
    const bool of_v = line >= kJoinRows;
    const float* from = p.sums + (of_v ? p.parts * all : 0) + ((int64_t)kv * p.seq.rows + top + local) * p.dim + col;
    const Tensor& t = of_v ? p.dv : p.dk;
    T* to = head_of<DTYPE>(t, kv) + (top + local) * t.stride + col;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    if (n == 4) {
      for (int part = 0; part < p.parts; ++part) sum += *reinterpret_cast<const f32x4_any*>(from + part * all);
    } else {
      for (int part = 0; part < p.parts; ++part)
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (e < n) sum[e] += from[part * all + e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) Value<DTYPE>::put(to + e, sum[e]);
  }
}

int check(const lsam_attention_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype)) return refuse(LSAM_EINVAL, "%s: dtype %d is none of LSAM_DTYPE_*", who, d->dtype);
  if (d->kv_heads < 1 || d->heads < 1 || d->heads > 65536 || d->heads % d->kv_heads)
    return refuse(LSAM_EINVAL, "%s: heads must be a multiple of kv_heads, in 1..65536", who);
  if (d->dim < 1 || d->dim > LSAM_ATTENTION_MAX_DIM) return refuse(LSAM_EINVAL, "%s: dim must be in 1..%d", who, LSAM_ATTENTION_MAX_DIM);
  if (d->seqs < 0 || d->seqs >= 1ll << 31) return refuse(LSAM_EINVAL, "%s: seqs must be in 0..2^31-1", who);
  if (d->rows < 0 || d->rows >= 1 << 30 || d->rows * d->heads >= 1 << 30)
    return refuse(LSAM_EINVAL, "%s: rows times heads must be below 2^30", who);      // launches of less than 2^32 lanes
  if (!(d->scale >= 0.f) || d->scale > LSAM_ATTENTION_MAX_SCALE) return refuse(LSAM_EINVAL, "%s: the scale must be in 0..2^100", who);
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
  p.padded = (d->rows + 191) / 64 * 64;
  return p;
}

// Wavefronts share rows where workgroups of 128 rows would leave units without work (us, forward and backward, heads of 128 bf16 numbers, shared against
// not: 1024 rows of 16 heads, 128 such workgroups, 21 and 68 against 26 and 78; 1024 rows of 32 heads, 256 of them, 34 and 120 against 27 and 83).  The heads of a
// group are shared where the workgroups for keys are fewer than kPerUnit a unit (4096 rows, 32 heads of 8: backward 571 us, with one workgroup for
// a group's heads 740).
constexpr int kUnits = 256, kPerUnit = 2;
// Workgroups for keys: of 128 or of 32 keys, and how many share the heads of a group.
struct OfKeys { bool share; int tiles, parts, apiece; };
OfKeys of_keys(int64_t rows, int kv_heads, int group) {
  const int64_t wide = (rows + kRowsOf<false> - 1) / kRowsOf<false>, narrow = (rows + kRowsOf<true> - 1) / kRowsOf<true>;
  OfKeys c;
  c.share = wide * kv_heads < kUnits;
  c.tiles = (int)(c.share ? narrow : wide);
  const int64_t all = (int64_t)c.tiles * kv_heads, want = all > 0 ? (kPerUnit * kUnits + all - 1) / all : 1;
  c.apiece = want < group ? (int)((group + want - 1) / want) : 1;
  c.parts = (group + c.apiece - 1) / c.apiece;
  return c;
}
size_t stats_bytes(const AttentionParams& p) { return ((size_t)p.heads * p.padded * 8 + 255) / 256 * 256; }

template <int DTYPE, int DP, bool DIRECT>
int launch(AttentionParams p, bool backward, hipStream_t s) {
  const int rows = p.seq.rows, kv = p.heads / p.group, wide = (rows + kRowsOf<false> - 1) / kRowsOf<false>, narrow = (rows + kRowsOf<true> - 1) / kRowsOf<true>;
  const bool share = (int64_t)wide * p.heads < kUnits;
  p.tiles = share ? narrow : wide;
  const unsigned all = workgroups(p.tiles, kv, p.group);
  if (!backward) {
    if (share) attention_kernel<DTYPE, DP, DIRECT, true><<<all, kThreads, 0, s>>>(p);
    else attention_kernel<DTYPE, DP, DIRECT, false><<<all, kThreads, 0, s>>>(p);
    return launched();
  }
  if (share) dq_kernel<DTYPE, DP, DIRECT, true><<<all, kThreads, 0, s>>>(p);
  else dq_kernel<DTYPE, DP, DIRECT, false><<<all, kThreads, 0, s>>>(p);
  const OfKeys c = of_keys(rows, kv, p.group);
  p.tiles = c.tiles;
  p.parts = c.parts;
  p.apiece = c.apiece;
  const unsigned groups = workgroups(c.tiles, kv, c.parts);
  if (c.share) dkv_kernel<DTYPE, DP, DIRECT, true, true><<<groups, kThreads, 0, s>>>(p);
  else if (c.parts > 1) dkv_kernel<DTYPE, DP, DIRECT, false, true><<<groups, kThreads, 0, s>>>(p);
  else dkv_kernel<DTYPE, DP, DIRECT, false, false><<<groups, kThreads, 0, s>>>(p);
  if (c.parts > 1) join_kernel<DTYPE><<<(unsigned)((rows + kJoinRows - 1) / kJoinRows * kv), 256, 0, s>>>(p);
  return launched();
}
template <int DTYPE, bool DIRECT>
int launch_wide(const AttentionParams& p, bool backward, hipStream_t s) {
  if (p.dim <= 32) return launch<DTYPE, 32, DIRECT>(p, backward, s);
  if (p.dim <= 64) return launch<DTYPE, 64, DIRECT>(p, backward, s);
  if (p.dim <= 96) return launch<DTYPE, 96, DIRECT>(p, backward, s);
  return launch<DTYPE, 128, DIRECT>(p, backward, s);
}
int launch_any(const AttentionParams& p, int dtype, bool backward, hipStream_t s) {
  const auto fits = [&](const Tensor& t) { return direct(t.p, t.stride, t.head, 0, p.dim, dtype); };
  const bool fast = fits(p.k) && fits(p.v) && (!backward || (fits(p.q) && fits(p.d_o)));
  if (dtype == LSAM_DTYPE_BF16) return fast ? launch_wide<LSAM_DTYPE_BF16, true>(p, backward, s) : launch_wide<LSAM_DTYPE_BF16, false>(p, backward, s);
  return fast ? launch_wide<LSAM_DTYPE_FP32, true>(p, backward, s) : launch_wide<LSAM_DTYPE_FP32, false>(p, backward, s);
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
  const OfKeys c = of_keys(d->rows, d->kv_heads, p.group);
  return stats_bytes(p) + (c.parts > 1 ? (size_t)2 * c.parts * d->kv_heads * d->rows * d->dim * 4 : 0);
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
  p.lse = const_cast<float*>(lse); p.stats = static_cast<f32x2*>(workspace);
  p.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + stats_bytes(p));
  return launch_any(p, d->dtype, true, static_cast<hipStream_t>(stream));
}
