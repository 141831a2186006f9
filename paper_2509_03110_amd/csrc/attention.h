// What the attention kernels share: operands of the matrix units, tiles of rows in LDS, and which rows see which.
//
// Products are 32 x 32 results over 16 numbers at a time.  A lane's part of a result is one column (lane % 32) and sixteen rows, 8 (r / 4) +
// 4 (lane / 32) + r % 4.  Its eight numbers of an operand may be any eight of the sixteen as long as both operands agree, so
// results r = 8 t .. 8 t + 7 are, as they lie, the operand of a next product that sums over rows 16 t .. 16 t + 15: probabilities go from
// one product into the next without leaving the lane.
#pragma once
#include "ops.h"
#include "planes.h"

namespace lsam {

#if defined(__HIPCC__)

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

template <int DTYPE> struct Operand;
template <> struct Operand<LSAM_DTYPE_BF16> {
  typedef bf16x8 F;
  static constexpr int PLANES = 1;
  static constexpr int PRODUCTS = 1;
  // Product i of PRODUCTS that make a b.
  static __device__ __forceinline__ f32x16 multiply(int, const F& a, const F& b, const f32x16& c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  // Results 8 t .. of a product as an operand of the next; `weights`: none is above 2^9.
  static __device__ __forceinline__ F from(const f32x16& s, int t, bool weights) {
    F f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = static_cast<__bf16>(s[8 * t + e]);
    return f;
  }
  // 0 in place of what is not finite, whose sign bits come into `found`.
  static __device__ __forceinline__ F clean(F f, unsigned& found) {
    u32x4 w = __builtin_bit_cast(u32x4, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned top = ((w[i] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;      // an exponent of ones carries into the sign's place
      found |= top;
      w[i] &= ~(top | (top - (top >> 15)));
    }
    return __builtin_bit_cast(F, w);
  }
  static __device__ __forceinline__ F set(const u32x4 (&w)[1]) { return __builtin_bit_cast(F, w[0]); }
};
// An fp32 number is three bfloat16 pieces, h + m + l, which hold all its digits; of their nine products the six that fp32 can tell
// from 0 are formed, the smallest first: l h, m m, h l, m h, h m, h h.  Six products of 32 cycles against eight of 64 of the fp32 unit over the same
// sixteen numbers.
template <> struct Operand<LSAM_DTYPE_FP32> {
  typedef Operand<LSAM_DTYPE_BF16> One;
  struct F { bf16x8 p[3]; };
  static constexpr int PLANES = 3;
  static constexpr int PRODUCTS = 6;
  static __device__ __forceinline__ f32x16 multiply(int i, const F& a, const F& b, const f32x16& c) {
    constexpr int left[6] = {2, 1, 0, 1, 0, 0}, right[6] = {0, 1, 2, 0, 1, 0};
    return One::multiply(0, a.p[left[i]], b.p[right[i]], c);
  }
  static __device__ __forceinline__ F split(const float (&v)[8], bool weights) {
    unsigned w[3][4];
    float most = 0.f;
    if (!weights) {
#pragma unroll
      for (int e = 0; e < 8; ++e) most = largest_of(most, v[e]);
    }
    if (__any(past_rounding(most))) split_words_any<3, 8>(v, w);
    else split_words<3, 8>(v, w);
    F f;
#pragma unroll
    for (int q = 0; q < 3; ++q) f.p[q] = __builtin_bit_cast(bf16x8, u32x4{w[q][0], w[q][1], w[q][2], w[q][3]});
    return f;
  }
  static __device__ __forceinline__ F from(const f32x16& s, int t, bool weights) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[8 * t + e];
    return split(v, weights);
  }
  static __device__ __forceinline__ F clean(const F& f, unsigned& found) { return F{One::clean(f.p[0], found), One::clean(f.p[1], found), One::clean(f.p[2], found)}; }
  static __device__ __forceinline__ F set(const u32x4 (&w)[3]) {
    return F{__builtin_bit_cast(bf16x8, w[0]), __builtin_bit_cast(bf16x8, w[1]), __builtin_bit_cast(bf16x8, w[2])};
  }
};

// Rows of DP numbers in LDS, in units of eight bfloat16 numbers, of fp32 numbers the pieces one behind the other.  A unit's place in its row goes
// by the row, so that neither sixteen lanes that read the same unit of sixteen rows nor sixteen that read 32 bytes of four rows meet in a bank.
template <int DTYPE, int DP>
struct Rows {
  static constexpr int WIDE = DP > 64 ? 128 : 64, U = WIDE / 8, PLANE = WIDE * 2, BYTES = PLANE * Operand<DTYPE>::PLANES;
  static __device__ __forceinline__ int turn(int row) {
    if constexpr (U == 16) return (row & 3) << 2 | (row >> 2 & 3);
    else return (row >> 1 & 1) << 2 | (row >> 2 & 3);
  }
  static __device__ __forceinline__ int place(int row, int unit) { return row * BYTES + ((unit ^ turn(row)) << 4); }
};

// A lane's places in a tile of rows, found once: what is read from a tile whose address is known when this is compiled takes an
// offset beside them and no arithmetic.
template <int DTYPE, int DP> struct Reader {
  typedef Rows<DTYPE, DP> R;
  typedef Operand<DTYPE> O;
  typedef typename O::F F;
  unsigned row[DP / 16], column[DP / 32][2];
  __device__ __forceinline__ Reader(int lane) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) row[s] = R::place(lane & 31, s * 2 + (lane >> 5));
    // sixteen lanes read four rows of sixteen columns, four columns a lane, and each gets a column
    const int r = (lane >> 5) * 4 + (lane >> 2 & 3), col = (lane & 16) + (lane & 3) * 4;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) column[t][i] = R::place(r + 8 * i, t * 4 + (col >> 3)) + (col & 7) * 2;
  }
  // Row row0 + lane % 32, numbers 16 step + 8 (lane / 32) .. + 7.
  __device__ __forceinline__ F along(const lds_byte* tile, int row0, int step) const {
    u32x4 w[O::PLANES];
#pragma unroll
    for (int q = 0; q < O::PLANES; ++q)
      w[q] = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(tile + row0 * R::BYTES + row[step] + q * R::PLANE);
    return O::set(w);
  }
  // Column 32 t + lane % 32, rows row0 + 4 (lane / 32) + 0 .. 3 and 8 further: the rows of a lane's results.
  __device__ __forceinline__ F across(const lds_byte* tile, int row0, int t) const {
    typedef __attribute__((address_space(3))) s16x4* quad_ptr;
    u32x4 w[O::PLANES];
#pragma unroll
    for (int q = 0; q < O::PLANES; ++q) {
      lds_byte* const p = const_cast<lds_byte*>(tile) + row0 * R::BYTES + q * R::PLANE;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((quad_ptr)(p + column[t][0]));
      const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((quad_ptr)(p + column[t][1]));
      w[q] = __builtin_bit_cast(u32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    return O::set(w);
  }
};

// Rows of a tensor for one head.
struct HeadRows { const void* p; int64_t stride; };

// Eight numbers of a row from unit u on, as they are stored; numbers behind `dim` count as 0.
template <int DTYPE> struct Unit;
template <> struct Unit<LSAM_DTYPE_BF16> { typedef u16x8 T; typedef u16x8_any Any; };
typedef f32x8 f32x8_any __attribute__((aligned(4)));
template <> struct Unit<LSAM_DTYPE_FP32> { typedef f32x8 T; typedef f32x8_any Any; };
template <int DTYPE>
__device__ __forceinline__ typename Unit<DTYPE>::T load_unit(const typename Value<DTYPE>::T* row, int u, int dim) {
  const int n = dim - u * 8;
  typename Unit<DTYPE>::T v;
  if (n >= 8) {
    v = *reinterpret_cast<const typename Unit<DTYPE>::Any*>(row + u * 8);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0;
    if (n > 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < n) v[e] = row[u * 8 + e];
    }
  }
  return v;
}
__device__ __forceinline__ Operand<LSAM_DTYPE_BF16>::F operand(u16x8 v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ Operand<LSAM_DTYPE_FP32>::F operand(f32x8 v) {
  const float x[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  return Operand<LSAM_DTYPE_FP32>::split(x, false);
}
__device__ __forceinline__ float number(unsigned short v) { return widen(v); }
__device__ __forceinline__ float number(float v) { return v; }
// A lane's part of a row in memory: numbers 16 step + 8 (lane / 32) .. + 7.
template <int DTYPE>
__device__ __forceinline__ typename Unit<DTYPE>::T load_part(const typename Value<DTYPE>::T* row, int step, int lane, int dim) {
  return load_unit<DTYPE>(row, step * 2 + (lane >> 5), dim);
}

// The bytes behind p, the same in all lanes.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const void* p, unsigned bytes) {
  const unsigned long long a = reinterpret_cast<unsigned long long>(p);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a), hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((unsigned long long)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// A workgroup's way of bringing ROWS rows into LDS; rows from `limit` on count as 0.  Whole units of eight numbers (DIRECT): bf16 rows go there
// without passing through registers, asked for a tile ahead, there when the wavefront has waited for its loads; fp32 rows pass through them, where
// they are cut into pieces, but no load waits for another and none is in a branch.  Other rows are looked at number by number.
template <int DTYPE, int DP, int ROWS, int THREADS, bool DIRECT>
struct Stage {
  typedef typename Value<DTYPE>::T T;
  typedef Rows<DTYPE, DP> R;
  static constexpr int N = ROWS * R::U / THREADS, PLANES = Operand<DTYPE>::PLANES, B = sizeof(T);
  static constexpr bool THROUGH = !DIRECT || PLANES > 1;     // registers
  static_assert(N * THREADS == ROWS * R::U, "whole rounds of loads");
  const T* p;
  int64_t stride;
  int dim;
  typename Unit<DTYPE>::T w[THROUGH ? N : 1];
  unsigned at[DIRECT ? N : 1];
  __device__ __forceinline__ void init(const HeadRows& t, int d) {
    p = static_cast<const T*>(t.p);
    stride = t.stride;
    dim = d;
    if constexpr (DIRECT) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x % THREADS + i * THREADS, row = n / R::U, unit = THROUGH ? n % R::U : (n % R::U) ^ R::turn(row);
        at[i] = unit * 8 < dim ? (unsigned)(row * stride * B) + unit * 8 * B : 0x7FFFFFC0u;
      }
    }
  }
  __device__ __forceinline__ void ask(lds_byte* tile, int64_t row0, int64_t limit) {
    if constexpr (DIRECT) {
      const int64_t rows = limit - row0 < ROWS ? limit - row0 : ROWS;
      const __amdgpu_buffer_rsrc_t from = resource(p + row0 * stride, rows > 0 ? (unsigned)(((rows - 1) * stride + dim) * B) : 0);
      const int wave = THREADS > 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (THROUGH) {
          const u32x4 a = __builtin_amdgcn_raw_buffer_load_b128(from, at[i], 0, 0), b = __builtin_amdgcn_raw_buffer_load_b128(from, at[i] + 16, 0, 0);
          w[i] = __builtin_bit_cast(typename Unit<DTYPE>::T, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
          __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(tile + (wave * 64 + i * THREADS) * 16), 16, at[i], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + i * THREADS, row = n / R::U;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[i][e] = 0;
        if (row0 + row < limit) w[i] = load_unit<DTYPE>(p + (row0 + row) * stride, n % R::U, dim);
      }
    }
  }
  __device__ __forceinline__ void put(lds_byte* tile) const {
    if constexpr (THROUGH) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + i * THREADS;
        const typename Operand<DTYPE>::F f = operand(w[i]);
        const bf16x8* pieces = reinterpret_cast<const bf16x8*>(&f);
#pragma unroll
        for (int q = 0; q < PLANES; ++q)
          *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(tile + R::place(n / R::U, n % R::U) + q * R::PLANE) = __builtin_bit_cast(u32x4, pieces[q]);
      }
    }
  }
};
// Waits for all but the last N of the wavefront's own loads.
template <int N> __device__ __forceinline__ void all_but() {
  static_assert(N < 16, "");
  __builtin_amdgcn_s_waitcnt(0x0F70 + N);
  asm volatile("" ::: "memory");
}
// Waits for the wavefront's own reads of LDS.
__device__ __forceinline__ void lds_read() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);
  asm volatile("" ::: "memory");
}
// Waits for the wavefront's own loads, and for the other wavefronts.
__device__ __forceinline__ void arrived() {
  __builtin_amdgcn_s_waitcnt(0x0070);                      // no load on its way, no LDS access
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Whether rows are whole units, a tile within 32-bit offsets, and rows behind the last one behind its bytes too, where loads give 0; bf16 ones have to be
// aligned to go to LDS directly.
inline bool direct(const void* p, int64_t stride, int64_t head, int64_t seq, int dim, int dtype) {
  if (dim % 8 || stride < dim || stride >= 1 << 20) return false;
  return dtype == LSAM_DTYPE_FP32 || (!misaligned(p, 16) && stride % 8 == 0 && head % 8 == 0 && seq % 8 == 0);
}

constexpr float kLog2e = 1.4426950408889634f;
// Scores as powers of 2; above 0, since 0 times the -inf of a masked score is not -inf.
__device__ __forceinline__ float exponent(float scale) { return __builtin_fmaxf(scale * kLog2e, 0x1p-126f); }

__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
// The row of a lane's result r.
__device__ __forceinline__ int result_row(int r, int lane) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }

// Several products at once: none waits for the one before it.
template <int DTYPE, int N> struct Few { typename Operand<DTYPE>::F f[N]; };
template <int DTYPE, int N, typename To, typename With>
__device__ __forceinline__ void multiply_few(const Few<DTYPE, N>& a, With with, To to) {
#pragma unroll
  for (int i = 0; i < Operand<DTYPE>::PRODUCTS; ++i)
#pragma unroll
    for (int n = 0; n < N; ++n) to(n) = Operand<DTYPE>::multiply(i, a.f[n], with(n), to(n));
}

// N products whose operand from LDS is asked for AHEAD products before: a wavefront's registers do not hold more than that of
// them, and vector arithmetic may move in between.  `beside(n)` is work of the vector units for the time that product n takes.
template <int N, int AHEAD, typename Load, typename Use, typename Beside>
__device__ __forceinline__ void products(Load load, Use use, Beside beside) {
  decltype(load(0)) ring[AHEAD];
#pragma unroll
  for (int n = 0; n < AHEAD && n < N; ++n) ring[n] = load(n);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    use(n, ring[n % AHEAD]);
    if (n + AHEAD < N) ring[n % AHEAD] = load(n + AHEAD);
    beside(n);
    __builtin_amdgcn_sched_barrier(0x0406);
  }
}
template <int N, int AHEAD, typename Load, typename Use>
__device__ __forceinline__ void products(Load load, Use use) { products<N, AHEAD>(load, use, [](int) {}); }
constexpr int kAhead = 3;

// acc += tile^T p over the 16 rows from row0 on, p a lane's column.  A column that does not see a row has p = 0 there, but 0 times infinity is not 0:
// with CLEAN what is not finite counts as 0 and is `found`, and add_what_is_seen() brings it to the columns that see it.
template <int DTYPE, int DP, bool CLEAN>
__device__ __forceinline__ void multiply_across(f32x16 (&acc)[DP / 32], const Reader<DTYPE, DP>& read, const lds_byte* tile, int row0,
                                                typename Operand<DTYPE>::F p, unsigned& found) {
  typedef Operand<DTYPE> O;
  if constexpr (O::PRODUCTS == 1) {
    products<DP / 32, kAhead>([&](int t) { return read.across(tile, row0, t); },
                              [&](int t, const typename O::F& a) { acc[t] = O::multiply(0, CLEAN ? O::clean(a, found) : a, p, acc[t]); });
  } else {
    Few<DTYPE, DP / 32> a;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) {
      a.f[t] = read.across(tile, row0, t);
      if constexpr (CLEAN) a.f[t] = O::clean(a.f[t], found);
    }
    multiply_few<DTYPE, DP / 32>(a, [&](int) -> const typename O::F& { return p; }, [&](int t) -> f32x16& { return acc[t]; });
  }
}
// Whether a lane's sums hold what is not finite.
template <int N>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[N]) {
  bool bad = false;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) bad |= !__builtin_isfinite(acc[t][r]);
  return bad;
}
// Adds what is not finite in rows from .. to - 1 to the lanes' columns that see the row, first .. last.  Where it was multiplied
// already, the sum is not finite either way.
template <int DTYPE, int DP>
__device__ __forceinline__ void add_what_is_seen(f32x16 (&acc)[DP / 32], const HeadRows& rows, int from, int to, int first, int last, int lane, int dim) {
#pragma unroll 1
  for (int j = from; j < to; ++j) {
    const typename Value<DTYPE>::T* row = static_cast<const typename Value<DTYPE>::T*>(rows.p) + j * rows.stride;
    const bool seen = j >= first && j <= last;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = t * 32 + result_row(r, lane);
        const float v = d < dim ? Value<DTYPE>::get(row + d) : 0.f;
        if (seen && !__builtin_isfinite(v)) acc[t][r] += v;
      }
  }
}

// factor times a lane's column of results to a row in memory.
template <int DTYPE, int DP>
__device__ __forceinline__ void store_column(const f32x16 (&acc)[DP / 32], float factor, typename Value<DTYPE>::T* row, int lane, int dim) {
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = t * 32 + g * 8 + (lane >> 5) * 4;
      if (d + 4 <= dim) {
        if constexpr (DTYPE == LSAM_DTYPE_BF16) {
          u16x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = narrow(acc[t][4 * g + e] * factor);
          *reinterpret_cast<u16x4_any*>(row + d) = w;
        } else {
          f32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = acc[t][4 * g + e] * factor;
          *reinterpret_cast<f32x4_any*>(row + d) = w;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (d + e < dim) Value<DTYPE>::put(row + d + e, acc[t][4 * g + e] * factor);
      }
    }
}

// What the other half of a wavefront holds in the same column.
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// ---- a walk over keys -----------------------------------------------------------------------------------
constexpr int kThreads = 256;              // of a workgroup
template <int DTYPE> constexpr int kWavesOf = DTYPE == LSAM_DTYPE_BF16 ? 2 : 1;    // of a SIMD
template <int DTYPE> constexpr int kTile = DTYPE == LSAM_DTYPE_BF16 ? 64 : 32;      // rows of a tile in LDS
template <int DTYPE, int DP> constexpr int kLds = 2 * kTile<DTYPE> * Rows<DTYPE, DP>::BYTES;   // a tile of two tensors

struct No { static constexpr bool value = false; };
struct Yes { static constexpr bool value = true; };

// Whether a lane of the workgroup says so.
__device__ __forceinline__ bool any_of_workgroup(bool v) {
  __shared__ int shared[kThreads / 64];
  const bool mine = __any(v);
  __syncthreads();                                           // an answer before has been read
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = mine;
  __syncthreads();
  bool all = false;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) all |= shared[i] != 0;
  return all;
}

// Keys lo .. hi in tiles, `f(tile of k, tile of v, first key)` for each.  Two tiles a turn in arrays of their own: so the compiler sees that what is
// read is not what is on its way, and their places are constants.
template <int DTYPE, int DP, bool DIRECT, typename F>
__device__ __forceinline__ void walk(lds_byte* even, lds_byte* odd, const HeadRows& k, const HeadRows& v, int lo, int hi, int dim, F f) {
  constexpr int BN = kTile<DTYPE>, BYTES = BN * Rows<DTYPE, DP>::BYTES;
  if (lo > hi) return;                                      // nothing is asked for that nothing waits for
  Stage<DTYPE, DP, BN, kThreads, DIRECT> sk, sv;
  sk.init(k, dim);
  sv.init(v, dim);
  sk.ask(even, lo, hi + 1);
  sv.ask(even + BYTES, lo, hi + 1);
  for (int j0 = lo; j0 <= hi;) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      lds_byte* const tk = b ? odd : even;
      lds_byte* const next = b ? even : odd;
      sk.put(tk);
      sv.put(tk + BYTES);
      arrived();
      if (j0 + BN <= hi) {
        sk.ask(next, j0 + BN, hi + 1);
        sv.ask(next + BYTES, j0 + BN, hi + 1);
      }
      f(tk, tk + BYTES, j0);
      j0 += BN;
      if (j0 > hi) return;
    }
  }
}

// A column's running sums.
template <int DP> struct Running {
  float m = -__builtin_inff(), base = 0.f, l = 0.f;          // the largest score, or one not far below; the same as a power of 2
  f32x16 acc[DP / 32];
};
// How far scores may be above the running maximum, as a power of 2, before sums are scaled to a new one.
constexpr float kSlack = 8.f;

// The first of a lane's result rows that lie in first .. last, and the last: rows of results 0 .. 15 are compared with them without the lane's part.
struct Seen {
  int first, last;
  __device__ __forceinline__ Seen(int f, int l, int lane) : first(f - 4 * (lane >> 5)), last(l - 4 * (lane >> 5)) {}
  __device__ __forceinline__ bool operator()(int tile, int r) const {
    const int row = tile * 32 + 8 * (r >> 2) + (r & 3);
    return row >= first && row <= last;
  }
};

// The pieces of an infinity are itself, 0 and 0, and those of a finite number have any signs: their products, or such that pass the range of fp32, make a
// NaN of a score that is -inf and weighs nothing.  So where sums are formed AGAIN because one is not finite, the scores of tile i, of rows
// row0 + 32 i .., that are not are formed from the numbers as they are: row `column` of `own`, a lane's, with the rows first .. last.  A column that has met a NaN
// or inf is `lost` either way.
template <int DTYPE, bool AGAIN>
struct Scores {
  typedef typename Value<DTYPE>::T T;
  HeadRows rows;
  int row0;
  HeadRows own;
  int column, first, last, lane, dim;
  bool& lost;
  __device__ __forceinline__ void operator()(f32x16& s, int i) const {
    if constexpr (AGAIN && Operand<DTYPE>::PLANES > 1) {
      const int top = row0 + i * 32;
      const Seen seen(first - top, last - top, lane);
      unsigned bad = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) bad |= seen(0, e) && !__builtin_isfinite(s[e]) ? 1u << e : 0u;
      while (bad && !lost) {
        const int r = __builtin_ctz(bad);
        bad &= bad - 1;
        const T* a = static_cast<const T*>(rows.p) + (top + result_row(r, lane)) * rows.stride;
        const T* b = static_cast<const T*>(own.p) + column * own.stride;
        float sum = 0.f;
#pragma unroll 1
        for (int d = 0; d < dim; ++d) sum += a[d] * b[d];
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = e == r ? sum : s[e];
        lost = !(sum < __builtin_inff());
      }
    }
  }
};

// What a tile's products say to those who bring tiles: that its keys have been read, that its values are read next.
struct Quiet {
  __device__ __forceinline__ void keys_read() const {}
  __device__ __forceinline__ void values_next() const {}
  __device__ __forceinline__ void both_next() const {}
  __device__ __forceinline__ void neither() const {}
};

template <int DTYPE, int DP, int TILES, bool CLEAN, typename B>
__device__ __forceinline__ void attend(Running<DP>& a, const Reader<DTYPE, DP>& read, const typename Operand<DTYPE>::F (&q)[DP / 16], const lds_byte* tk,
                                       const lds_byte* tv, float c, int lane, bool masked, int first, int last, unsigned& found,
                                       const Scores<DTYPE, CLEAN>& again, const B& bring) {
  typedef Operand<DTYPE> O;
  constexpr int STEPS = DP / 16;
  f32x16 s[TILES];
  {
    // two sums in turn: of two tiles, or of every other step of one
    f32x16 two[2] = {zero16(), zero16()};
    products<TILES * STEPS / 2, 2>([&](int n) { return Few<DTYPE, 2>{TILES == 2 ? read.along(tk, 0, n) : read.along(tk, 0, 2 * n), TILES == 2 ? read.along(tk, 32, n) : read.along(tk, 0, 2 * n + 1)}; },
                                   [&](int n, const Few<DTYPE, 2>& k) {
                                     multiply_few<DTYPE, 2>(k, [&](int i) -> const typename O::F& { return q[TILES == 2 ? n : 2 * n + i]; },
                                                            [&](int i) -> f32x16& { return two[i]; });
                                   });
    static_assert(TILES == 1 || TILES == 2, "");
    s[0] = TILES == 2 ? two[0] : two[0] + two[1];
    if constexpr (TILES == 2) s[1] = two[1];
  }
  bring.keys_read();
#pragma unroll
  for (int i = 0; i < TILES; ++i) again(s[i], i);
  if (masked) {
    const Seen seen(first, last, lane);
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[i][e] = seen(i, e) ? s[i][e] : -__builtin_inff();
  }
  float most = a.m;
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) most = __builtin_fmaxf(most, s[i][e]);
  most = __builtin_fmaxf(most, other_half(most));
  const bool grown = (most - a.m) * c > kSlack;              // of this lane's column alone: no other column's scores change its bits
  if (__any(grown)) {
    const float base = grown ? most * c : a.base, less = !grown ? 1.f : a.m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(a.base - base);
    a.m = grown ? most : a.m;
    a.base = base;
    a.l *= less;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) a.acc[t] *= less;
  }
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      s[i][e] = __builtin_amdgcn_exp2f(s[i][e] * c - a.base);
      a.l += s[i][e];
    }
  bring.values_next();
#pragma unroll
  for (int n = 0; n < TILES * 2; ++n) multiply_across<DTYPE, DP, CLEAN>(a.acc, read, tv, n * 16, O::from(s[n / 2], n & 1, true), found);
}

// ---- wavefronts that share columns ------------------------------------------------------------------------
// Where there are few columns for the chip a workgroup's wavefronts share 32, and take 32 keys each of a tile of as many as have room in LDS.
template <int DTYPE> constexpr int kSharing = 2 * kTile<DTYPE> / 32;

// The sums of a workgroup's wavefronts in its first one; `even` and `odd` are free.
template <int DTYPE, int DP>
__device__ __forceinline__ void join_sums(f32x16 (&acc)[DP / 32], int wave, int lane, unsigned char* even, unsigned char* odd) {
  constexpr int BLOCK = DP * 32 * 4;
  static_assert(2 * BLOCK <= kLds<DTYPE, DP> && kSharing<DTYPE> <= 4, "two wavefronts' sums in an array");
  const auto block = [&](int w) { return reinterpret_cast<float*>(w <= 2 ? even + (w - 1) * BLOCK : odd); };
  if (wave > 0 && wave < kSharing<DTYPE>) {
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) block(wave)[(t * 16 + r) * 64 + lane] = acc[t][r];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int t = 0; t < DP / 32; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int w = 1; w < kSharing<DTYPE>; ++w) acc[t][r] += block(w)[(t * 16 + r) * 64 + lane];
}
// The same for running sums: each column's maximum first.  l comes whole, of both halves.
template <int DTYPE, int DP>
__device__ __forceinline__ void join_running(Running<DP>& a, float c, int wave, int lane, unsigned char* even, unsigned char* odd) {
  constexpr int N = kSharing<DTYPE>;
  __shared__ float of_waves[2][N][32];
  a.l += other_half(a.l);
  if (lane < 32 && wave < N) of_waves[0][wave][lane] = a.m;
  __syncthreads();
  float most = of_waves[0][0][lane & 31];
#pragma unroll
  for (int w = 1; w < N; ++w) most = __builtin_fmaxf(most, of_waves[0][w][lane & 31]);
  const float base = most == -__builtin_inff() ? 0.f : most * c, less = a.m == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(a.base - base);
  if (lane < 32 && wave < N) of_waves[1][wave][lane] = a.l * less;
  if (wave < N) {
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) a.acc[t] *= less;
  }
  join_sums<DTYPE, DP>(a.acc, wave, lane, even, odd);
  a.m = most;
  a.base = base;
  a.l = 0.f;
#pragma unroll
  for (int w = 0; w < N; ++w) a.l += of_waves[1][w][lane & 31];
}
// Rows of bf16 that go to LDS directly are each wavefront's own business: it asks for its next keys when those it has are read, for its next
// values when those are, and waits for neither longer than it has to.
template <int DTYPE, int DP>
struct Ahead {
  typedef Stage<DTYPE, DP, 32, 64, true> S;
  S k, v;
  lds_byte *tk, *tv;
  int next, end;
  __device__ __forceinline__ void keys_read() const {
    lds_read();
    const_cast<S&>(k).ask(tk, next, end);
  }
  __device__ __forceinline__ void values_next() const { all_but<S::N>(); }      // the next keys are behind them
  __device__ __forceinline__ void both_next() const { all_but<0>(); }
  __device__ __forceinline__ void neither() const {
    all_but<0>();
    keys_read();
  }
  __device__ __forceinline__ void values_read() const {
    lds_read();
    const_cast<S&>(v).ask(tv, next, end);
  }
};
// Keys lo .. hi in tiles of kSharing x 32, `f(its keys, their values, the first of them, who brings them)` for each wavefront that has some.  Other rows
// come one tile at a time; two workgroups of a unit take turns.
template <int DTYPE, int DP, bool DIRECT, typename F>
__device__ __forceinline__ void walk_shared(unsigned char* even, unsigned char* odd, const HeadRows& k, const HeadRows& v, int lo, int hi, int dim, F f) {
  constexpr int ROWS = kSharing<DTYPE> * 32, EACH = 32 * Rows<DTYPE, DP>::BYTES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if constexpr (DIRECT && Operand<DTYPE>::PLANES == 1) {
    static_assert(ROWS == kThreads / 64 * 32, "every wavefront takes part");
    Ahead<DTYPE, DP> a;
    a.k.init(k, dim);
    a.v.init(v, dim);
    a.tk = (lds_byte*)even + wave * EACH;
    a.tv = (lds_byte*)odd + wave * EACH;
    a.end = hi + 1;
    a.next = lo + wave * 32;
    if (a.next <= hi) {
      a.keys_read();
      a.values_read();
      for (int j0 = a.next; j0 <= hi; j0 = a.next) {
        a.next = j0 + ROWS;
        all_but<Ahead<DTYPE, DP>::S::N>();
        f(a.tk, a.tv, j0, a);
        a.values_read();
      }
    }
    all_but<0>();                                            // what was asked for behind the last
  } else {
    Stage<DTYPE, DP, ROWS, kThreads, DIRECT> sk, sv;
    sk.init(k, dim);
    sv.init(v, dim);
    for (int j0 = lo; j0 <= hi; j0 += ROWS) {
      if (j0 > lo) __syncthreads();
      sk.ask((lds_byte*)even, j0, hi + 1);
      sv.ask((lds_byte*)odd, j0, hi + 1);
      sk.put((lds_byte*)even);
      sv.put((lds_byte*)odd);
      arrived();
      if (wave < kSharing<DTYPE> && j0 + wave * 32 <= hi) f((lds_byte*)even + wave * EACH, (lds_byte*)odd + wave * EACH, j0 + wave * 32, Quiet());
    }
  }
  __syncthreads();                                           // the arrays are free
}

// ---- sequences --------------------------------------------------------------------------------------
// Sequence s is rows offsets[s] .. offsets[s + 1] - 1.  Whatever the offsets hold, no row outside 0..rows is touched.
struct Sequences { const int64_t* offsets; int n; int rows; };

// The last of `n` sequences that begins at or before `row`, or -1; the same row in all lanes, the last 64 candidates together.
__device__ __forceinline__ int last_before(const Sequences& q, int64_t row) {
  int lo = 0, hi = q.n;
  while (hi - lo > 64) {
    const int mid = lo + ((hi - lo) >> 1);
    if (q.offsets[mid] <= row) lo = mid + 1; else hi = mid;
  }
  const int i = (int)(threadIdx.x & 63) < hi - lo ? lo + (int)(threadIdx.x & 63) : -1;
  return lo + __popcll(__ballot(i >= 0 && q.offsets[i < 0 ? 0 : i] <= row)) - 1;
}
__device__ __forceinline__ int from_lane(int v, int lane) { return __builtin_amdgcn_ds_bpermute(lane << 2, v); }

// Begin and end of the sequence of a lane's row; both 0 where it has none.  And, the same in all lanes, the begin of the sequence of row
// `top` (top itself where it has none) and the end of that of row `bottom` (behind bottom where it has none): all rows between are in
// sequences that begin and end within.  64 offsets lie side by side in the lanes and are searched there: one load for up to 63 sequences.
struct Span { int begin, end, top_begin, bottom_end; };
__device__ __forceinline__ Span span_of(const Sequences& q, int row, int top, int bottom) {
  constexpr int kNone = 0x7FFFFFFF;
  const int lane = threadIdx.x & 63;
  int s0 = q.n > 63 ? last_before(q, top) : 0;
  s0 = s0 < 0 ? 0 : s0;
  const bool there = lane <= q.n - s0;
  const int64_t offset = q.offsets[there ? s0 + lane : q.n];
  const int w = !there ? kNone : offset < 0 ? 0 : offset < q.rows ? (int)offset : q.rows;
  Span r{0, 0, top, bottom + 1};
  if (__builtin_amdgcn_readlane(w, 63) > bottom) {
    int n = 0;                                              // offsets at or before the lane's row
#pragma unroll
    for (int step = 32; step; step >>= 1)
      if (from_lane(w, n + step - 1) <= row) n += step;
    const int b = from_lane(w, n > 0 ? n - 1 : 0), e = from_lane(w, n);
    if (n > 0 && row < e && e != kNone) { r.begin = b; r.end = e; }       // (the search says 63 at most: for a row behind the last that may be its end)
    const int above = __popcll(__ballot(w <= top)), below = __popcll(__ballot(w <= bottom));
    if (above > 0 && above < 64 && __builtin_amdgcn_readlane(w, above < 64 ? above : 63) != kNone) r.top_begin = __builtin_amdgcn_readlane(w, above - 1);
    const int behind = below > 0 && below < 64 ? __builtin_amdgcn_readlane(w, below) : kNone;
    if (behind != kNone) r.bottom_end = behind;
  } else {                                                  // more than 62 sequences in the tile: each lane searches for itself
    const auto find = [&](int of, int& begin, int& end) {
      int lo = 0, hi = q.n;
      while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if (q.offsets[mid] <= of) lo = mid + 1; else hi = mid;
      }
      if (lo == 0 || of >= q.rows) return;
      const int64_t b = q.offsets[lo - 1], e = q.offsets[lo];
      if (of < e) { begin = b < 0 ? 0 : (int)b; end = e < q.rows ? (int)e : q.rows; }
    };
    find(row, r.begin, r.end);
    int first = top, last = 0, none = 0;
    find(top, first, none);
    find(bottom, none, last);
    r.top_begin = first;
    if (last > 0) r.bottom_end = last;
  }
  r.top_begin = __builtin_amdgcn_readfirstlane(r.top_begin < top ? r.top_begin : top);
  r.bottom_end = __builtin_amdgcn_readfirstlane(r.bottom_end > bottom ? r.bottom_end : bottom + 1);
  return r;
}

#endif

}  // namespace lsam
