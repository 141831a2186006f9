// What the attention kernels share: operands of the matrix units, tiles of rows in LDS, and which rows see which.
//
// Products are 32 x 32 results over 16 numbers at a time.  A lane's part of a result is one column (lane % 32) and sixteen rows, 8 (r / 4) +
// 4 (lane / 32) + r % 4.  Its eight numbers of an operand may be any eight of the sixteen as long as both operands agree, so
// results r = 8 t .. 8 t + 7 are, as they lie, the operand of a next product that sums over rows 16 t .. 16 t + 15: probabilities go from
// one product into the next without leaving the lane.
#pragma once
#include "ops.h"

namespace lsam {

#if defined(__HIPCC__)

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) unsigned char lds_byte;

template <int DTYPE> struct Operand;
template <> struct Operand<LSAM_DTYPE_BF16> {
  typedef bf16x8 F;
  static constexpr int B = 2;
  static __device__ __forceinline__ f32x16 multiply(F a, F b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ __forceinline__ F from(const f32x16& s, int t) {
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
};
// fp32 products stay in fp32: eight products over two numbers.
template <> struct Operand<LSAM_DTYPE_FP32> {
  typedef f32x8 F;
  static constexpr int B = 4;
  static __device__ __forceinline__ f32x16 multiply(F a, F b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ F from(const f32x16& s, int t) {
    F f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = s[8 * t + e];
    return f;
  }
  static __device__ __forceinline__ F clean(F f, unsigned& found) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool fine = __builtin_isfinite(f[e]);
      found |= fine ? 0u : 1u;
      f[e] = fine ? f[e] : 0.f;
    }
    return f;
  }
};

// Rows of DP numbers in LDS, in units of 16 bytes.  A unit's place in its row goes by the row, so that neither sixteen lanes that read
// the same unit of sixteen rows nor sixteen that read 32 bytes of four rows meet in a bank.
template <int DTYPE, int DP>
struct Rows {
  typedef typename Operand<DTYPE>::F F;
  static constexpr int B = Operand<DTYPE>::B, WIDE = DP > 64 ? 128 : 64, U = WIDE * B / 16, BYTES = WIDE * B;
  static __device__ __forceinline__ int turn(int row) {
    if constexpr (DTYPE == LSAM_DTYPE_FP32) return row & 15 & (U - 1);
    else if constexpr (U == 16) return (row & 3) << 2 | (row >> 2 & 3);
    else return (row >> 1 & 1) << 2 | (row >> 2 & 3);
  }
  static __device__ __forceinline__ int place(int row, int unit) { return row * BYTES + ((unit ^ turn(row)) << 4); }

};

// A lane's places in a tile of rows, found once: what is read from a tile whose address is known when this is compiled takes an
// offset beside them and no arithmetic.
template <int DTYPE, int DP> struct Reader;
template <int DP> struct Reader<LSAM_DTYPE_BF16, DP> {
  typedef Rows<LSAM_DTYPE_BF16, DP> R;
  typedef bf16x8 F;
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
    return __builtin_bit_cast(F, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(tile + row0 * R::BYTES + row[step]));
  }
  // Column 32 t + lane % 32, rows row0 + 4 (lane / 32) + 0 .. 3 and 8 further: the rows of a lane's results.
  __device__ __forceinline__ F across(const lds_byte* tile, int row0, int t) const {
    typedef __attribute__((address_space(3))) s16x4* quad_ptr;
    lds_byte* const p = const_cast<lds_byte*>(tile) + row0 * R::BYTES;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((quad_ptr)(p + column[t][0]));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((quad_ptr)(p + column[t][1]));
    return __builtin_bit_cast(F, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};
template <int DP> struct Reader<LSAM_DTYPE_FP32, DP> {
  typedef Rows<LSAM_DTYPE_FP32, DP> R;
  typedef f32x8 F;
  int lane;
  __device__ __forceinline__ Reader(int l) : lane(l) {}
  __device__ __forceinline__ F along(const lds_byte* tile, int row0, int step) const {
    typedef const __attribute__((address_space(3))) u32x4* unit_ptr;
    const int r = row0 + (lane & 31), u = step * 4 + (lane >> 5) * 2;
    const f32x4 a = __builtin_bit_cast(f32x4, *reinterpret_cast<unit_ptr>(tile + R::place(r, u)));
    const f32x4 b = __builtin_bit_cast(f32x4, *reinterpret_cast<unit_ptr>(tile + R::place(r, u + 1)));
    return F{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
  __device__ __forceinline__ F across(const lds_byte* tile, int row0, int t) const {
    const int col = t * 32 + (lane & 31);
    F f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = row0 + (lane >> 5) * 4 + (e & 3) + (e >> 2) * 8;
      f[e] = *reinterpret_cast<const __attribute__((address_space(3))) float*>(tile + R::place(r, col >> 2) + (col & 3) * 4);
    }
    return f;
  }
};

// Rows of a tensor for one head.
struct HeadRows { const void* p; int64_t stride; };

// 16 bytes of a row from unit u on; numbers behind `dim` count as 0.
template <int DTYPE>
__device__ __forceinline__ u32x4 load_unit(const typename Value<DTYPE>::T* row, int u, int dim) {
  constexpr int N = 16 / Operand<DTYPE>::B;
  const int n = dim - u * N;
  u32x4 w = {0, 0, 0, 0};
  if constexpr (DTYPE == LSAM_DTYPE_BF16) {
    if (n >= N) {
      w = __builtin_bit_cast(u32x4, *reinterpret_cast<const u16x8_any*>(row + u * N));
    } else if (n > 0) {
      u16x8 v;
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < n ? row[u * N + e] : (unsigned short)0;
      w = __builtin_bit_cast(u32x4, v);
    }
  } else {
    if (n >= N) {
      w = __builtin_bit_cast(u32x4, *reinterpret_cast<const f32x4_any*>(row + u * N));
    } else if (n > 0) {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < n ? row[u * N + e] : 0.f;
      w = __builtin_bit_cast(u32x4, v);
    }
  }
  return w;
}

// A lane's operand straight from a row in memory: numbers 16 step + 8 (lane / 32) .. + 7.
template <int DTYPE>
__device__ __forceinline__ typename Operand<DTYPE>::F load_operand(const typename Value<DTYPE>::T* row, int step, int lane, int dim) {
  if constexpr (DTYPE == LSAM_DTYPE_BF16) {
    return __builtin_bit_cast(bf16x8, load_unit<DTYPE>(row, step * 2 + (lane >> 5), dim));
  } else {
    const int u = step * 4 + (lane >> 5) * 2;
    const f32x4 a = __builtin_bit_cast(f32x4, load_unit<DTYPE>(row, u, dim)), b = __builtin_bit_cast(f32x4, load_unit<DTYPE>(row, u + 1, dim));
    return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  }
}

// A workgroup's way of bringing ROWS rows into LDS; rows from `limit` on count as 0.  Rows that are aligned to 16 bytes (DIRECT) go there
// without passing through registers: asked for a tile ahead, there when the wavefront has waited for its loads.  Others
// are asked for a tile ahead as well, and put there when they are needed.
template <int DTYPE, int DP, int ROWS, int THREADS, bool DIRECT>
struct Stage {
  typedef typename Value<DTYPE>::T T;
  typedef Rows<DTYPE, DP> R;
  static constexpr int N = ROWS * R::U / THREADS;
  static_assert(N * THREADS == ROWS * R::U, "whole rounds of loads");
  const T* p;
  int64_t stride;
  int dim;
  u32x4 w[DIRECT ? 1 : N];
  unsigned at[DIRECT ? N : 1];
  __device__ __forceinline__ void init(const HeadRows& t, int d) {
    p = static_cast<const T*>(t.p);
    stride = t.stride;
    dim = d;
    if constexpr (DIRECT) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + i * THREADS, row = n / R::U, unit = (n % R::U) ^ R::turn(row);
        at[i] = unit * 16 < dim * R::B ? (unsigned)(row * stride * R::B) + unit * 16 : 0x7FFFFFF0u;
      }
    }
  }
  __device__ __forceinline__ void ask(lds_byte* tile, int64_t row0, int64_t limit) {
    if constexpr (DIRECT) {
      const int64_t rows = limit - row0 < ROWS ? limit - row0 : ROWS;
      const unsigned bytes = rows > 0 ? (unsigned)(((rows - 1) * stride + dim) * R::B) : 0;
      const unsigned long long a = reinterpret_cast<unsigned long long>(p + row0 * stride);
      const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a), hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
      const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((unsigned long long)hi << 32 | lo), 0,
                                                                            __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
      for (int i = 0; i < N; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)(tile + (wave * 64 + i * THREADS) * 16), 16, at[i], 0, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + i * THREADS, row = n / R::U;
        w[i] = u32x4{0, 0, 0, 0};
        if (row0 + row < limit) w[i] = load_unit<DTYPE>(p + (row0 + row) * stride, n % R::U, dim);
      }
    }
  }
  __device__ __forceinline__ void put(lds_byte* tile) const {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int n = threadIdx.x + i * THREADS;
        *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(tile + R::place(n / R::U, n % R::U)) = w[i];
      }
    }
  }
};
// Waits for the wavefront's own loads, and for the other wavefronts.
__device__ __forceinline__ void arrived() {
  __builtin_amdgcn_s_waitcnt(0x0070);                      // no load on its way, no LDS access
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Whether rows can go to LDS directly: 16-byte units all the way, and a tile within 32-bit offsets.
inline bool direct(const void* p, int64_t stride, int64_t head, int64_t seq, int dim, int dtype) {
  const int b = dtype_bytes(dtype);
  return !misaligned(p, 16) && stride * b % 16 == 0 && head * b % 16 == 0 && seq * b % 16 == 0 && dim * b % 16 == 0 && stride < 1 << 20;
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
  products<DP / 32, kAhead>([&](int t) { return read.across(tile, row0, t); },
                            [&](int t, const typename O::F& a) { acc[t] = O::multiply(CLEAN ? O::clean(a, found) : a, p, acc[t]); });
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

// ---- sequences --------------------------------------------------------------------------------------
// Sequence s is rows offsets[s] .. offsets[s + 1] - 1.  Whatever the offsets hold, no row outside 0..rows is touched.
struct Sequences { const int64_t* offsets; int n; int rows; };

// The last of `n` sequences that begins at or before `row`, or -1; the same row in all lanes, the last 64 candidates together.
__device__ __forceinline__ int last_before(const Sequences& q, int64_t row) {
  int lo = 0, hi = q.n;
  while (hi - lo > 64) {
    const int mid = (lo + hi) >> 1;
    if (q.offsets[mid] <= row) lo = mid + 1; else hi = mid;
  }
  const int i = lo + (int)(threadIdx.x & 63);
  return lo + __popcll(__ballot(i < hi && q.offsets[i < hi ? i : 0] <= row)) - 1;
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
  const int64_t offset = q.offsets[s0 + lane <= q.n ? s0 + lane : q.n];
  const int w = s0 + lane > q.n ? kNone : offset < 0 ? 0 : offset < q.rows ? (int)offset : q.rows;
  Span r{0, 0, top, bottom + 1};
  if (__builtin_amdgcn_readlane(w, 63) > bottom) {
    int n = 0;                                              // offsets at or before the lane's row
#pragma unroll
    for (int step = 32; step; step >>= 1)
      if (from_lane(w, n + step - 1) <= row) n += step;
    const int b = from_lane(w, n > 0 ? n - 1 : 0), e = from_lane(w, n);
    if (n > 0 && e != kNone) { r.begin = b; r.end = e; }
    const int above = __popcll(__ballot(w <= top)), below = __popcll(__ballot(w <= bottom));
    if (above > 0 && above < 64 && __builtin_amdgcn_readlane(w, above < 64 ? above : 63) != kNone) r.top_begin = __builtin_amdgcn_readlane(w, above - 1);
    const int behind = below > 0 && below < 64 ? __builtin_amdgcn_readlane(w, below) : kNone;
    if (behind != kNone) r.bottom_end = behind;
  } else {                                                  // more than 62 sequences in the tile: each lane searches for itself
    const auto find = [&](int of, int& begin, int& end) {
      int lo = 0, hi = q.n;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
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
