// lsam_adapter, lsam_adapter_backward: y = x W^T + bias + scale (x A_a^T) B_a^T, W shared by all rows and a the adapter of
// the row's segment, and the gradients of x, A and B.
//
// The products run on the bf16 matrix units with fp32 sums.  bf16 operands are multiplied as they are; an fp32 number is
// split into three bfloat16 pieces h + m + l (24 bits: exact), of whose nine products the six that reach fp32's last bit are
// formed.  The rank-sized results u = x A^T and du = scale dy B stay in fp32 between the kernels.
//
//   shrink_kernel   u or du: [rows, rank], 64 rows of one segment a workgroup, the long contraction cut over its wavefronts
//   product_kernel  y or dx: tiles of W's product; then, for every segment that the tile's rows belong to, a few more steps
//                   of the same loop over the pieces of u and B (or du and A), rows of other segments being zero
//   few_rows_kernel y or dx where there are at most 64 rows: reads W once, 16 outputs a workgroup, no tile of x, no copy of W
//   grads_kernel    dA = sum du^T x and dB = scale sum dy^T u over the rows of an adapter, no sum split over workgroups
//   planes_kernel   pieces, aligned copies and the transposed W of the backward pass
#include "ops.h"
#include "planes.h"

namespace lsam {
namespace {

typedef __attribute__((address_space(3))) unsigned char lds_byte;

constexpr int kMaxRank = LSAM_ADAPTER_MAX_RANK;

// ---- segments ---------------------------------------------------------------------------------------
// Segment s is rows begin[s] .. begin[s + 1] - 1 with adapter which[s]; rows of no segment, and of one whose adapter does not
// exist, have none.  Whatever the arrays hold, no row outside the matrix and no adapter that is not there is touched.
struct Segments {
  const int32_t* begin; const int32_t* which;
  int n, adapters;
  bool each;                                          // copies for product_kernel: one for each segment, else for each adapter
};
__device__ __forceinline__ int64_t seg_row(const Segments& g, int s, int64_t rows) {
  const int64_t b = g.begin[s];
  return b < 0 ? 0 : b > rows ? rows : b;
}
// The last segment that begins at or before `row`, or -1; the same row in all lanes.  The last 64 candidates are looked at
// together: one load to wait for instead of six.
__device__ __forceinline__ int seg_at(const Segments& g, int64_t row) {
  int lo = 0, hi = g.n;
  while (hi - lo > 64) {
    const int mid = (lo + hi) >> 1;
    if (g.begin[mid] <= row) lo = mid + 1; else hi = mid;
  }
  const int i = lo + (int)(threadIdx.x & 63);
  return lo + __popcll(__ballot(i < hi && g.begin[i < hi ? i : 0] <= row)) - 1;
}
__device__ __forceinline__ int seg_adapter(const Segments& g, int s) {
  const int a = g.which[s];
  return a >= 0 && a < g.adapters ? a : -1;
}
// The copy of the adapter of segment s for product_kernel, or -1.
__device__ __forceinline__ int seg_copy(const Segments& g, int s) {
  const int a = seg_adapter(g, s);
  return a >= 0 && g.each ? s : a;
}
// The adapter of a row, another row in every lane.
__device__ __forceinline__ int row_adapter(const Segments& g, int64_t row, int64_t rows) {
  int lo = 0, hi = g.n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (g.begin[mid] <= row) lo = mid + 1; else hi = mid;
  }
  return lo > 0 && row < seg_row(g, lo, rows) ? seg_adapter(g, lo - 1) : -1;
}

// What is written above stays above: a run of loads goes out before the first of them is waited for.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// ---- operands of the matrix units -------------------------------------------------------------------
// Eight numbers as NP words of eight bfloat16 pieces.
template <int NP> struct Pieces { bf16x8 p[NP]; };

__device__ __forceinline__ void split8(const float (&v)[8], Pieces<3>& o) {
  unsigned w[3][4];
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = largest_of(most, v[e]);
  if (past_rounding(most)) split_words_any<3, 8>(v, w);
  else split_words<3, 8>(v, w);
#pragma unroll
  for (int q = 0; q < 3; ++q) o.p[q] = __builtin_bit_cast(bf16x8, u32x4{w[q][0], w[q][1], w[q][2], w[q][3]});
}

// Pieces of a stored type: numbers that are bfloat16 already are their own.
template <int DTYPE> constexpr int kPieces = DTYPE == LSAM_DTYPE_BF16 ? 1 : 3;

// Eight numbers from p on, `step` apart (UNIT: neighbours).  A run of such loads waits for nothing in between.
template <int DTYPE, bool UNIT>
__device__ __forceinline__ void load8(const typename Value<DTYPE>::T* p, int64_t step, Pieces<kPieces<DTYPE>>& o) {
  if constexpr (DTYPE == LSAM_DTYPE_BF16) {
    u16x8 w;
    if constexpr (UNIT) {
      w = *reinterpret_cast<const u16x8_any*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = p[e * step];
    }
    o.p[0] = __builtin_bit_cast(bf16x8, w);
  } else {
    float v[8];
    if constexpr (UNIT) {
      Value<DTYPE>::load8(p, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = p[e * step];
    }
    split8(v, o);
  }
}
// The same where only the first n are there (n may be negative); the others count as 0.
template <int DTYPE>
__device__ __forceinline__ void load8_some(const typename Value<DTYPE>::T* p, int64_t step, int n, Pieces<kPieces<DTYPE>>& o) {
  if constexpr (DTYPE == LSAM_DTYPE_BF16) {
    u16x8 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = e < n ? p[e * step] : (unsigned short)0;
    o.p[0] = __builtin_bit_cast(bf16x8, w);
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e * step] : 0.f;
    split8(v, o);
  }
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// c += a b^T over 32 numbers of each row, from their pieces; small products first.
template <int NA, int NB>
__device__ __forceinline__ f32x4 multiply(const Pieces<NA>& a, const Pieces<NB>& b, f32x4 c) {
  constexpr int most = NA > NB ? NA : NB;
#pragma unroll
  for (int sum = most - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i <= sum; ++i)
      if (i < NA && sum - i < NB) c = mfma16(a.p[i], b.p[sum - i], c);
  return c;
}

// The six products of three pieces each that fp32 can tell from 0, the smallest first, four bits for a piece: l h, m m, h l,
// m h, h m, h h.
constexpr unsigned kSixLeft = 0x001012u, kSixRight = 0x010210u;

// A number's leading bfloat16 piece, as split_planes makes it, and its piece `which`.
__device__ __forceinline__ unsigned short leading_piece(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x), mag = u & 0x7FFFFFFFu;
  return mag >= 0x7F7F8000u && mag <= 0x7F800000u ? (unsigned short)(u >> 16) : narrow(x);
}
__device__ __forceinline__ unsigned short piece(float x, unsigned which) {
  float r = x;
  for (unsigned q = 0; q < which; ++q) r = __builtin_fabsf(r) < __builtin_inff() ? r - widen(leading_piece(r)) : 0.f;
  return leading_piece(r);
}

// The low-rank part of a product as more steps of its contraction: for each pair of pieces a copy of u and of the adapter, rank
// padded to 8 (`padded`), side by side.
struct LowRank {
  int rank, padded, pairs;
  unsigned left, right;                               // the pieces of each pair, four bits each
  int k() const { return pairs * padded; }
};

constexpr int waitcnt(int vm, int lgkm) { return (vm & 0xF) | ((vm >> 4) << 14) | (0x7 << 4) | ((lgkm & 0xF) << 8); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, unsigned bytes) {
  const unsigned long long a = reinterpret_cast<unsigned long long>(base);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a);
  const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
  void* ptr = reinterpret_cast<void*>(((unsigned long long)hi << 32) | lo);
  return __builtin_amdgcn_make_buffer_rsrc(ptr, 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}

// The wavefront's own loads, those to LDS among them: at most LEFT are still on their way.
template <int LEFT>
__device__ __forceinline__ void wait_loads() {
  __builtin_amdgcn_s_waitcnt(waitcnt(LEFT, 15));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_lds() {
  __builtin_amdgcn_s_waitcnt(waitcnt(63, 0));
  asm volatile("" ::: "memory");
}
// Waits until at most LEFT of the wavefront's own loads, those to LDS among them, are on their way, and then for the workgroup.
template <int LEFT>
__device__ __forceinline__ void arrived() {
  __builtin_amdgcn_s_waitcnt(waitcnt(LEFT, 0));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- a few rows of two matrices against each other ---------------------------------------------------
// Sums acc[x tile][left tile] of 16 x 16 results over all of K, each wavefront for its own steps of 64 numbers (wave, wave + WAVES,
// ...).  The matrix unit wants neighbouring lanes in different rows, which the address unit takes one line at a time: 64 cycles
// a load instead of 16, 18 us for 32 rows against 4096 x 4096.  So the rows go to LDS directly, whole lines of 128 bytes in
// neighbouring lanes, into a ring of S steps that belongs to the wavefront alone.  Rows that are not aligned for that are read
// straight into the matrix unit's layout.
//
// ROWS rows of 64 numbers of a step: bf16 in a line, fp32 in two.  Unit q (16 bytes) of a line of row r is at position
// q ^ (r / 2 % 8).
template <int DTYPE, int ROWS>
struct Lines {
  static constexpr int EACH = DTYPE == LSAM_DTYPE_BF16 ? 1 : 2;       // lines of a row in a step
  static constexpr int BYTES = ROWS * 128 * EACH, NLOAD = ROWS / 8 * EACH;
  static constexpr int B = DTYPE == LSAM_DTYPE_BF16 ? 2 : 4;
  unsigned goff[ROWS / 8];
  __device__ __forceinline__ void init(int64_t stride, int lane) {
#pragma unroll
    for (int j = 0; j < ROWS / 8; ++j) goff[j] = (unsigned)((j * 8 + (lane >> 3)) * stride * B);
  }
  // Rows past the resource's end and units past K arrive as zeros.
  __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rsrc, lds_byte* tile, int k0, int K, int lane) const {
#pragma unroll
    for (int l = 0; l < EACH; ++l)
#pragma unroll
      for (int j = 0; j < ROWS / 8; ++j) {
        const int row = j * 8 + (lane >> 3), at = k0 + l * 32 + ((lane & 7) ^ ((row >> 1) & 7)) * (16 / B);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(tile + (l * ROWS / 8 + j) * 1024), 16,
                                                 at < K ? goff[j] + (unsigned)(at * B) : 0x7FFFFFF0u, 0, 0, 0);
      }
  }
  // Eight numbers of row `row`: 32 kc + 8 quarter ..
  __device__ __forceinline__ void read(const lds_byte* tile, int row, int kc, int quarter, Pieces<kPieces<DTYPE>>& o) const {
    typedef const __attribute__((address_space(3))) u32x4* lds_unit;
    const int turn = (row >> 1) & 7;
    if constexpr (DTYPE == LSAM_DTYPE_BF16) {
      o.p[0] = __builtin_bit_cast(bf16x8, *reinterpret_cast<lds_unit>(tile + row * 128 + (((kc * 4 + quarter) ^ turn) << 4)));
    } else {
      const lds_byte* line = tile + kc * ROWS * 128 + row * 128;
      const f32x4 a = __builtin_bit_cast(f32x4, *reinterpret_cast<lds_unit>(line + (((quarter * 2) ^ turn) << 4)));
      const f32x4 b = __builtin_bit_cast(f32x4, *reinterpret_cast<lds_unit>(line + (((quarter * 2 + 1) ^ turn) << 4)));
      const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      split8(v, o);
    }
  }
};

// The left rows are contiguous along K (UNIT) or along the rows; `some`: how many there are.
template <int TYPE> struct Rows {
  const typename Value<TYPE>::T* p;
  int64_t stride, step;                               // from row to row, along K
  int some;
};
template <int DTYPE>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const Rows<DTYPE>& r, int K) {
  return make_rsrc(r.p, (unsigned)(((r.some - 1) * r.stride + K) * (DTYPE == LSAM_DTYPE_BF16 ? 2 : 4)));
}

// Bytes of a wavefront's part of a stage; wavefronts of a workgroup and stages, as many as the LDS of a compute unit has room for
// (more wavefronts rather than more stages: fp32's pieces are cut by the vector units, one wavefront at a time).
template <int LTYPE, int XTYPE, bool UNIT, int NL, int NX>
constexpr int kStageBytes = Lines<XTYPE, NX * 16>::BYTES + (UNIT ? Lines<LTYPE, NL * 16>::BYTES : 0);
constexpr int kRoom = 156 << 10;
constexpr int waves_for(int bytes) { return 8 * 2 * bytes <= kRoom ? 8 : 4 * 2 * bytes <= kRoom ? 4 : 2; }
constexpr int ring_for(int bytes) { return waves_for(bytes) * 3 * bytes <= kRoom ? 3 : 2; }

// A wavefront's way along K.
template <int LTYPE, int XTYPE, bool UNIT, int NL, int NX, int WAVES>
struct Staged {
  static constexpr int RING = ring_for(kStageBytes<LTYPE, XTYPE, UNIT, NL, NX>);
  typedef Lines<XTYPE, NX * 16> LX;
  typedef Lines<LTYPE, NL * 16> LL;
  static constexpr int LOADS = LX::NLOAD + (UNIT ? LL::NLOAD : 0);
  Rows<LTYPE> left;
  Rows<XTYPE> x;
  LX lx;
  LL ll;
  int K, lane, k, k_next;

  __device__ __forceinline__ void request(lds_byte* stage) {
    lx.issue(resource(x, K), stage, k_next, K, lane);
    if constexpr (UNIT) ll.issue(resource(left, K), stage + LX::BYTES, k_next, K, lane);
    k_next += WAVES * 64;
  }
  // Multiplies a stage and asks for the step RING steps later in its place.
  __device__ __forceinline__ void step(lds_byte* stage, f32x4 (&acc)[NX][NL]) {
    const int l16 = lane & 15, quarter = lane >> 4;
    Pieces<kPieces<LTYPE>> fl[2][NL];
    if constexpr (!UNIT) {
      // not staged: neighbouring lanes are neighbours in memory
#pragma unroll
      for (int kc = 0; kc < 2; ++kc)
#pragma unroll
        for (int r = 0; r < NL; ++r) {
          const int at = k + kc * 32 + quarter * 8;
          const typename Value<LTYPE>::T* p = left.p + (r * 16 + l16 < left.some ? r * 16 + l16 : left.some - 1) * left.stride + at * left.step;
          if (k + 64 <= K) load8<LTYPE, false>(p, left.step, fl[kc][r]);
          else load8_some<LTYPE>(p, left.step, K - at, fl[kc][r]);
        }
    }
    wait_loads<(RING - 1) * LOADS>();
    Pieces<kPieces<XTYPE>> fx[2][NX];
#pragma unroll
    for (int kc = 0; kc < 2; ++kc) {
#pragma unroll
      for (int t = 0; t < NX; ++t) lx.read(stage, t * 16 + l16, kc, quarter, fx[kc][t]);
      if constexpr (UNIT) {
#pragma unroll
        for (int r = 0; r < NL; ++r) ll.read(stage + LX::BYTES, r * 16 + l16, kc, quarter, fl[kc][r]);
      }
    }
    wait_lds();                                       // the fragments are here: the stage may be filled again
    request(stage);
#pragma unroll
    for (int kc = 0; kc < 2; ++kc)
#pragma unroll
      for (int t = 0; t < NX; ++t)
#pragma unroll
        for (int r = 0; r < NL; ++r) acc[t][r] = multiply(fl[kc][r], fx[kc][t], acc[t][r]);
    k += WAVES * 64;
  }
};

template <int LTYPE, int XTYPE, bool UNIT, int NL, int NX, int WAVES>
__device__ __forceinline__ void contract_staged(const Rows<LTYPE>& left, const Rows<XTYPE>& x, int K, int wave, int lane, lds_byte* s0,
                                                lds_byte* s1, lds_byte* s2, f32x4 (&acc)[NX][NL]) {
  Staged<LTYPE, XTYPE, UNIT, NL, NX, WAVES> o;
  o.left = left;
  o.x = x;
  o.K = K;
  o.lane = lane;
  o.k = o.k_next = wave * 64;
  o.lx.init(x.stride, lane);
  if constexpr (UNIT) o.ll.init(left.stride, lane);
  o.request(s0);
  o.request(s1);
  if constexpr (o.RING > 2) o.request(s2);            // past K: zeros
  while (o.k < K) {
    o.step(s0, acc);
    o.step(s1, acc);
    if constexpr (o.RING > 2) o.step(s2, acc);
  }
  wait_loads<0>();                                    // nothing may still be on its way to LDS
}

template <int LTYPE, int XTYPE, bool UNIT, int NL, int NX, int WAVES>
__device__ __forceinline__ void contract_straight(const Rows<LTYPE>& left, const Rows<XTYPE>& rows, int K, int wave, int lane,
                                                  f32x4 (&acc)[NX][NL]) {
  const int l16 = lane & 15, quarter = lane >> 4;
  // rows past the last one read the last one again, and their results are dropped
  const typename Value<XTYPE>::T* x[NX];
  const typename Value<LTYPE>::T* A[NL];
#pragma unroll
  for (int t = 0; t < NX; ++t) x[t] = rows.p + (t * 16 + l16 < rows.some ? t * 16 + l16 : rows.some - 1) * rows.stride;
#pragma unroll
  for (int r = 0; r < NL; ++r) A[r] = left.p + (r * 16 + l16 < left.some ? r * 16 + l16 : left.some - 1) * left.stride;
  // 16 numbers for each quarter of the lanes: two loads that share a line of 128 bytes
  const int k_lane = quarter * 16;
  int k = wave * 64;
  for (; k + 64 <= K; k += WAVES * 64) {
    Pieces<kPieces<LTYPE>> fa[2][NL];
    Pieces<kPieces<XTYPE>> fx[2][NX];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = k + k_lane + j * 8;
#pragma unroll
      for (int t = 0; t < NX; ++t) load8<XTYPE, true>(x[t] + at, 1, fx[j][t]);
#pragma unroll
      for (int r = 0; r < NL; ++r) load8<LTYPE, UNIT>(A[r] + at * left.step, left.step, fa[j][r]);
    }
    in_order();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < NX; ++t)
#pragma unroll
        for (int r = 0; r < NL; ++r) acc[t][r] = multiply(fa[j][r], fx[j][t], acc[t][r]);
  }
  if (k < K) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = k + k_lane + j * 8, n = K - at;
      Pieces<kPieces<LTYPE>> fa[NL];
#pragma unroll
      for (int r = 0; r < NL; ++r) load8_some<LTYPE>(A[r] + at * left.step, left.step, n, fa[r]);
#pragma unroll
      for (int t = 0; t < NX; ++t) {
        Pieces<kPieces<XTYPE>> fx;
        load8_some<XTYPE>(x[t] + at, 1, n, fx);
#pragma unroll
        for (int r = 0; r < NL; ++r) acc[t][r] = multiply(fa[r], fx, acc[t][r]);
      }
    }
  }
}

// The segments of a tile's rows, `step` numbers of the low-rank part at a time.  The next 64 segments are held a lane each.
struct SegmentsOf {
  const Segments& g;
  int m0, m_here, low_k, step;
  int64_t rows;
  int window, i, begins, copies;
  int lo, hi, copy, k0;                                // rows of the tile, copy of the adapter, first number
  bool done;
  __device__ __forceinline__ SegmentsOf(const Segments& g_, int64_t m0_, int m_here_, int64_t rows_, int low_k_, int step_)
      : g(g_), m0((int)m0_), m_here(m_here_), low_k(low_k_), step(step_), rows(rows_), i(0), k0(low_k_), done(g_.n == 0) {
    const int found = done ? 0 : seg_at(g, m0_);
    window = found < 0 ? 0 : found;
    if (!done) load();
  }
  __device__ __forceinline__ void load() {
    const int s = window + (int)(threadIdx.x & 63);
    begins = (int)seg_row(g, s < g.n ? s : g.n, rows);
    copies = s < g.n ? seg_copy(g, s) : -1;
  }
  __device__ __forceinline__ bool next() {
    if (done) return false;
    k0 += step;
    if (k0 < low_k) return true;
    while (true) {
      if (i == 63) {
        window += 63;
        i = 0;
        load();
      }
      const int l = __builtin_amdgcn_readlane(begins, i) - m0, h = __builtin_amdgcn_readlane(begins, i + 1) - m0;
      if (window + i >= g.n || l >= m_here) {
        done = true;
        return false;
      }
      copy = __builtin_amdgcn_readlane(copies, i);
      ++i;
      lo = l > 0 ? l : 0;
      hi = h < m_here ? h : m_here;
      if (copy >= 0 && lo < hi) {
        k0 = 0;
        return true;
      }
    }
  }
};

// ---- u = x A^T, du = scale dy B ---------------------------------------------------------------------
struct ShrinkParams {
  const void* x; int64_t x_stride;
  const void* A; int64_t a_adapter, a_rank, a_k;      // strides from adapter to adapter, and along rank and contraction
  float* u;
  int64_t rows; int K, rank;
  float scale;
  unsigned short* copy; float copy_scale; LowRank low; int low_k;      // pieces of copy_scale u for product_kernel, or null
  int* adapter;                                       // receives the adapter of every row, or null
  Segments g;
};

template <int DTYPE, int ATYPE, bool UNIT, int NR, int RT>
constexpr int kShrinkWaves = waves_for(kStageBytes<ATYPE, DTYPE, UNIT, NR, RT>);

// Workgroup (tile, j, r): ranks 16 NR r and on of the j-th, j + groups-th, ... segment of the tile's 16 RT rows, the contraction
// cut over its wavefronts.  Bound by reading x where segments are long (16384 x 4096 bf16, 134 MB, rank 16 with fp32 adapters,
// whose pieces the vector units cut: 43-48 us, 2.8-3.1 TB/s), by reading A where each row has its own (32 rows of 32 adapters,
// 4096 -> rank 16: 7 us, half of it the wait for the segments and then the first rows).  UNIT: the contraction is contiguous in A.
template <int DTYPE, int ATYPE, bool UNIT, int NR, int RT, int WAVES, bool STAGED>
__global__ __launch_bounds__(WAVES * 64) void shrink_kernel(ShrinkParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef typename Value<ATYPE>::T TA;
  constexpr int ROWS = RT * 16;
  constexpr int PITCH = NR * 16 + 1;
  constexpr int STAGE = kStageBytes<ATYPE, DTYPE, UNIT, NR, RT>;
  constexpr int PART = WAVES * 16 * PITCH * 4;
  constexpr int FIRST = STAGED && WAVES * STAGE > PART ? WAVES * STAGE : PART;      // the sums go where a stage was
  // an array for each stage, so that the compiler knows the one that is read from those that are on their way
  __shared__ __attribute__((aligned(1024))) unsigned char st0[FIRST];
  __shared__ __attribute__((aligned(1024))) unsigned char st1[STAGED ? WAVES * STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st2[STAGED && ring_for(STAGE) > 2 ? WAVES * STAGE : 16];
  float (*part)[16][PITCH] = reinterpret_cast<float (*)[16][PITCH]>(st0);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, quarter = lane >> 4;
  const int64_t row0 = (int64_t)blockIdx.x * ROWS, row1 = row0 + ROWS < p.rows ? row0 + ROWS : p.rows;
  const int groups = (int)gridDim.y - 1, rank0 = (int)blockIdx.z * (NR * 16);
  if ((int)blockIdx.y == groups) {
    if (rank0 > 0) return;
    // the last one: adapters of rows, and the rows without one (a search that the others need not wait for)
    for (int i = tid; i < ROWS; i += WAVES * 64) {
      if (row0 + i >= row1) break;
      const int a = row_adapter(p.g, row0 + i, p.rows);
      if (p.adapter) p.adapter[row0 + i] = a;
      if (a < 0)
        for (int r = 0; r < p.rank; ++r) p.u[(row0 + i) * p.rank + r] = 0.f;
    }
    return;
  }
  const int found = seg_at(p.g, row0);
  for (int s = (found < 0 ? 0 : found) + (int)blockIdx.y; s < p.g.n; s += groups) {
    int64_t lo = seg_row(p.g, s, p.rows), hi = seg_row(p.g, s + 1, p.rows);
    if (lo >= row1) break;
    lo = lo > row0 ? lo : row0;
    hi = hi < row1 ? hi : row1;
    const int a = seg_adapter(p.g, s);
    if (a < 0 || lo >= hi) continue;
    f32x4 acc[RT][NR];
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int r = 0; r < NR; ++r) acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int ranks = p.rank - rank0 < NR * 16 ? p.rank - rank0 : NR * 16;
    const Rows<ATYPE> left{static_cast<const TA*>(p.A) + a * p.a_adapter + rank0 * p.a_rank, p.a_rank, p.a_k, ranks};
    const Rows<DTYPE> x{static_cast<const T*>(p.x) + lo * p.x_stride, p.x_stride, 1, (int)(hi - lo)};
    if constexpr (STAGED)
      contract_staged<ATYPE, DTYPE, UNIT, NR, RT, WAVES>(left, x, p.K, wave, lane, (lds_byte*)st0 + wave * STAGE, (lds_byte*)st1 + wave * STAGE,
                                                         (lds_byte*)st2 + (ring_for(STAGE) > 2 ? wave * STAGE : 0), acc);
    else
      contract_straight<ATYPE, DTYPE, UNIT, NR, RT, WAVES>(left, x, p.K, wave, lane, acc);
    // lane: row l16 of a tile, ranks 4 quarter .. + 3
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (lo + t * 16 < hi) {              // the same for all
        __syncthreads();
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i) part[wave][l16][r * 16 + quarter * 4 + i] = acc[t][r][i];
        __syncthreads();
        for (int i = tid; i < 16 * NR * 16; i += WAVES * 64) {
          const int row = i / (NR * 16), r = rank0 + i % (NR * 16);
          if (r < p.low.padded && lo + t * 16 + row < hi) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += part[w][row][r - rank0];
            sum = r < p.rank ? p.scale * sum : 0.f;
            if (r < p.rank) p.u[(lo + t * 16 + row) * p.rank + r] = sum;
            if (p.copy)
              for (int q = 0; q < p.low.pairs; ++q)
                p.copy[(lo + t * 16 + row) * p.low_k + q * p.low.padded + r] = piece(p.copy_scale * sum, (p.low.left >> (4 * q)) & 15u);
          }
        }
      }
    }
    __syncthreads();
  }
}

// ---- the adapters' pieces for product_kernel --------------------------------------------------------
struct CopiesParams {
  const void* Q; int64_t q_adapter, q_n, q_r;         // strides along adapter, output and rank
  unsigned short* copy; unsigned char* odd;           // [copies][N][low_k], [copies][N]
  int N, low_k;
  LowRank low;
  Segments g; int64_t rows;
};
// An infinity or NaN in an adapter would reach the rows of other segments in its tile, whose 0 it is multiplied with: it is left
// out here, and the outputs it belongs to are marked.  There is a copy for each segment or for each adapter, whichever are fewer: what
// a call costs does not go by adapters that it does not use.  16 adapters of 8192 x 32 in bf16 23-25 us.
template <int QTYPE>
__global__ __launch_bounds__(256) void copies_kernel(CopiesParams p) {
  typedef typename Value<QTYPE>::T TQ;
  const int n = (int)(blockIdx.x * 256 + threadIdx.x), c = (int)blockIdx.y;
  const int a = !p.g.each ? c : seg_row(p.g, c, p.rows) < seg_row(p.g, c + 1, p.rows) ? seg_adapter(p.g, c) : -1;
  if (a < 0 || n >= p.N) return;
  const int64_t at = (int64_t)c * p.N + n;
  const TQ* q = static_cast<const TQ*>(p.Q) + a * p.q_adapter + n * p.q_n;
  bool odd = false;
  for (int r0 = 0; r0 < p.low.padded; r0 += 8) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = r0 + e < p.low.rank ? r0 + e : p.low.rank - 1;
      v[e] = Value<QTYPE>::get(q + r * p.q_r);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (r0 + e >= p.low.rank) v[e] = 0.f;
      if (!(__builtin_fabsf(v[e]) < __builtin_inff())) { v[e] = 0.f; odd = true; }
    }
    Pieces<3> o;
    split8(v, o);
    for (int i = 0; i < p.low.pairs; ++i) {
      const unsigned w = (p.low.right >> (4 * i)) & 15u;
      *reinterpret_cast<bf16x8*>(p.copy + at * p.low_k + i * p.low.padded + r0) = w == 0 ? o.p[0] : w == 1 ? o.p[1] : o.p[2];
    }
  }
  p.odd[at] = odd;
}

// ---- y or dx, many rows -----------------------------------------------------------------------------
struct ProductParams {
  const unsigned short* X; int64_t ldx, plane_x;      // [pieces][M][ldx], K of each row
  const unsigned short* W; int64_t ldw, plane_w;      // [pieces][N][ldw]
  int64_t M; int N, K;                                // K a multiple of 8, rows 16-byte aligned
  void* Y; int64_t ldy;
  const float* bias;
  const unsigned short* u; const unsigned short* Q;   // copies: [M][low_k], [copies][N][low_k]
  const unsigned char* odd;                           // [copies][N]
  int low_k;
  int tilesM, tilesN;
  Segments g;
};

// One operand's tile of R rows by BK numbers in LDS.  BK = 64: row r is a line of 128 bytes, 8 units of 16, unit q at position
// q ^ (r / 2 % 8); BK = 32: 64 bytes, 4 units, unit q at q ^ (r / 4 % 4).  The sixteen lanes whose fragments LDS serves together
// (0-3, 12-15, 20-23, 24-27 and so on) then read from different banks (no conflict counted).  Global memory goes to LDS
// directly, whole rows in neighbouring lanes; the lane order of that copy is fixed, so a lane asks for the unit that belongs at
// its position.
template <int BK>
__device__ __forceinline__ int turned(int row, int unit) { return BK == 64 ? unit ^ ((row >> 1) & 7) : unit ^ ((row >> 2) & 3); }

template <int R, int NW, int BK>
struct RowTile {
  static constexpr int BYTES = R * BK * 2;
  static constexpr int EACH = 512 / BK;              // rows of an instruction
  static constexpr int NLOAD = R / EACH / NW;
  static_assert(R % (EACH * NW) == 0, "whole instructions for every wavefront");
  unsigned goff[NLOAD];        // of this lane's unit, at step 0
  int k[NLOAD];                // the first number of the unit
  static __device__ __forceinline__ int row(int j, int lane, int wave) { return (wave * NLOAD + j) * EACH + lane / (BK / 8); }
  static __device__ __forceinline__ int first(int j, int lane, int wave) { return turned<BK>(row(j, lane, wave), lane % (BK / 8)) * 8; }
  __device__ __forceinline__ void init(int64_t ld, int lane, int wave) {
#pragma unroll
    for (int j = 0; j < NLOAD; ++j) {
      k[j] = first(j, lane, wave);
      goff[j] = (unsigned)((row(j, lane, wave) * ld + k[j]) * 2);
    }
  }
  // Numbers k0 .. k0 + BK - 1 of every row; units past K, and rows past the resource's end, arrive as zeros.
  __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rsrc, lds_byte* tile, int k0, int K, int wave) const {
#pragma unroll
    for (int j = 0; j < NLOAD; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(tile + (wave * NLOAD + j) * 1024), 16,
                                               k0 + k[j] < K ? goff[j] + (unsigned)k0 * 2u : 0x7FFFFFF0u, 0, 0, 0);
  }
  // The same of the first `rows` rows of [rows][ld], K = ld, as zeros the rows outside lo .. hi - 1.
  static __device__ __forceinline__ void issue_some(const unsigned short* base, int ld, int rows, int lo, int hi, lds_byte* tile, int k0,
                                                    int lane, int wave) {
    const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(base, (unsigned)(rows * ld * 2));
#pragma unroll
    for (int j = 0; j < NLOAD; ++j) {
      const int r = row(j, lane, wave), at = k0 + first(j, lane, wave);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(tile + (wave * NLOAD + j) * 1024), 16,
                                               r >= lo && r < hi && at < ld ? (unsigned)(r * ld + at) * 2u : 0x7FFFFFF0u, 0, 0, 0);
    }
  }
};
// The 16 bytes that a lane feeds to the matrix unit: row `row`, numbers 16 kc + 8 half ..
template <int BK>
__device__ __forceinline__ u32x4 fragment(const lds_byte* tile, int row, int kc, int half) {
  return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(tile + row * BK * 2 + (turned<BK>(row, kc * 2 + half) << 4));
}

// Lays N instructions of the kinds in MASK (0x100 LDS reads, 0x20 loads) evenly among M of the matrix unit, instead of the
// compiler's order, which reads fragments just before they are multiplied and waits for them.
template <int MASK, int N, int M, int I = 0>
__device__ __forceinline__ void interleave() {
  constexpr int now = N * (I + 1) / M - N * I / M;
  if constexpr (now > 0) __builtin_amdgcn_sched_group_barrier(MASK, now, 0);
  __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
  if constexpr (I + 1 < M) interleave<MASK, N, M, I + 1>();
}

// BM x BN outputs by four wavefronts, each a block of 32 x 32 results TM x TN times.  S steps of BK numbers of the operands are in
// LDS: one is multiplied, the others are on their way.  fp32 results: all three pieces of both operands are there together, and
// their six products are formed from the same fragments (one product after the other, each with tiles of its own, read
// twice as much: the whole call 777 x 1000 -> 1501 96 us, 71 so).
// 16384 x 4096 -> 4096 bf16 without segments 466 us (1.18 PFLOP/s; the library's product of the same numbers 352, 1.56, the matrix
// units alone 2.09), 500-590 with eight segments of rank 16 and whatever else runs around it.  The matrix units work 59 % of the
// cycles, memory and LDS are far from theirs; what they wait for is open: rings of smaller steps, other orders of the loads and
// of the fragments all measured the same, and zeros take 378 us (the library 256).  fp32 4096 x 4096 -> 4096: 0.98 PFLOP/s of its pieces.
template <int OTYPE, int BM, int BN, int BK, int S>
__device__ __forceinline__ void product_tile(const ProductParams& p) {
  constexpr int NW = 4, WN = 2;
  constexpr int TM = BM / 64, TN = BN / 64, NP = OTYPE == LSAM_DTYPE_FP32 ? 3 : 1, NC = BK / 16;
  typedef RowTile<BM, NW, BK> OX;
  typedef RowTile<BN, NW, BK> OW;
  constexpr bool SMALL = NP == 1 && TM * TN == 1;
  static_assert(SMALL ? S == 8 && NC == 4 : S >= 2 && S <= 4, "small tiles have eight stages, others two to four");
  // an array for each stage, so that the compiler knows the one that is read from those that are on their way
  constexpr int PART_W = NP * OX::BYTES, STAGE = NP * (OX::BYTES + OW::BYTES), NL = NP * (OX::NLOAD + OW::NLOAD);
  __shared__ __attribute__((aligned(1024))) unsigned char st0[STAGE];
  __shared__ __attribute__((aligned(1024))) unsigned char st1[STAGE];
  __shared__ __attribute__((aligned(1024))) unsigned char st2[S > 2 ? STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st3[S > 3 ? STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st4[S > 4 ? STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st5[S > 4 ? STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st6[S > 4 ? STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st7[S > 4 ? STAGE : 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const int wm = (wave / WN) * (TM * 32), wn = (wave % WN) * (TN * 32);

  // Workgroups go round the eight XCDs; an XCD takes a run of tiles, eight rows of tiles at a time, so that what runs there
  // together shares the rows of x and W that its L2 holds.
  const unsigned total = (unsigned)p.tilesM * (unsigned)p.tilesN, xcd = blockIdx.x % 8, each = total / 8, more = total % 8;
  const unsigned id = xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8;
  constexpr unsigned kBand = 8;
  const unsigned band = id / (kBand * p.tilesN), in_band = id % (kBand * p.tilesN);
  const unsigned rows_of_band = p.tilesM - band * kBand < kBand ? p.tilesM - band * kBand : kBand;
  const int64_t m0 = (int64_t)(band * kBand + in_band % rows_of_band) * BM;
  const int n0 = (int)(in_band / rows_of_band) * BN;
  const int64_t m_here = p.M - m0 < BM ? p.M - m0 : BM;
  const int n_here = p.N - n0 < BN ? p.N - n0 : BN;

  OX ox;
  OW ow;
  ox.init(p.ldx, lane, wave);
  ow.init(p.ldw, lane, wave);
  const unsigned bytes_x = (unsigned)(((m_here - 1) * p.ldx + p.K) * 2), bytes_w = (unsigned)(((n_here - 1) * p.ldw + p.K) * 2);
  const unsigned short* X = p.X + m0 * p.ldx;
  const unsigned short* W = p.W + (int64_t)n0 * p.ldw;
  lds_byte *const a0 = (lds_byte*)st0, *const a1 = (lds_byte*)st1, *const a2 = (lds_byte*)st2, *const a3 = (lds_byte*)st3;
  lds_byte *const a4 = (lds_byte*)st4, *const a5 = (lds_byte*)st5, *const a6 = (lds_byte*)st6, *const a7 = (lds_byte*)st7;

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // A chunk is 16 numbers of the contraction.
  u32x4 fx[2][NP][TM], fw[2][NP][TN];
  auto read = [&](const lds_byte* tile, int kc, int buf) {
#pragma unroll
    for (int q = 0; q < NP; ++q) {
#pragma unroll
      for (int i = 0; i < TM; ++i) fx[buf][q][i] = fragment<BK>(tile + q * OX::BYTES, wm + i * 32 + l32, kc, half);
#pragma unroll
      for (int j = 0; j < TN; ++j) fw[buf][q][j] = fragment<BK>(tile + PART_W + q * OW::BYTES, wn + j * 32 + l32, kc, half);
    }
  };
  constexpr int PAIRS = NP == 3 ? 6 : 1;
  auto multiply_chunk = [&](int buf) {
#pragma unroll
    for (int q = 0; q < PAIRS; ++q) {
      const unsigned px = NP == 3 ? (kSixLeft >> (4 * q)) & 15u : 0u, pw = NP == 3 ? (kSixRight >> (4 * q)) & 15u : 0u;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma32(fw[buf][pw][j], fx[buf][px][i], acc[i][j]);
    }
  };

  // S - 1 steps are on their way while one is multiplied; behind the last one zeros are, which add nothing, so that the loop
  // runs in whole rounds of the stages and the loads to wait for are as many in every step.
  const int steps = (p.K + BK - 1) / BK;
  int next_k = 0;
  auto request = [&](lds_byte* tile) {
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      ox.issue(make_rsrc(X + q * p.plane_x, bytes_x), tile + q * OX::BYTES, next_k, p.K, wave);
      ow.issue(make_rsrc(W + q * p.plane_w, bytes_w), tile + PART_W + q * OW::BYTES, next_k, p.K, wave);
    }
    next_k = next_k < p.K ? next_k + BK : p.K;
  };
  request(a0);
  request(a1);
  if constexpr (S > 2) request(a2);
  if constexpr (S > 3) request(a3);
  if constexpr (S > 4) { request(a4); request(a5); request(a6); request(a7); }
  arrived<(S - 1) * NL>();
  if constexpr (SMALL) {
    // One block of results a wavefront: too little to multiply while a fragment comes from LDS.  All of the next step's
    // fragments are read while this one's are multiplied, into two sums, so that they do not wait for each other.
    u32x4 gx[2][4], gw[2][4];
    f32x16 other;
#pragma unroll
    for (int e = 0; e < 16; ++e) other[e] = 0.f;
    auto read_all = [&](const lds_byte* tile, int buf) {
#pragma unroll
      for (int kc = 0; kc < 4; ++kc) {
        gx[buf][kc] = fragment<BK>(tile, wm + l32, kc, half);
        gw[buf][kc] = fragment<BK>(tile + PART_W, wn + l32, kc, half);
      }
    };
    read_all(a0, 0);
    auto step = [&](lds_byte* now, lds_byte* then, int buf) {
      arrived<(S - 2) * NL>();
      request(now);
      read_all(then, buf ^ 1);
#pragma unroll
      for (int kc = 0; kc < 4; kc += 2) {
        acc[0][0] = mfma32(gw[buf][kc], gx[buf][kc], acc[0][0]);
        other = mfma32(gw[buf][kc + 1], gx[buf][kc + 1], other);
      }
    };
    for (int s = 0; s < steps; s += S) {
      step(a0, a1, 0);
      step(a1, a2, 1);
      step(a2, a3, 0);
      step(a3, a4, 1);
      step(a4, a5, 0);
      step(a5, a6, 1);
      step(a6, a7, 0);
      step(a7, a0, 1);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[0][0][e] += other[e];
  } else {
    read(a0, 0, 0);
    auto step = [&](lds_byte* now, lds_byte* then) {
#pragma unroll
      for (int c = 0; c + 1 < NC; ++c) {
        read(now, c + 1, (c + 1) & 1);
        multiply_chunk(c & 1);
        interleave<0x100, NP * (TM + TN), PAIRS * TM * TN>();
      }
      // Every wavefront has taken its last fragment of this step, and the next one has arrived.
      arrived<(S - 2) * NL>();
      request(now);
      read(then, 0, 0);                    // behind the last step: never multiplied
      multiply_chunk((NC - 1) & 1);
      interleave<0x120, NP * (TM + TN) + NL, PAIRS * TM * TN>();
    };
    for (int s = 0; s < steps; s += S) {
      step(a0, a1);
      if constexpr (S == 2) {
        step(a1, a0);
      } else {
        step(a1, a2);
        if constexpr (S == 3) {
          step(a2, a0);
        } else {
          step(a2, a3);
          step(a3, a0);
        }
      }
    }
  }
  arrived<0>();                          // nothing may still be on its way to LDS

  // Every segment that rows of the tile belong to: the copies of u and of its adapter, rows of other segments being zeros.  BK
  // numbers of them in each stage, then all stages are multiplied: many segments of few rows would wait one by one.
  const unsigned short* const u = p.u + m0 * p.low_k;
  auto multiply_low = [&](const lds_byte* tile, int k0) {
#pragma unroll
    for (int kc = 0; kc < NC; ++kc) {
      if (k0 + kc * 16 < p.low_k) {
#pragma unroll
        for (int i = 0; i < TM; ++i) fx[0][0][i] = fragment<BK>(tile, wm + i * 32 + l32, kc, half);
#pragma unroll
        for (int j = 0; j < TN; ++j) fw[0][0][j] = fragment<BK>(tile + PART_W, wn + j * 32 + l32, kc, half);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = mfma32(fw[0][0][j], fx[0][0][i], acc[i][j]);
      }
    }
  };
  SegmentsOf walk(p.g, m0, (int)m_here, p.M, p.low_k, BK);
  unsigned marks = 0;                    // whether any of their adapters has a number that is not finite
  while (true) {
    int k[S];
    unsigned mark[S][BN / 64];
#pragma unroll
    for (int i = 0; i < S; ++i) {
      k[i] = -1;
#pragma unroll
      for (int j = 0; j < BN / 64; ++j) mark[i][j] = 0;
      if (!walk.next()) continue;
      lds_byte* const tile = i == 0 ? a0 : i == 1 ? a1 : i == 2 ? a2 : i == 3 ? a3 : i == 4 ? a4 : i == 5 ? a5 : i == 6 ? a6 : a7;
      k[i] = walk.k0;
      OX::issue_some(u, p.low_k, (int)m_here, walk.lo, walk.hi, tile, walk.k0, lane, wave);
      OW::issue_some(p.Q + ((int64_t)walk.copy * p.N + n0) * p.low_k, p.low_k, n_here, 0, n_here, tile + PART_W, walk.k0, lane, wave);
      const unsigned char* const odd = p.odd + (int64_t)walk.copy * p.N + n0;
#pragma unroll
      for (int j = 0; j < BN / 64; ++j) mark[i][j] = odd[j * 64 + lane < n_here ? j * 64 + lane : 0];
    }
    if (k[0] < 0) break;
    arrived<0>();
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int j = 0; j < BN / 64; ++j) marks |= mark[i][j];
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (k[i] >= 0)
        multiply_low(i == 0 ? a0 : i == 1 ? a1 : i == 2 ? a2 : i == 3 ? a3 : i == 4 ? a4 : i == 5 ? a5 : i == 6 ? a6 : a7, k[i]);
    if (walk.done) break;
    arrived<0>();
  }

  typedef Value<OTYPE> VO;
  typedef typename VO::T TO;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = wm + i * 32 + l32;
    if (row < m_here) {
      TO* y = static_cast<TO*>(p.Y) + (m0 + row) * p.ldy + n0;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = wn + j * 32 + q * 8 + half * 4;
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[i][j][q * 4 + e] + (p.bias && col + e < n_here ? p.bias[n0 + col + e] : 0.f);
          if (col + 4 <= n_here) {
            if constexpr (OTYPE == LSAM_DTYPE_BF16) {
              *reinterpret_cast<u16x4_any*>(y + col) = u16x4{narrow(v[0]), narrow(v[1]), narrow(v[2]), narrow(v[3])};
            } else {
              *reinterpret_cast<f32x4_any*>(y + col) = f32x4{v[0], v[1], v[2], v[3]};
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (col + e < n_here) VO::put(y + col + e, v[e]);
          }
        }
    }
  }

  // Outputs that a number of their adapter's belongs to which is not finite: the lane that stored them says so.
  if (__ballot(marks != 0) == 0) return;
  const int found = seg_at(p.g, m0);
  for (int s = found < 0 ? 0 : found; s < p.g.n; ++s) {
    const int64_t l = seg_row(p.g, s, p.M) - m0, h = seg_row(p.g, s + 1, p.M) - m0;
    if (l >= m_here) break;
    const int copy = seg_copy(p.g, s);
    if (copy < 0 || l >= h) continue;
    const unsigned char* odd = p.odd + (int64_t)copy * p.N + n0;
    for (int i = 0; i < TM; ++i) {
      const int row = wm + i * 32 + l32;
      if (row < l || row >= h || row >= m_here) continue;
      TO* y = static_cast<TO*>(p.Y) + (m0 + row) * p.ldy + n0;
      for (int c = 0; c < TN * 16; ++c) {
        const int col = wn + (c >> 4) * 32 + ((c >> 2) & 3) * 8 + half * 4 + (c & 3);
        if (col < n_here && odd[col]) VO::put(y + col, __builtin_nanf(""));
      }
    }
  }
}

template <int OTYPE, int BM, int BN, int BK, int S>
__global__ __launch_bounds__(256) void product_kernel(ProductParams p) {
  product_tile<OTYPE, BM, BN, BK, S>(p);
}

// ---- y or dx, at most 64 rows -----------------------------------------------------------------------
struct FewRowsParams {
  const void* X; int64_t ldx;
  const void* W; int64_t ldw;
  int M, N, K;
  void* Y; int64_t ldy;
  const float* bias;
  const float* u; float scale;
  const void* Q; int64_t q_adapter, q_n, q_r;
  int rank;
  const int* adapter;                                 // of every row
};
constexpr int kFewRows = 64;
constexpr int kHead = 16;                             // ranks that are read ahead

// A workgroup's 16 outputs, the contraction cut over its wavefronts.  Bound by reading W, each workgroup's share of it in one go, and
// by x, which every workgroup reads from L2: 32 rows, 4096 -> 4096 bf16, 34 MB, 13-14 us (2.5 TB/s).  Backward (not UNIT) W's rows
// lie along the outputs and go to the matrix unit as they are: no transposed copy, no copies of the adapters (dx of 8 rows,
// 4096 -> 4096, with du before it: bf16 25 us against 45 in tiles, fp32 53 against 100; 64 rows 31 against 46, 76 against 115).
template <int DTYPE, int RT, bool UNIT>
constexpr int kFewWaves = waves_for(kStageBytes<DTYPE, DTYPE, UNIT, 1, RT>);
constexpr int kNeighbours = 4;                        // workgroups that share the lines of W's rows, in one XCD (not UNIT)

template <int DTYPE, int QTYPE, int RT, int WAVES, bool STAGED, bool UNIT>
__global__ __launch_bounds__(WAVES * 64) void few_rows_kernel(FewRowsParams p) {
  typedef typename Value<DTYPE>::T T;
  typedef typename Value<QTYPE>::T TQ;
  constexpr int STAGE = kStageBytes<DTYPE, DTYPE, UNIT, 1, RT>;
  constexpr int PART = WAVES * RT * 16 * 17 * 4;
  constexpr int FIRST = STAGED && WAVES * STAGE > PART ? WAVES * STAGE : PART;      // the sums go where a stage was
  __shared__ __attribute__((aligned(1024))) unsigned char st0[FIRST];
  __shared__ __attribute__((aligned(1024))) unsigned char st1[STAGED ? WAVES * STAGE : 16];
  __shared__ __attribute__((aligned(1024))) unsigned char st2[STAGED && ring_for(STAGE) > 2 ? WAVES * STAGE : 16];
  float (*part)[RT * 16][17] = reinterpret_cast<float (*)[RT * 16][17]>(st0);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, quarter = lane >> 4;
  const unsigned local = blockIdx.x / 8;
  const unsigned tile = UNIT ? blockIdx.x : (local / kNeighbours * 8 + blockIdx.x % 8) * kNeighbours + local % kNeighbours;
  if (tile >= ((unsigned)p.N + 15) / 16) return;
  const int n0 = (int)tile * 16;
  // This lane's outputs, rows row0 + EACH o of column `col`, and what their low-rank part needs: asked for before W is.
  constexpr int EACH = WAVES * 4, OUT = RT * 16 > EACH ? RT * 16 / EACH : 1;
  const int row0 = tid >> 4, col = n0 + (tid & 15);
  int adapter[OUT];
  float u[OUT][kHead], q[OUT][kHead];
#pragma unroll
  for (int o = 0; o < OUT; ++o) adapter[o] = row0 + o * EACH < p.M ? p.adapter[row0 + o * EACH] : -1;
#pragma unroll
  for (int o = 0; o < OUT; ++o)
#pragma unroll
    for (int e = 0; e < kHead; ++e) {
      const int r = e < p.rank ? e : p.rank - 1;
      u[o][e] = adapter[o] >= 0 && col < p.N ? p.u[(int64_t)(row0 + o * EACH) * p.rank + r] : 0.f;
      q[o][e] = adapter[o] >= 0 && col < p.N
                    ? Value<QTYPE>::get(static_cast<const TQ*>(p.Q) + adapter[o] * p.q_adapter + col * p.q_n + r * p.q_r) : 0.f;
    }
  in_order();
  f32x4 acc[RT][1];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[t][0] = f32x4{0.f, 0.f, 0.f, 0.f};
  const Rows<DTYPE> left{static_cast<const T*>(p.W) + n0 * (UNIT ? p.ldw : 1), UNIT ? p.ldw : 1, UNIT ? 1 : p.ldw, p.N - n0 < 16 ? p.N - n0 : 16};
  const Rows<DTYPE> x{static_cast<const T*>(p.X), p.ldx, 1, p.M};
  if constexpr (STAGED)
    contract_staged<DTYPE, DTYPE, UNIT, 1, RT, WAVES>(left, x, p.K, wave, lane, (lds_byte*)st0 + wave * STAGE, (lds_byte*)st1 + wave * STAGE,
                                                      (lds_byte*)st2 + (ring_for(STAGE) > 2 ? wave * STAGE : 0), acc);
  else
    contract_straight<DTYPE, DTYPE, UNIT, 1, RT, WAVES>(left, x, p.K, wave, lane, acc);
  __syncthreads();
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) part[wave][t * 16 + l16][quarter * 4 + i] = acc[t][0][i];
  __syncthreads();
#pragma unroll
  for (int o = 0; o < OUT; ++o) {
    const int row = row0 + o * EACH;
    if (row >= p.M || row >= RT * 16 || col >= p.N) continue;
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < WAVES; ++v) sum += part[v][row][tid & 15];
    if (adapter[o] >= 0) {
      float low = 0.f;
#pragma unroll
      for (int e = 0; e < kHead; ++e)
        if (e < p.rank) low = __builtin_fmaf(u[o][e], q[o][e], low);
      const TQ* const more = static_cast<const TQ*>(p.Q) + adapter[o] * p.q_adapter + col * p.q_n;
      for (int r = kHead; r < p.rank; ++r) low = __builtin_fmaf(p.u[(int64_t)row * p.rank + r], Value<QTYPE>::get(more + r * p.q_r), low);
      sum = __builtin_fmaf(p.scale, low, sum);
    }
    if (p.bias) sum += p.bias[col];
    Value<DTYPE>::put(static_cast<T*>(p.Y) + row * p.ldy + col, sum);
  }
}

// ---- dA, dB -----------------------------------------------------------------------------------------
struct GradsParams {
  struct Side {
    const void* V; int64_t stride; int cols;           // x or dy
    const float* S;                                    // du or u: [rows][rank]
    float* G; int64_t adapter, col, rank;              // strides of dA or dB
    float scale;
  } side[2];
  int tiles0;                                          // tiles of 64 columns of side 0
  int64_t rows; int rank;
  Segments g;
};
constexpr int kGradWaves = 8;

// G[c][r] = scale sum_t V[t][c] S[t][r] over the rows t of an adapter's segments: 64 columns of one adapter a workgroup, whose
// wavefronts take 32 rows each in turn.  Bound by reading V: 16384 rows of 4096 + 4096 columns bf16, 268 MB, 57-59 us (4.6 TB/s;
// the whole call 75 us with 8 wavefronts, 90 with 4, 100 with 16).  The matrix unit wants eight successive t of a column in a
// lane: a lane loads four neighbouring columns of eight rows and deals them out.
template <int DTYPE, int NR>
__global__ __launch_bounds__(kGradWaves * 64) void grads_kernel(GradsParams p) {
  typedef typename Value<DTYPE>::T T;
  constexpr int PITCH = NR * 16 + 1;
  __shared__ float part[kGradWaves / 2][64][PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, quarter = lane >> 4;
  const bool second = (int)blockIdx.x >= p.tiles0;
  const GradsParams::Side& d = p.side[second ? 1 : 0];
  const int c0 = ((int)blockIdx.x - (second ? p.tiles0 : 0)) * 64, a = blockIdx.y;
  const int c = c0 + l16 * 4, nc = d.cols - c;         // this lane's columns
  f32x4 acc[4][NR];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int r = 0; r < NR; ++r) acc[q][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  const T* V = static_cast<const T*>(d.V) + (nc > 0 ? c : 0);
  int rank[NR];                                        // past the last: the last again, and dropped
#pragma unroll
  for (int r = 0; r < NR; ++r) rank[r] = r * 16 + l16 < p.rank ? r * 16 + l16 : p.rank - 1;
  bool any = false;
  int turn = 0;                                        // pieces of 32 rows go round the wavefronts, from segment to segment
  for (int s0 = 0; s0 < p.g.n; s0 += 64) {
    // 64 segments at a time, a lane each
    const int s = s0 + lane;
    const int begin = s < p.g.n ? (int)seg_row(p.g, s, p.rows) : 0, end = s < p.g.n ? (int)seg_row(p.g, s + 1, p.rows) : 0;
    unsigned long long mine = __ballot(begin < end && p.g.which[s < p.g.n ? s : 0] == a);
    while (mine) {
      const int at = __builtin_ctzll(mine);
      mine &= mine - 1;
      any = true;
      const int64_t lo = __builtin_amdgcn_readlane(begin, at), hi = __builtin_amdgcn_readlane(end, at);
      const int64_t first = lo + ((wave - turn) & (kGradWaves - 1)) * 32;
      turn += (int)((hi - lo + 31) / 32) & (kGradWaves - 1);
      for (int64_t t0 = first; t0 < hi; t0 += kGradWaves * 32) {
        const int64_t t = t0 + quarter * 8;
        const int nt = hi - t < 8 ? (int)(hi - t) : 8;   // rows that are the segment's: others' may hold anything
        typedef T T4 __attribute__((ext_vector_type(4)));
        typedef T4 T4_any __attribute__((aligned(sizeof(T))));
        T4 w[8];
        Pieces<3> fs[NR];
        if (t0 + 32 <= hi && c0 + 64 <= d.cols) {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const T4_any*>(V + (t + j) * d.stride);
#pragma unroll
          for (int r = 0; r < NR; ++r) load8<LSAM_DTYPE_FP32, false>(d.S + t * p.rank + rank[r], p.rank, fs[r]);
        } else {
          // places that are not there: the nearest that is, so that no load depends on a condition, and 0 afterwards
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int64_t row = t + j < hi ? t + j : hi - 1;
            if (c0 + 64 <= d.cols) {
              w[j] = *reinterpret_cast<const T4_any*>(V + row * d.stride);
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q) w[j][q] = V[row * d.stride + (q < nc ? q : nc > 0 ? nc - 1 : 0)];
            }
          }
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = d.S[(t + j < hi ? t + j : hi - 1) * p.rank + rank[r]];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < nt ? v[j] : 0.f;
            split8(v, fs[r]);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j >= nt) w[j] = T4{0, 0, 0, 0};
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          Pieces<kPieces<DTYPE>> fv;
          if constexpr (DTYPE == LSAM_DTYPE_BF16) {
            u16x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = w[j][q];
            fv.p[0] = __builtin_bit_cast(bf16x8, o);
          } else {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = w[j][q];
            split8(o, fv);
          }
#pragma unroll
          for (int r = 0; r < NR; ++r) acc[q][r] = multiply(fv, fs[r], acc[q][r]);
        }
      }
    }
  }
  if (!any) {                                          // the same for the whole workgroup
    for (int i = tid; i < 64 * p.rank; i += kGradWaves * 64) {
      const int col = d.col == 1 ? i % 64 : i / p.rank, r = d.col == 1 ? i / 64 : i % p.rank;
      if (c0 + col < d.cols) d.G[a * d.adapter + (c0 + col) * d.col + r * d.rank] = 0.f;
    }
    return;
  }
  // lane: rank r 16 + l16, column 4 (4 quarter + i) + q.  The upper half of the wavefronts hand over to the lower, twice.
  constexpr int H = kGradWaves / 2;
  if (wave >= H) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave - H][(quarter * 4 + i) * 4 + q][r * 16 + l16] = acc[q][r][i];
  }
  __syncthreads();
  if (wave < H) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][(quarter * 4 + i) * 4 + q][r * 16 + l16] += acc[q][r][i];
  }
  __syncthreads();
  // lanes along what is contiguous in G
  for (int i = tid; i < 64 * p.rank; i += kGradWaves * 64) {
    const int col = d.col == 1 ? i % 64 : i / p.rank, r = d.col == 1 ? i / 64 : i % p.rank;
    if (c0 + col >= d.cols) continue;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < H; ++w) sum += part[w][col][r];
    d.G[a * d.adapter + (c0 + col) * d.col + r * d.rank] = d.scale * sum;
  }
}

// ---- pieces, aligned and transposed copies ----------------------------------------------------------
struct PlanesParams {
  const void* src; int64_t stride; int64_t rows; int cols;
  unsigned short* dst; int64_t ld, plane;              // [pieces][rows][ld], or transposed [pieces][cols][ld]; ld a multiple of 8
};
// The matrix unit wants numbers along the contraction side by side; W of the backward pass has them a row apart: 64 x 64 numbers
// turn in LDS, whole lines in and out.  Bound by memory: 4096 x 4096 bf16, 67 MB, 15 us (4.5 TB/s).
template <int DTYPE, bool TRANSPOSE>
__global__ __launch_bounds__(256) void planes_kernel(PlanesParams p) {
  typedef typename Value<DTYPE>::T T;
  constexpr int NP = kPieces<DTYPE>;
  const int tid = threadIdx.x;
  if constexpr (!TRANSPOSE) {
    const unsigned units = (unsigned)(p.ld / 8);
    const int64_t at = (int64_t)blockIdx.x * 256 + tid, row = at / units;
    const int c = (int)(at - row * units) * 8;
    if (row >= p.rows) return;
    Pieces<NP> o;
    load8_some<DTYPE>(static_cast<const T*>(p.src) + row * p.stride + c, 1, p.cols - c, o);
#pragma unroll
    for (int q = 0; q < NP; ++q) *reinterpret_cast<bf16x8*>(p.dst + q * p.plane + row * p.ld + c) = o.p[q];
  } else {
    __shared__ T tile[64][66];
    const unsigned across = (unsigned)((p.cols + 63) / 64);
    const int64_t r0 = (int64_t)(blockIdx.x / across) * 64;
    const int c0 = (int)(blockIdx.x % across) * 64;
    typedef T T8 __attribute__((ext_vector_type(8)));
    typedef T8 T8_any __attribute__((aligned(sizeof(T))));
    T8 w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t r = r0 + j * 32 + tid / 8;
      const int c = c0 + (tid % 8) * 8;
      const T* src = static_cast<const T*>(p.src) + r * p.stride + c;
      if (r < p.rows && c + 8 <= p.cols) {
        w[j] = *reinterpret_cast<const T8_any*>(src);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[j][e] = r < p.rows && c + e < p.cols ? src[e] : (T)0;
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[j * 32 + tid / 8][(tid % 8) * 8 + e] = w[j][e];
    __syncthreads();
    for (int i = tid; i < 64 * 8; i += 256) {
      const int c = i / 8, r = (i % 8) * 8;
      if (c0 + c >= p.cols || r0 + r >= p.ld) continue;
      Pieces<NP> o;
      if constexpr (DTYPE == LSAM_DTYPE_BF16) {
        u16x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = tile[r + e][c];
        o.p[0] = __builtin_bit_cast(bf16x8, w);
      } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[r + e][c];
        split8(v, o);
      }
#pragma unroll
      for (int q = 0; q < NP; ++q) *reinterpret_cast<bf16x8*>(p.dst + q * p.plane + (int64_t)(c0 + c) * p.ld + r0 + r) = o.p[q];
    }
  }
}

// ---- host -------------------------------------------------------------------------------------------
int64_t up8(int64_t n) { return (n + 7) & ~7ll; }
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Whether rows can go to LDS as they lie: whole aligned units of 16 bytes, tiles within 31 bits.
bool whole_units(const void* p, int64_t stride, int cols, int dtype) {
  const int n = 16 / dtype_bytes(dtype);
  return !misaligned(p, 16) && stride % n == 0 && cols % n == 0 && stride <= 1 << 21;
}
// The same for the tiles of product_kernel, which are bf16.
bool straight(const void* p, int64_t stride, int cols, int dtype) { return dtype == LSAM_DTYPE_BF16 && whole_units(p, stride, cols, dtype); }
// The same from the descriptor alone: what a workspace must be large enough for.
size_t planes_bytes(int64_t rows, int cols, int dtype) { return up256((size_t)(dtype == LSAM_DTYPE_BF16 ? 1 : 3) * rows * up8(cols) * 2); }

// Pieces of u and of the adapter that lose none of their digits: u, or du, is fp32 whatever the result's type is, and so may the
// adapter be; a bfloat16 is its own piece.
LowRank low_rank(const lsam_adapter_desc* d) {
  LowRank l;
  l.rank = d->rank;
  l.padded = (d->rank + 7) & ~7;
  if (d->adapter_dtype == LSAM_DTYPE_FP32) { l.pairs = 6; l.left = kSixLeft; l.right = kSixRight; }
  else { l.pairs = 3; l.left = 0x012u; l.right = 0x000u; }
  return l;
}

// Offsets in the workspace: copies of x or dy and of W, of u and of the adapters, marks, adapters of rows, du.
//
// Few rows of one forward call go to few_rows_kernel, whose workgroups each read all of x from L2 for 16 outputs, or, where that
// costs more than the further launch for the adapters' copies, to product_kernel in tiles of 64 x 64.  us, bf16, one segment of
// rank 16: 4096 -> 4096 19 against 27 for 16 rows and 27 against 28 for 64; 4096 -> 14336 40 against 33 and 82 against 34.  A copy
// has to serve four rows (of the 16, 32, 48 or 64 that the workgroups take): 4096 -> 14336, 16 rows with 4 copies 40 against 36, with 16 40
// against 52; 64 rows with 16 copies 82 against 53, with 64 83 against 104, of rank 64 175 against 144 and 222 against 541.
// Only if x and W go to LDS as they lie: a copy of W would cost more than it brings (fp32, 4096 -> 4096: 58 against 113 us for
// 16 rows, 115 against 127 for 64).
int copies_of(const lsam_adapter_desc* d) { return d->segs < d->adapters ? d->segs : d->adapters; }
struct Layout { size_t x, w, u, q, odd, adapter, du, total; bool tiles, copies; };
Layout layout(const lsam_adapter_desc* d, bool backward) {
  Layout l;
  const int N = backward ? d->in : d->out;
  l.copies = d->rows > kFewRows;
  const int64_t tall = (d->rows + 15) / 16;            // tiles of 16 rows
  l.tiles = l.copies || (!backward && d->dtype == LSAM_DTYPE_BF16 && copies_of(d) <= 4 * tall && (int64_t)N * (tall > 2 ? tall : 2) > 16384);
  l.x = 0;
  l.w = l.x + (l.copies ? planes_bytes(d->rows, backward ? d->out : d->in, d->dtype) : 0);
  // the backward pass reads W transposed
  l.u = l.w + (!l.copies ? 0 : backward ? planes_bytes(d->in, d->out, d->dtype) : planes_bytes(d->out, d->in, d->dtype));
  const size_t low_k = (size_t)low_rank(d).k();
  l.q = l.u + (l.tiles ? up256((size_t)d->rows * low_k * 2) : 0);
  l.odd = l.q + (l.tiles ? up256((size_t)copies_of(d) * N * low_k * 2) : 0);
  l.adapter = l.odd + (l.tiles ? up256((size_t)copies_of(d) * N) : 0);
  l.du = l.adapter + (l.copies ? 0 : up256((size_t)d->rows * 4));
  l.total = l.du + (backward ? up256((size_t)d->rows * d->rank * 4) : 0);
  return l;
}

int check(const lsam_adapter_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype) || !known_dtype(d->adapter_dtype)) return refuse(LSAM_EINVAL, "%s: a dtype is none of LSAM_DTYPE_*", who);
  if (d->rows < 0 || d->rows >= 1ll << 28) return refuse(LSAM_EINVAL, "%s: rows outside 0..2^28-1", who);
  if (d->in < 1 || d->in > 1 << 21 || d->out < 1 || d->out > 1 << 21) return refuse(LSAM_EINVAL, "%s: in and out must be in 1..2^21", who);
  if (d->rank < 1 || d->rank > kMaxRank) return refuse(LSAM_EINVAL, "%s: rank outside 1..LSAM_ADAPTER_MAX_RANK", who);
  if (d->adapters < 0 || d->adapters > 65535 || d->segs < 0) return refuse(LSAM_EINVAL, "%s: adapters outside 0..65535, or segs below 0", who);
  const int64_t wide = d->in > d->out ? d->in : d->out;
  if ((int64_t)d->in * d->out > 1ll << 35 || d->rows * wide > 1ll << 35) return refuse(LSAM_EINVAL, "%s: the matrices are too large", who);
  return LSAM_OK;
}

template <int DTYPE, int ATYPE, bool UNIT, int NR, int RT>
void launch_shrink_tile(const ShrinkParams& p, dim3 grid, bool staged, hipStream_t s) {
  constexpr int waves = kShrinkWaves<DTYPE, ATYPE, UNIT, NR, RT>;
  if (staged) shrink_kernel<DTYPE, ATYPE, UNIT, NR, RT, waves, true><<<grid, waves * 64, 0, s>>>(p);
  else shrink_kernel<DTYPE, ATYPE, UNIT, NR, RT, waves, false><<<grid, waves * 64, 0, s>>>(p);
}
template <int DTYPE, int ATYPE, bool UNIT, int NR>
void launch_shrink_rank(const ShrinkParams& p, hipStream_t s) {
  // Tiles of 64 rows read the adapter least often; of 32 or 16 rows where those leave units idle or segments are short.  Calls
  // with 8 outputs, 4096 -> rank 16 in fp32 adapters, us in tiles of 64 / 32 / 16 rows: 16384 rows 61 / 76 / 104, 8191 47 / 58 / 75,
  // 6144 45 / 41 / 56, 4096 45 / 40 / 41, 1024 44 / 37 / 37; 1024 rows of 512 segments, bf16, 52 / 48 / 45.
  // A launch has less than 2^32 lanes (more wrap, without an error): from 2^26 rows on tiles have 64 whatever the segments are.
  const bool brief = p.rows <= 16ll * p.g.n && p.rows < 1ll << 26;
  const int64_t rows = !brief && p.rows >= 64 * 112 ? 64 : !brief && p.rows >= 32 * 192 ? 32 : 16;
  const int64_t tiles = (p.rows + rows - 1) / rows;
  int64_t y = p.g.n / tiles + 2;                      // two segments meet in many a tile: a workgroup for each
  y = y > 64 ? 64 : y > p.g.n ? (p.g.n > 0 ? p.g.n : 1) : y;
  const dim3 grid((unsigned)tiles, (unsigned)y + 1, (unsigned)(p.rank + NR * 16 - 1) / (NR * 16));
  const bool staged = whole_units(p.x, p.x_stride, p.K, DTYPE) &&
                      (!UNIT || (whole_units(p.A, p.a_rank, p.K, ATYPE) && p.a_adapter % (16 / dtype_bytes(ATYPE)) == 0));
  if (rows == 64) launch_shrink_tile<DTYPE, ATYPE, UNIT, NR, 4>(p, grid, staged, s);
  else if (rows == 32) launch_shrink_tile<DTYPE, ATYPE, UNIT, NR, 2>(p, grid, staged, s);
  else launch_shrink_tile<DTYPE, ATYPE, UNIT, NR, 1>(p, grid, staged, s);
}
// A workgroup has at most 32 ranks, which leaves LDS for more wavefronts to cut fp32's pieces; all 64 where there is nothing to
// cut and many rows would be read twice.  Rank 64, 4096 numbers, calls with 8 outputs, us with 64 / 32 ranks a workgroup: 30 rows
// fp32 120 / 71, bf16 24 / 22; 1024 rows fp32 154 / 98, bf16 35 / 31; 16384 rows fp32 440 / 499, bf16 with fp32 adapters 137 / 101,
// bf16 68 / 93.
template <int DTYPE, int ATYPE, bool UNIT>
void launch_shrink_along(const ShrinkParams& p, hipStream_t s) {
  if (p.rank <= 16) return launch_shrink_rank<DTYPE, ATYPE, UNIT, 1>(p, s);
  if constexpr (DTYPE == LSAM_DTYPE_BF16 && ATYPE == LSAM_DTYPE_BF16)
    if (p.rank > 32 && p.rows >= 64 * 112) return launch_shrink_rank<DTYPE, ATYPE, UNIT, 4>(p, s);
  launch_shrink_rank<DTYPE, ATYPE, UNIT, 2>(p, s);
}
template <int DTYPE, int ATYPE>
void launch_shrink(const ShrinkParams& p, hipStream_t s) {
  if (p.a_k == 1) launch_shrink_along<DTYPE, ATYPE, true>(p, s);
  else launch_shrink_along<DTYPE, ATYPE, false>(p, s);
}
void launch_shrink_any(const ShrinkParams& p, int dtype, int atype, hipStream_t s) {
  if (dtype == LSAM_DTYPE_BF16) {
    if (atype == LSAM_DTYPE_BF16) launch_shrink<LSAM_DTYPE_BF16, LSAM_DTYPE_BF16>(p, s);
    else launch_shrink<LSAM_DTYPE_BF16, LSAM_DTYPE_FP32>(p, s);
  } else {
    if (atype == LSAM_DTYPE_BF16) launch_shrink<LSAM_DTYPE_FP32, LSAM_DTYPE_BF16>(p, s);
    else launch_shrink<LSAM_DTYPE_FP32, LSAM_DTYPE_FP32>(p, s);
  }
}

template <int DTYPE>
void launch_planes(const void* src, int64_t stride, int64_t rows, int cols, bool transpose, unsigned short* dst, hipStream_t s) {
  PlanesParams p;
  p.src = src; p.stride = stride; p.rows = rows; p.cols = cols; p.dst = dst;
  p.ld = up8(transpose ? rows : cols);
  p.plane = (transpose ? cols : rows) * p.ld;
  if (transpose) {
    const int64_t groups = ((rows + 63) / 64) * ((cols + 63) / 64);
    planes_kernel<DTYPE, true><<<(unsigned)groups, 256, 0, s>>>(p);
  } else {
    // a launch has less than 2^32 lanes: more rows take further launches
    const int64_t most = (1ll << 31) / (p.ld / 8);
    for (int64_t r0 = 0; r0 < rows; r0 += most) {
      p.rows = rows - r0 < most ? rows - r0 : most;
      p.src = static_cast<const char*>(src) + r0 * stride * dtype_bytes(DTYPE);
      p.dst = dst + r0 * p.ld;
      const int64_t groups = (p.rows * (p.ld / 8) + 255) / 256;
      planes_kernel<DTYPE, false><<<(unsigned)groups, 256, 0, s>>>(p);
    }
  }
}
void launch_planes_any(const void* src, int64_t stride, int64_t rows, int cols, int dtype, bool transpose, unsigned short* dst, hipStream_t s) {
  if (dtype == LSAM_DTYPE_BF16) launch_planes<LSAM_DTYPE_BF16>(src, stride, rows, cols, transpose, dst, s);
  else launch_planes<LSAM_DTYPE_FP32>(src, stride, rows, cols, transpose, dst, s);
}

template <int OTYPE, int BM, int BN, int BK, int S>
void launch_product_tile(ProductParams p, hipStream_t s) {
  p.tilesM = (int)((p.M + BM - 1) / BM);
  p.tilesN = (p.N + BN - 1) / BN;
  product_kernel<OTYPE, BM, BN, BK, S><<<(unsigned)p.tilesM * (unsigned)p.tilesN, 256, 0, s>>>(p);
}
// Large tiles reuse what they read most, and are taken where they still fill the 256 units; the smaller ones where the next
// larger would leave units idle.  Whole calls, us, in tiles of 256 / 128 / 64 a side, bf16: 16384 x 4096 -> 4096 517 / 635 / 1009,
// 4096 x 2048 -> 3584 (224 tiles of 256) 83 / 105 / 145, 2048 x 2048 -> 3584 (112 of 256, 448 of 128) 73 / 57 / 80,
// 1024 x 2048 -> 1024 (64 of 128) 66 / 32 / 24, and 64 x 4096 -> 65536, whose tiles of 256 are mostly empty, 167 / 152 / 147.
// fp32: 4096 x 4096 -> 4096 819 in tiles of 256 x 128, 868 of 128 x 128; 2048 x 2048 -> 2048 141 of
// 128 x 128, 164 of 128 x 64, 184 of 64 x 64; 777 x 1000 -> 1501 85 of 128 x 128, 71 of 128 x 64, 81 of 64 x 64 (312 tiles: a
// second round for 56 of them); 1024 x 1024 -> 1024 60 of 128 x 64, 53 of 64 x 64.
void launch_product(const ProductParams& p, int dtype, hipStream_t s) {
  auto tiles = [&](int64_t m, int64_t n) { return ((p.M + m - 1) / m) * ((p.N + n - 1) / n); };
  if (dtype == LSAM_DTYPE_BF16) {
    if (p.M > 128 && tiles(256, 256) >= 224) launch_product_tile<LSAM_DTYPE_BF16, 256, 256, 64, 2>(p, s);
    else if (tiles(128, 128) >= 160) launch_product_tile<LSAM_DTYPE_BF16, 128, 128, 64, 4>(p, s);
    else launch_product_tile<LSAM_DTYPE_BF16, 64, 64, 64, 8>(p, s);
  } else {
    if (tiles(64, 64) <= 256) launch_product_tile<LSAM_DTYPE_FP32, 64, 64, 32, 3>(p, s);
    else if (tiles(128, 64) <= 256) launch_product_tile<LSAM_DTYPE_FP32, 128, 64, 32, 3>(p, s);
    else if (p.M <= 128 || tiles(256, 128) < 448) launch_product_tile<LSAM_DTYPE_FP32, 128, 128, 32, 3>(p, s);
    else launch_product_tile<LSAM_DTYPE_FP32, 256, 128, 32, 2>(p, s);
  }
}

template <int DTYPE, int QTYPE, int RT, bool UNIT>
void launch_few_rows_tile(const FewRowsParams& p, hipStream_t s) {
  const unsigned tiles = (unsigned)((p.N + 15) / 16), all = 8 * kNeighbours, grid = UNIT ? tiles : (tiles + all - 1) / all * all;
  constexpr int waves = kFewWaves<DTYPE, RT, UNIT>;
  const bool staged = whole_units(p.X, p.ldx, p.K, DTYPE) && (!UNIT || whole_units(p.W, p.ldw, p.K, DTYPE));
  if (staged) few_rows_kernel<DTYPE, QTYPE, RT, waves, true, UNIT><<<grid, waves * 64, 0, s>>>(p);
  else few_rows_kernel<DTYPE, QTYPE, RT, waves, false, UNIT><<<grid, waves * 64, 0, s>>>(p);
}
template <int DTYPE, int QTYPE, int RT>
void launch_few_rows_along(const FewRowsParams& p, bool transposed, hipStream_t s) {
  if (transposed) launch_few_rows_tile<DTYPE, QTYPE, RT, false>(p, s);
  else launch_few_rows_tile<DTYPE, QTYPE, RT, true>(p, s);
}
template <int DTYPE, int QTYPE>
void launch_few_rows(const FewRowsParams& p, bool transposed, hipStream_t s) {
  if (p.M <= 16) launch_few_rows_along<DTYPE, QTYPE, 1>(p, transposed, s);
  else if (p.M <= 32) launch_few_rows_along<DTYPE, QTYPE, 2>(p, transposed, s);
  else launch_few_rows_along<DTYPE, QTYPE, 4>(p, transposed, s);
}
void launch_few_rows_any(const FewRowsParams& p, bool transposed, int dtype, int qtype, hipStream_t s) {
  if (dtype == LSAM_DTYPE_BF16) {
    if (qtype == LSAM_DTYPE_BF16) launch_few_rows<LSAM_DTYPE_BF16, LSAM_DTYPE_BF16>(p, transposed, s);
    else launch_few_rows<LSAM_DTYPE_BF16, LSAM_DTYPE_FP32>(p, transposed, s);
  } else {
    if (qtype == LSAM_DTYPE_BF16) launch_few_rows<LSAM_DTYPE_FP32, LSAM_DTYPE_BF16>(p, transposed, s);
    else launch_few_rows<LSAM_DTYPE_FP32, LSAM_DTYPE_FP32>(p, transposed, s);
  }
}

template <int DTYPE>
void launch_grads(const GradsParams& p, int adapters, hipStream_t s) {
  const dim3 grid((unsigned)(p.tiles0 + (p.side[1].cols + 63) / 64), (unsigned)adapters);
  if (p.rank <= 16) grads_kernel<DTYPE, 1><<<grid, kGradWaves * 64, 0, s>>>(p);
  else if (p.rank <= 32) grads_kernel<DTYPE, 2><<<grid, kGradWaves * 64, 0, s>>>(p);
  else grads_kernel<DTYPE, 4><<<grid, kGradWaves * 64, 0, s>>>(p);
}

// y = X W'^T + bias + scale u Q: W' is [N][K], or for the backward pass the transposed copy of [K][N].
struct Product {
  const lsam_adapter_desc* d;
  const void* X; int64_t x_stride; int K;
  const void* W; bool transposed; int N;
  void* Y; int64_t y_stride;
  const float* bias; const float* u; float scale;
  const void* Q; int64_t q_adapter, q_n, q_r;
  char* ws; Layout l;
  Segments g;
};
void run_product(const Product& o, hipStream_t s) {
  const lsam_adapter_desc* d = o.d;
  unsigned short* const ws_x = reinterpret_cast<unsigned short*>(o.ws + o.l.x);
  unsigned short* const ws_w = reinterpret_cast<unsigned short*>(o.ws + o.l.w);
  const int64_t ld = up8(o.K);
  if (!o.l.tiles) {
    FewRowsParams p;
    p.X = o.X; p.ldx = o.x_stride; p.W = o.W; p.ldw = d->w_stride;
    p.M = (int)d->rows; p.N = o.N; p.K = o.K; p.Y = o.Y; p.ldy = o.y_stride; p.bias = o.bias; p.u = o.u; p.scale = o.scale;
    p.Q = o.Q; p.q_adapter = o.q_adapter; p.q_n = o.q_n; p.q_r = o.q_r; p.rank = d->rank;
    p.adapter = reinterpret_cast<const int*>(o.ws + o.l.adapter);
    launch_few_rows_any(p, o.transposed, d->dtype, d->adapter_dtype, s);
    return;
  }
  ProductParams p;
  p.M = d->rows; p.N = o.N;
  if (straight(o.X, o.x_stride, o.K, d->dtype)) {
    p.X = static_cast<const unsigned short*>(o.X); p.ldx = o.x_stride; p.plane_x = 0;
  } else {
    launch_planes_any(o.X, o.x_stride, d->rows, o.K, d->dtype, false, ws_x, s);
    p.X = ws_x; p.ldx = ld; p.plane_x = d->rows * ld;
  }
  if (!o.transposed && straight(o.W, d->w_stride, o.K, d->dtype)) {
    p.W = static_cast<const unsigned short*>(o.W); p.ldw = d->w_stride; p.plane_w = 0;
  } else {
    launch_planes_any(o.W, d->w_stride, d->out, d->in, d->dtype, o.transposed, ws_w, s);
    p.W = ws_w; p.ldw = ld; p.plane_w = o.N * ld;
  }
  p.K = (int)ld;                                      // where that is more than K, both are copies, padded with zeros
  p.Y = o.Y; p.ldy = o.y_stride; p.bias = o.bias; p.g = o.g;
  const LowRank low = low_rank(d);
  p.low_k = low.k();
  p.u = reinterpret_cast<const unsigned short*>(o.ws + o.l.u);          // written by shrink_kernel
  unsigned short* const q = reinterpret_cast<unsigned short*>(o.ws + o.l.q);
  unsigned char* const odd = reinterpret_cast<unsigned char*>(o.ws + o.l.odd);
  p.Q = q; p.odd = odd;
  if (o.g.n > 0) {
    const CopiesParams c{o.Q, o.q_adapter, o.q_n, o.q_r, q, odd, o.N, p.low_k, low, o.g, d->rows};
    const dim3 grid((unsigned)(o.N + 255) / 256, (unsigned)copies_of(d));
    if (d->adapter_dtype == LSAM_DTYPE_BF16) copies_kernel<LSAM_DTYPE_BF16><<<grid, 256, 0, s>>>(c);
    else copies_kernel<LSAM_DTYPE_FP32><<<grid, 256, 0, s>>>(c);
  }
  launch_product(p, d->dtype, s);
}

Segments segments(const lsam_adapter_desc* d, const int32_t* begin, const int32_t* which) {
  Segments g;
  g.begin = begin; g.which = which; g.n = d->adapters > 0 ? d->segs : 0; g.adapters = d->adapters;
  g.each = d->segs < d->adapters;
  return g;
}

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" size_t lsam_adapter_workspace_bytes(const lsam_adapter_desc* d, int32_t backward) {
  return check(d, "adapter") == LSAM_OK ? layout(d, backward != 0).total : 0;
}

extern "C" int lsam_adapter(const lsam_adapter_desc* d, const void* x, const void* W, const float* bias, const void* A, const void* B,
                            const int32_t* seg_begin, const int32_t* seg_adapter, float* u, void* y, void* workspace,
                            size_t workspace_bytes, void* stream) {
  int rc = check(d, "adapter");
  if (rc != LSAM_OK) return rc;
  if (d->rows == 0) return LSAM_OK;
  const int b = dtype_bytes(d->dtype), ba = dtype_bytes(d->adapter_dtype);
  const Arg args[] = {
      matrices("x", x, 1, 0, d->rows, d->x_stride, d->in, b, false),
      matrices("W", W, 1, 0, d->out, d->w_stride, d->in, b, false),
      {"bias", bias, bias ? d->out * 4ll : 0, 4, false},
      matrices("A", A, d->adapters, d->a_adapter, d->rank, d->a_stride, d->in, ba, false),
      matrices("B", B, d->adapters, d->b_adapter, d->out, d->b_stride, d->rank, ba, false),
      {"seg_begin", seg_begin, d->segs ? (d->segs + 1) * 4ll : 0, 4, false},
      {"seg_adapter", seg_adapter, d->segs * 4ll, 4, false},
      {"u", u, d->rows * d->rank * 4, 4, true},
      matrices("y", y, 1, 0, d->rows, d->y_stride, d->out, b, true)};
  constexpr int n = sizeof args / sizeof args[0];
  Layout l = layout(d, false);
  rc = check_values(args, n, "adapter");
  if (rc == LSAM_OK) rc = check_apart(args, n, "adapter");
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, l.total, 256, "adapter");
  if (rc != LSAM_OK) return rc;
  if (!l.copies && !(straight(x, d->x_stride, d->in, d->dtype) && straight(W, d->w_stride, d->in, d->dtype))) l.tiles = false;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Segments g = segments(d, seg_begin, seg_adapter);
  const LowRank low = low_rank(d);
  unsigned short* const copy = l.tiles ? reinterpret_cast<unsigned short*>(static_cast<char*>(workspace) + l.u) : nullptr;
  launch_shrink_any(ShrinkParams{x, d->x_stride, A, d->a_adapter, d->a_stride, 1, u, d->rows, d->in, d->rank, 1.f, copy, d->scale, low,
                                 low.k(), l.tiles ? nullptr : reinterpret_cast<int*>(static_cast<char*>(workspace) + l.adapter), g}, d->dtype, d->adapter_dtype, s);
  run_product(Product{d, x, d->x_stride, d->in, W, false, d->out, y, d->y_stride, bias, u, d->scale, B, d->b_adapter, d->b_stride, 1,
                      static_cast<char*>(workspace), l, g}, s);
  return launched();
}

extern "C" int lsam_adapter_backward(const lsam_adapter_desc* d, const void* x, const void* W, const void* A, const void* B,
                                     const int32_t* seg_begin, const int32_t* seg_adapter, const float* u, const void* dy, void* dx,
                                     float* dA, float* dB, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d, "adapter_backward");
  if (rc != LSAM_OK) return rc;
  if ((dA == nullptr) != (dB == nullptr)) return refuse(LSAM_EINVAL, "adapter_backward: dA and dB are wanted together");
  const int b = dtype_bytes(d->dtype), ba = dtype_bytes(d->adapter_dtype);
  Arg args[] = {
      matrices("x", x, 1, 0, dA ? d->rows : 0, d->x_stride, d->in, b, false),
      matrices("W", W, 1, 0, dx && d->rows ? d->out : 0, d->w_stride, d->in, b, false),
      matrices("A", A, d->rows ? d->adapters : 0, d->a_adapter, d->rank, d->a_stride, d->in, ba, false),
      matrices("B", B, d->rows ? d->adapters : 0, d->b_adapter, d->out, d->b_stride, d->rank, ba, false),
      {"seg_begin", seg_begin, d->segs ? (d->segs + 1) * 4ll : 0, 4, false},
      {"seg_adapter", seg_adapter, d->segs * 4ll, 4, false},
      {"u", u, dA ? d->rows * d->rank * 4 : 0, 4, false},
      matrices("dy", dy, 1, 0, d->rows, d->dy_stride, d->out, b, false),
      matrices("dx", dx, 1, 0, dx ? d->rows : 0, d->dx_stride, d->in, b, true),
      matrices("dA", dA, dA ? d->adapters : 0, d->da_adapter, d->rank, d->da_stride, d->in, 4, true),
      matrices("dB", dB, dB ? d->adapters : 0, d->db_adapter, d->out, d->db_stride, d->rank, 4, true)};
  if (dA && !apart(d->adapters, d->da_adapter, d->rank, d->da_stride, d->in)) args[9].bytes = -1;
  if (dB && !apart(d->adapters, d->db_adapter, d->out, d->db_stride, d->rank)) args[10].bytes = -1;
  constexpr int n = sizeof args / sizeof args[0];
  const Layout l = layout(d, true);
  rc = check_values(args, n, "adapter_backward");
  if (rc == LSAM_OK) rc = check_apart(args, n, "adapter_backward");
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, l.total, 256, "adapter_backward");
  if (rc != LSAM_OK) return rc;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const Segments g = segments(d, seg_begin, seg_adapter);
  const LowRank low = low_rank(d);
  float* const du = reinterpret_cast<float*>(static_cast<char*>(workspace) + l.du);
  unsigned short* const copy = dx && l.tiles ? reinterpret_cast<unsigned short*>(static_cast<char*>(workspace) + l.u) : nullptr;
  int* const adapter = dx && !l.tiles ? reinterpret_cast<int*>(static_cast<char*>(workspace) + l.adapter) : nullptr;
  if (d->rows > 0)
    launch_shrink_any(ShrinkParams{dy, d->dy_stride, B, d->b_adapter, 1, d->b_stride, du, d->rows, d->out, d->rank, d->scale, copy, 1.f, low,
                                   low.k(), adapter, g}, d->dtype, d->adapter_dtype, s);
  if (dx && d->rows > 0)
    run_product(Product{d, dy, d->dy_stride, d->out, W, true, d->in, dx, d->dx_stride, nullptr, du, 1.f, A, d->a_adapter, 1, d->a_stride,
                        static_cast<char*>(workspace), l, g}, s);
  if (dA && d->adapters > 0) {
    GradsParams p;
    p.side[0] = {x, d->x_stride, d->in, du, dA, d->da_adapter, 1, d->da_stride, 1.f};
    p.side[1] = {dy, d->dy_stride, d->out, u, dB, d->db_adapter, d->db_stride, 1, d->scale};
    p.tiles0 = (d->in + 63) / 64;
    p.rows = d->rows; p.rank = d->rank; p.g = g;
    if (d->dtype == LSAM_DTYPE_BF16) launch_grads<LSAM_DTYPE_BF16>(p, d->adapters, s);
    else launch_grads<LSAM_DTYPE_FP32>(p, d->adapters, s);
  }
  return launched();
}
