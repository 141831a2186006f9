// lsam_recurrence, lsam_recurrence_backward: h_t = a_t h_{t-1} + (1 - a_t) x_t, a_t = sigmoid(f_t), for every channel of
// every sequence, and its gradient.
//
// A run of steps maps the state that enters it to A h + H, A the product of its a_t and H what it makes of 0; runs
// are joined by (A, H) then (A', H') = (A A', A' H + H').  A workgroup owns 64 neighbouring channels of a sequence and
// goes along time in tiles: each wavefront takes a few rows of the tile into registers (a channel a lane), finds
// its own (A, H), and from those of the wavefronts before it, exchanged through LDS, the state that enters its rows.
// So every value is read once and written once.  Where sequences and channels are too few to fill the chip, the
// tiles of a sequence are cut into runs for several workgroups: a first launch leaves (A, H) of every run.
//
// Backward: with e_t = a_t (dh_t + e_{t+1}) -- what step t hands to the one before it, the same kind of recurrence from
// the other end -- d_t = dh_t + e_{t+1},  dx_t = (1 - a_t) d_t,  df_t = a_t (1 - a_t) d_t (h_{t-1} - x_t).
// The h_{t-1} are formed again, in fp32, from the state that the forward pass saved at the head of each tile (128 rows, 16 with one wavefront).
#include "ops.h"

namespace lsam {
namespace {

// Rows of a tile that one wavefront takes, and wavefronts of a workgroup (one where sequences are no longer than its rows, packed ones on the average).
// 8 x 4096 x 2048 bf16 forward and backward take 252 us with 16 rows and 8 wavefronts, 318 with 8 rows, 289 with 8 rows and 16
// wavefronts, 456 with 16 and 16 (too few registers); a tile more on its way 250, at twice the registers.
constexpr int kRows = 16;
constexpr int kWaves = 8;
constexpr int kChannels = 64;        // of a workgroup: one for each lane
constexpr int kMaxSplits = 64;
// Workgroups of neighbouring channels that share an XCD.  4 x 2000 x 1001 fp32 36 us against 44 where each is on its own,
// 8 x 4096 x 1001 bf16 70 against 100; no difference where rows begin on lines; 4 and 16 as 8.
constexpr int kTogether = 8;

struct Tensor { const void* p; int64_t stride, seq; };

struct RecurrenceParams {
  Tensor f, x, h, dh, df, dx;
  const int64_t* offsets;            // packed sequences: seqs + 1 row numbers, else null
  int64_t seq0, rows, D;             // rows of each sequence, or of all
  unsigned seqs;                     // of this launch
  int64_t tiles_of_each;             // saved states of a sequence (not packed)
  int splits, slabs;
  int64_t run_tiles;                 // tiles of a run
  const float* h0; float* last; float* states;
  const float* dlast; float* dh0;
  float* runs;                       // [seqs][splits][2][D]: A and H (or E) of every run
};

// a = sigmoid(f) and 1 - a, neither from the other: both keep their digits where they are small.
__device__ __forceinline__ void gates(float f, float& a, float& b) {
  const float e = __expf(-__builtin_fabsf(f)), r = __builtin_amdgcn_rcpf(1.f + e), small = e * r;
  a = f >= 0.f ? r : small;
  b = f >= 0.f ? small : r;
}

// A = the product of gates: where it underflows although all of them are positive, the smallest number above 0 stands for it, so
// that an infinite state passes a run as it passes its steps (0 x inf would be NaN).
constexpr float kLeast = 0x1p-149f;
__device__ __forceinline__ float product_of(const float (&a)[kRows]) {
  float A = 1.f;
#pragma unroll
  for (int i = 0; i < kRows; ++i) A *= a[i];
  if (A == 0.f) {
    float least = a[0];
#pragma unroll
    for (int i = 1; i < kRows; ++i) least = __builtin_fminf(least, a[i]);
    A = least > 0.f ? kLeast : 0.f;
  }
  return A;
}
__device__ __forceinline__ float product_of(float A, float B) {
  const float AB = A * B;
  return AB == 0.f && A > 0.f && B > 0.f ? kLeast : AB;
}

// kRows rows of a tensor from row t0 on, zeros for rows that are not there.  The usual case, all rows there, is a run of
// loads that nothing waits between.
template <typename T>
__device__ __forceinline__ void load_rows(T (&r)[kRows], const T* p, int64_t stride, int64_t t0, int64_t len) {
  if (t0 >= 0 && t0 + kRows <= len) {
    const T* q = p + t0 * stride;
#pragma unroll
    for (int i = 0; i < kRows; ++i) r[i] = q[i * stride];
  } else {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      r[i] = 0;
      if (t0 + i >= 0 && t0 + i < len) r[i] = p[(t0 + i) * stride];
    }
  }
}
template <int DTYPE>
__device__ __forceinline__ void store_rows(const float (&v)[kRows], typename Value<DTYPE>::T* p, int64_t stride, int64_t t0,
                                           int64_t len, bool mine) {
  if (!mine) return;
  if (t0 >= 0 && t0 + kRows <= len) {
    typename Value<DTYPE>::T* q = p + t0 * stride;
#pragma unroll
    for (int i = 0; i < kRows; ++i) Value<DTYPE>::put(q + i * stride, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kRows; ++i)
      if (t0 + i >= 0 && t0 + i < len) Value<DTYPE>::put(p + (t0 + i) * stride, v[i]);
  }
}
__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(unsigned short v) { return widen(v); }

// Where a workgroup's sequence lies and which of its tiles are the workgroup's.
struct Place {
  int64_t seq, begin, len;      // begin: row number in packed tensors
  int64_t phase, state0;        // tile j: rows j R - phase ..; its saved state: states[state0 + j], j > 0
  int64_t first, end;           // tiles of this workgroup's run
  int split, last;              // number of the run, and of the sequence's last one
  bool here;                    // there is such a workgroup
  int64_t ch; bool mine;        // this lane's channel; a lane without one reads the last and keeps nothing
  template <typename T>
  __device__ __forceinline__ T* at(const Tensor& t) const {
    return static_cast<T*>(const_cast<void*>(t.p)) + seq * t.seq + begin * t.stride + ch;
  }
};

template <int R>
__device__ __forceinline__ Place place(const RecurrenceParams& p) {
  Place w;
  // Workgroups go round the eight XCDs in turn.  kTogether neighbours of a run meet in one XCD, whose L2 then serves the
  // lines that two of them read where rows do not begin on lines.
  const unsigned per_run = ((unsigned)p.slabs + kTogether - 1) / kTogether, local = blockIdx.x / 8;
  const unsigned unit = local / kTogether * 8 + blockIdx.x % 8, rest = unit / per_run;
  const unsigned slab = unit % per_run * kTogether + local % kTogether;
  w.split = (int)(rest % (unsigned)p.splits);
  const unsigned seq = rest / (unsigned)p.splits;
  w.seq = p.seq0 + seq;
  w.here = seq < p.seqs && slab < (unsigned)p.slabs;
  if (!w.here) return w;
  w.begin = 0;
  w.len = p.rows;
  w.phase = 0;
  w.state0 = w.seq * p.tiles_of_each;
  if (p.offsets) {
    // whatever the offsets hold, no row outside the tensors is touched
    int64_t b = p.offsets[w.seq], e = p.offsets[w.seq + 1];
    b = b < 0 ? 0 : b > p.rows ? p.rows : b;
    e = e < b ? b : e > p.rows ? p.rows : e;
    w.begin = b;
    w.len = e - b;
    w.phase = b % R;
    w.state0 = b / R;
  }
  const int64_t tiles = w.len > 0 ? (w.phase + w.len + R - 1) / R : 0;
  w.last = tiles > 0 ? (int)((tiles - 1) / p.run_tiles) : 0;
  w.first = w.split * p.run_tiles;
  w.end = w.first + p.run_tiles < tiles ? w.first + p.run_tiles : tiles;
  const int64_t ch = (int64_t)slab * kChannels + (threadIdx.x & 63);
  w.mine = ch < p.D;
  w.ch = w.mine ? ch : p.D - 1;
  return w;
}

// RUNS: only (A, H) of the workgroup's run, for a launch that follows.
// 8 x 4096 x 2048 bf16, 403 MB, 100-105 us: 3.9 TB/s, the vector units half busy.  A lane moves two bytes an instruction, and a tile
// more on its way brings 1 %: likely bound by the address unit, which takes such narrow accesses no faster than wide ones.  131073 x
// 1000 fp32 in runs, 1.05 GB read for the runs in 225-230 us and 1.57 GB in 322-349 us (4.5-4.9 TB/s), rows of 4000 bytes that do
// not begin on lines.
template <int DTYPE, int NW, bool RUNS>
__global__ __launch_bounds__(NW * 64) void recurrence_kernel(RecurrenceParams p) {
  typedef typename Value<DTYPE>::T T;
  constexpr int R = NW * kRows;
  __shared__ float shA[2][NW][64], shH[2][NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place w = place<R>(p);
  if (!w.here || w.split > w.last) return;
  const T* f = w.at<const T>(p.f);
  const T* x = w.at<const T>(p.x);
  T* h = RUNS ? nullptr : w.at<T>(p.h);
  float carry = 0.f, whole = 1.f;
  if constexpr (!RUNS) {
    if (p.h0) carry = p.h0[w.seq * p.D + w.ch];
    for (int q = 0; q < w.split; ++q) {
      const float* run = p.runs + (w.seq * p.splits + q) * 2 * p.D + w.ch;
      carry = run[0] * carry + run[p.D];
    }
  }
  T rf[kRows], rx[kRows];
  auto fetch = [&](int64_t j) {
    const int64_t t0 = j * R - w.phase + wave * kRows, len = j < w.end ? w.len : 0;
    load_rows(rf, f, p.f.stride, t0, len);
    load_rows(rx, x, p.x.stride, t0, len);
  };
  fetch(w.first);
  int b = 0;
  for (int64_t j = w.first; j < w.end; ++j) {
    const int64_t t0 = j * R - w.phase + wave * kRows;
    float a[kRows], v[kRows], H = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      float k;
      gates(wide(rf[i]), a[i], k);
      v[i] = k * wide(rx[i]);
    }
    fetch(j + 1);
    if (t0 < 0 || t0 + kRows > w.len) {
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (t0 + i < 0 || t0 + i >= w.len) { a[i] = 1.f; v[i] = 0.f; }      // outside the sequence the state stays
    }
    const float A = product_of(a);
#pragma unroll
    for (int i = 0; i < kRows; ++i) H = a[i] * H + v[i];
    if constexpr (!RUNS)
      if (wave == 0 && p.states && j > 0 && w.mine) p.states[(w.state0 + j) * p.D + w.ch] = carry;
    float s = carry;
    if constexpr (NW > 1) {
      shA[b][wave][lane] = A;
      shH[b][wave][lane] = H;
      __syncthreads();
#pragma unroll
      for (int q = 0; q < NW; ++q) {
        const float qa = shA[b][q][lane];
        if (q == wave) s = carry;
        carry = qa * carry + shH[b][q][lane];
        if constexpr (RUNS) whole = product_of(whole, qa);
      }
      b ^= 1;
    } else {
      carry = A * carry + H;
      if constexpr (RUNS) whole = product_of(whole, A);
    }
    if constexpr (!RUNS) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) v[i] = s = a[i] * s + v[i];
      store_rows<DTYPE>(v, h, p.h.stride, t0, w.len, w.mine);
    }
  }
  if (wave != 0 || !w.mine) return;
  if constexpr (RUNS) {
    float* run = p.runs + (w.seq * p.splits + w.split) * 2 * p.D + w.ch;
    run[0] = whole;
    run[p.D] = carry;
  } else if (w.split == w.last && p.last) {
    p.last[w.seq * p.D + w.ch] = carry;
  }
}

// RUNS: only (A, E) of the workgroup's run.
// 8 x 4096 x 2048 bf16, 671 MB, 152-155 us (4.4 TB/s), bound as the forward pass is; 131073 x 1000 fp32, 1.05 GB for the runs in
// 225-242 us and 2.62 GB in 546-555 us (4.8 TB/s).
template <int DTYPE, int NW, bool RUNS>
__global__ __launch_bounds__(NW * 64) void recurrence_grad_kernel(RecurrenceParams p) {
  typedef typename Value<DTYPE>::T T;
  constexpr int R = NW * kRows;
  __shared__ float shA[2][NW][64], shE[2][NW][64], shH[2][NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place w = place<R>(p);
  if (!w.here || w.split > w.last) return;
  const T* f = w.at<const T>(p.f);
  const T* x = RUNS ? nullptr : w.at<const T>(p.x);
  const T* dh = w.at<const T>(p.dh);
  T* df = RUNS ? nullptr : w.at<T>(p.df);
  T* dx = RUNS ? nullptr : w.at<T>(p.dx);
  float carry = 0.f, whole = 1.f;
  if constexpr (!RUNS) {
    if (p.dlast) carry = p.dlast[w.seq * p.D + w.ch];
    for (int q = w.last; q > w.split; --q) {
      const float* run = p.runs + (w.seq * p.splits + q) * 2 * p.D + w.ch;
      carry = run[0] * carry + run[p.D];
    }
  }
  T rf[kRows], rx[kRows], rd[kRows];
  float entry = 0.f;
  auto fetch = [&](int64_t j) {
    const int64_t t0 = j * R - w.phase + wave * kRows, len = j >= w.first ? w.len : 0;
    load_rows(rf, f, p.f.stride, t0, len);
    if constexpr (!RUNS) load_rows(rx, x, p.x.stride, t0, len);
    load_rows(rd, dh, p.dh.stride, t0, len);
    if constexpr (!RUNS) {
      entry = 0.f;
      if (len > 0 && j > 0) entry = p.states[(w.state0 + j) * p.D + w.ch];
      else if (len > 0 && p.h0) entry = p.h0[w.seq * p.D + w.ch];
    }
  };
  if (w.end > w.first) fetch(w.end - 1);
  int b = 0;
  for (int64_t j = w.end - 1; j >= w.first; --j) {
    const int64_t t0 = j * R - w.phase + wave * kRows;
    float a[kRows], k[kRows], xv[kRows], d[kRows], E = 0.f, H = 0.f, s = entry;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      gates(wide(rf[i]), a[i], k[i]);
      if constexpr (!RUNS) xv[i] = wide(rx[i]);
      d[i] = wide(rd[i]);
    }
    fetch(j - 1);
    if (t0 < 0 || t0 + kRows > w.len) {
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (t0 + i < 0 || t0 + i >= w.len) { a[i] = 1.f; k[i] = 0.f; }
    }
    const float A = product_of(a);
    if constexpr (!RUNS) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) H = a[i] * H + k[i] * xv[i];
    }
#pragma unroll
    for (int i = kRows - 1; i >= 0; --i) E = a[i] * (d[i] + E);
    float e = carry;
    if constexpr (NW > 1) {
      shA[b][wave][lane] = A;
      shE[b][wave][lane] = E;
      if constexpr (!RUNS) shH[b][wave][lane] = H;
      __syncthreads();
#pragma unroll
      for (int q = NW - 1; q >= 0; --q) {
        const float qa = shA[b][q][lane];
        if (q == wave) e = carry;
        carry = qa * carry + shE[b][q][lane];
        if constexpr (RUNS) whole = product_of(whole, qa);
      }
      if constexpr (!RUNS) {
#pragma unroll
        for (int q = 0; q < NW - 1; ++q)
          if (q < wave) s = shA[b][q][lane] * s + shH[b][q][lane];
      }
      b ^= 1;
    } else {
      carry = A * carry + E;
      if constexpr (RUNS) whole = product_of(whole, A);
    }
    if constexpr (!RUNS) {
      float g[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        g[i] = s - xv[i];
        s = a[i] * s + k[i] * xv[i];
      }
#pragma unroll
      for (int i = kRows - 1; i >= 0; --i) {
        const float whole_d = d[i] + e, kd = k[i] * whole_d;
        g[i] *= a[i] * kd;
        d[i] = kd;
        e = a[i] * whole_d;
      }
      store_rows<DTYPE>(d, dx, p.dx.stride, t0, w.len, w.mine);
      store_rows<DTYPE>(g, df, p.df.stride, t0, w.len, w.mine);
    }
  }
  if (wave != 0 || !w.mine) return;
  if constexpr (RUNS) {
    float* run = p.runs + (w.seq * p.splits + w.split) * 2 * p.D + w.ch;
    run[0] = whole;
    run[p.D] = carry;
  } else if (w.split == 0 && p.dh0) {
    p.dh0[w.seq * p.D + w.ch] = carry;
  }
}

// One step of every sequence (generation): eight channels a lane.  Bound by the launch: 64 x 4096 take 3.2 us, 9.7 where
// workgroups of one wavefront walk tiles of which one row is there.
template <int DTYPE>
__global__ __launch_bounds__(256) void recurrence_step_kernel(RecurrenceParams p) {
  typedef Value<DTYPE> V;
  typedef typename V::T T;
  const unsigned pieces = (unsigned)((p.D + 7) / 8);
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, seq = at / pieces, ch = (at - seq * pieces) * 8;
  if (seq >= p.seqs) return;
  const int64_t q = p.seq0 + seq, state = q * p.D + ch;
  const T* f = static_cast<const T*>(p.f.p) + q * p.f.seq + ch;
  const T* x = static_cast<const T*>(p.x.p) + q * p.x.seq + ch;
  T* h = static_cast<T*>(const_cast<void*>(p.h.p)) + q * p.h.seq + ch;
  const int n = p.D - ch < 8 ? (int)(p.D - ch) : 8;
  float vf[8], vx[8], s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (n == 8) {
    V::load8(f, vf);
    V::load8(x, vx);
    if (p.h0) Value<LSAM_DTYPE_FP32>::load8(p.h0 + state, s);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      vf[e] = e < n ? V::get(f + e) : 0.f;
      vx[e] = e < n ? V::get(x + e) : 0.f;
      if (p.h0 && e < n) s[e] = p.h0[state + e];
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float a, b;
    gates(vf[e], a, b);
    s[e] = a * s[e] + b * vx[e];
  }
  if (n == 8) {
    V::store8(h, s);
    if (p.last) Value<LSAM_DTYPE_FP32>::store8(p.last + state, s);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) {
        V::put(h + e, s[e]);
        if (p.last) p.last[state + e] = s[e];
      }
  }
}

// How a call is cut.  One wavefront where sequences are no longer than its rows, packed ones on the average.  Runs where sequences
// times channels give fewer workgroups than there are units: all of one length, so that below that number sequences of any
// lengths fill the chip evenly, as many as give it kRunGroups workgroups, of at least four tiles each (131073 x 1000 fp32, both
// directions: 1330-1360 us with 1024, 1350 with 2048; 1 x 32768 x 4096 bf16 forward 310, 309 with 512).  The lengths of packed
// sequences are not known here: where there are workgroups enough a long one among many short ones is walked by its own alone (64
// sequences x 256 channels bf16, one of half the rows, 307 us forward, of equal lengths 27; 255 of one row and one of 4000, 4096 channels,
// 260, one sequence of as many rows 51).
constexpr int kRunGroups = 1024;
struct Plan { int waves, splits, slabs; int64_t run_tiles, tiles_of_each, states; };
Plan plan(const lsam_recurrence_desc* d) {
  Plan c;
  const int64_t mean = d->packed ? (d->seqs ? (d->rows + d->seqs - 1) / d->seqs : 0) : d->rows;
  c.waves = mean <= kRows ? 1 : kWaves;
  const int64_t R = (int64_t)c.waves * kRows;
  c.slabs = (int)((d->dim + kChannels - 1) / kChannels);
  c.tiles_of_each = d->packed ? 0 : (d->rows + R - 1) / R;
  c.states = d->packed ? d->rows / R + 1 : d->seqs * c.tiles_of_each;
  // the most tiles a sequence can have (a packed one may begin and end inside a tile), and those of all together
  const int64_t most = d->packed ? d->rows / R + 2 : c.tiles_of_each, all = d->packed ? most : d->seqs * most;
  c.run_tiles = most > 0 ? most : 1;
  c.splits = 1;
  if (d->seqs * c.slabs < 256 && most > 4) {
    int64_t tiles = (all * c.slabs + kRunGroups - 1) / kRunGroups;
    if (tiles < (most + kMaxSplits - 1) / kMaxSplits) tiles = (most + kMaxSplits - 1) / kMaxSplits;
    c.run_tiles = tiles < 4 ? 4 : tiles;
    c.splits = (int)((most + c.run_tiles - 1) / c.run_tiles);
  }
  return c;
}

int check(const lsam_recurrence_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype)) return refuse(LSAM_EINVAL, "%s: dtype %d is none of LSAM_DTYPE_*", who, d->dtype);
  if (d->packed != 0 && d->packed != 1) return refuse(LSAM_EINVAL, "%s: packed is neither 0 nor 1", who);
  if (d->seqs < 0 || d->seqs >= 1ll << 31 || d->rows < 0 || d->rows >= 1ll << 40 || d->dim < 1 || d->dim >= 1ll << 28)
    return refuse(LSAM_EINVAL, "%s: seqs must be in 0..2^31-1, rows in 0..2^40-1, dim in 1..2^28-1", who);
  const __int128 all = (__int128)(d->packed ? 1 : d->seqs) * d->rows * d->dim, state = (__int128)d->seqs * d->dim;
  if (all >= (__int128)1 << 44 || state >= (__int128)1 << 40) return refuse(LSAM_EINVAL, "%s: the arrays are too large", who);
  return LSAM_OK;
}

// A tensor as an argument; sequences of an output have to lie apart from each other.
Arg arg(const lsam_recurrence_desc* d, const char* name, const void* p, const lsam_rows& t, bool output) {
  const int64_t mats = d->packed ? 1 : d->seqs;
  Arg a = matrices(name, p, mats, t.seq, d->rows, t.stride, d->dim, dtype_bytes(d->dtype), output);
  if (output && !apart(mats, t.seq, d->rows, t.stride, d->dim)) a.bytes = -1;
  return a;
}

Tensor tensor(const void* p, const lsam_rows& r, bool packed) { return Tensor{p, r.stride, packed ? 0 : r.seq}; }

template <int DTYPE, int NW, bool GRAD>
void launch(RecurrenceParams p, int64_t seqs, hipStream_t s) {
  // a launch has less than 2^32 lanes: more sequences take further launches
  const int64_t per_run = (p.slabs + kTogether - 1) / kTogether;
  const int64_t most = ((1ll << 31) / (NW * 64)) / (p.splits * per_run * kTogether) - 8;
  const int64_t step = most < 1 ? 1 : most;
  for (int64_t s0 = 0; s0 < seqs; s0 += step) {
    p.seq0 = s0;
    p.seqs = (unsigned)(seqs - s0 < step ? seqs - s0 : step);
    const unsigned grid = (unsigned)((p.seqs * p.splits * per_run + 7) / 8 * 8 * kTogether);
    if constexpr (GRAD) {
      if (p.splits > 1) recurrence_grad_kernel<DTYPE, NW, true><<<grid, NW * 64, 0, s>>>(p);
      recurrence_grad_kernel<DTYPE, NW, false><<<grid, NW * 64, 0, s>>>(p);
    } else {
      if (p.splits > 1) recurrence_kernel<DTYPE, NW, true><<<grid, NW * 64, 0, s>>>(p);
      recurrence_kernel<DTYPE, NW, false><<<grid, NW * 64, 0, s>>>(p);
    }
  }
}
void launch_step(RecurrenceParams p, int dtype, int64_t seqs, hipStream_t s) {
  const int64_t pieces = (p.D + 7) / 8, most = (1ll << 31) / pieces, step = most < 1 ? 1 : most;
  for (p.seq0 = 0; p.seq0 < seqs; p.seq0 += step) {
    p.seqs = (unsigned)(seqs - p.seq0 < step ? seqs - p.seq0 : step);
    const unsigned grid = (unsigned)((p.seqs * pieces + 255) / 256);
    if (dtype == LSAM_DTYPE_BF16) recurrence_step_kernel<LSAM_DTYPE_BF16><<<grid, 256, 0, s>>>(p);
    else recurrence_step_kernel<LSAM_DTYPE_FP32><<<grid, 256, 0, s>>>(p);
  }
}
template <bool GRAD>
void launch_any(const RecurrenceParams& p, const lsam_recurrence_desc* d, int waves, hipStream_t s) {
  if (d->dtype == LSAM_DTYPE_BF16) {
    if (waves == 1) launch<LSAM_DTYPE_BF16, 1, GRAD>(p, d->seqs, s); else launch<LSAM_DTYPE_BF16, kWaves, GRAD>(p, d->seqs, s);
  } else {
    if (waves == 1) launch<LSAM_DTYPE_FP32, 1, GRAD>(p, d->seqs, s); else launch<LSAM_DTYPE_FP32, kWaves, GRAD>(p, d->seqs, s);
  }
}

RecurrenceParams params(const lsam_recurrence_desc* d, const Plan& c, const int64_t* offsets, void* workspace) {
  RecurrenceParams p{};
  p.offsets = d->packed ? offsets : nullptr;
  p.rows = d->rows; p.D = d->dim;
  p.tiles_of_each = c.tiles_of_each;
  p.splits = c.splits; p.slabs = c.slabs; p.run_tiles = c.run_tiles;
  p.runs = static_cast<float*>(workspace);
  return p;
}

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" size_t lsam_recurrence_workspace_bytes(const lsam_recurrence_desc* d) {
  if (check(d, "recurrence") != LSAM_OK) return 0;
  const Plan c = plan(d);
  return c.splits > 1 ? (size_t)d->seqs * c.splits * 2 * (size_t)d->dim * 4 : 0;
}

extern "C" int64_t lsam_recurrence_states(const lsam_recurrence_desc* d) {
  const int rc = check(d, "recurrence");
  return rc != LSAM_OK ? rc : plan(d).states;
}

extern "C" int lsam_recurrence(const lsam_recurrence_desc* d, const int64_t* offsets, const void* f, const void* x, const float* h0,
                               void* h, float* last, float* states, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d, "recurrence");
  if (rc != LSAM_OK) return rc;
  if (d->seqs == 0) return LSAM_OK;
  if (d->packed && !offsets) return refuse(LSAM_EINVAL, "recurrence: packed sequences need offsets");
  const Plan c = plan(d);
  const int64_t state = d->seqs * d->dim * 4;
  const Arg args[] = {arg(d, "f", f, d->f, false), arg(d, "x", x, d->x, false),
                      arg(d, "h", h, d->h, true), {"h0", h0, h0 ? state : 0, 4, false},
                      {"last", last, last ? state : 0, 4, true}, {"states", states, states ? c.states * d->dim * 4 : 0, 4, true},
                      {"offsets", d->packed ? offsets : nullptr, d->packed ? (d->seqs + 1) * 8 : 0, 8, false}};
  constexpr int n = sizeof args / sizeof args[0];
  rc = check_values(args, n, "recurrence");
  if (rc == LSAM_OK) rc = check_apart(args, n, "recurrence");
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, lsam_recurrence_workspace_bytes(d), 16, "recurrence");
  if (rc != LSAM_OK) return rc;
  RecurrenceParams p = params(d, c, offsets, workspace);
  p.f = tensor(f, d->f, d->packed); p.x = tensor(x, d->x, d->packed); p.h = tensor(h, d->h, d->packed);
  p.h0 = h0; p.last = last; p.states = states;
  if (!d->packed && d->rows == 1) launch_step(p, d->dtype, d->seqs, static_cast<hipStream_t>(stream));
  else launch_any<false>(p, d, c.waves, static_cast<hipStream_t>(stream));
  return launched();
}

extern "C" int lsam_recurrence_backward(const lsam_recurrence_desc* d, const int64_t* offsets, const void* f, const void* x,
                                        const float* h0, const float* states, const void* dh, const float* dlast, void* df,
                                        void* dx, float* dh0, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(d, "recurrence_backward");
  if (rc != LSAM_OK) return rc;
  if (d->seqs == 0) return LSAM_OK;
  if (d->packed && !offsets) return refuse(LSAM_EINVAL, "recurrence_backward: packed sequences need offsets");
  const Plan c = plan(d);
  const int64_t state = d->seqs * d->dim * 4;
  const Arg args[] = {arg(d, "f", f, d->f, false), arg(d, "x", x, d->x, false),
                      arg(d, "dh", dh, d->dh, false), arg(d, "df", df, d->df, true),
                      arg(d, "dx", dx, d->dx, true), {"h0", h0, h0 ? state : 0, 4, false},
                      {"dlast", dlast, dlast ? state : 0, 4, false}, {"dh0", dh0, dh0 ? state : 0, 4, true},
                      {"states", states, c.states * d->dim * 4, 4, false},
                      {"offsets", d->packed ? offsets : nullptr, d->packed ? (d->seqs + 1) * 8 : 0, 8, false}};
  constexpr int n = sizeof args / sizeof args[0];
  rc = check_values(args, n, "recurrence_backward");
  if (rc == LSAM_OK) rc = check_apart(args, n, "recurrence_backward");
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, lsam_recurrence_workspace_bytes(d), 16, "recurrence_backward");
  if (rc != LSAM_OK) return rc;
  RecurrenceParams p = params(d, c, offsets, workspace);
  p.f = tensor(f, d->f, d->packed); p.x = tensor(x, d->x, d->packed); p.dh = tensor(dh, d->dh, d->packed);
  p.df = tensor(df, d->df, d->packed); p.dx = tensor(dx, d->dx, d->packed);
  p.h0 = h0; p.states = const_cast<float*>(states); p.dlast = dlast; p.dh0 = dh0;
  launch_any<true>(p, d, c.waves, static_cast<hipStream_t>(stream));
  return launched();
}
