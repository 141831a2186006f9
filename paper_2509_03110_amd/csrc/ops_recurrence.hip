// lsam_recurrence, lsam_recurrence_backward: h_t = a_t h_{t-1} + (1 - a_t) x_t, a_t = sigmoid(f_t), for every channel of
// every sequence, and its gradient.
//
// A run of steps maps the state that enters it to A h + H, A the product of its a_t and H what it makes of 0; runs
// are joined by (A, H) then (A', H') = (A A', A' H + H').  A workgroup owns 128 neighbouring channels of a sequence and
// goes along time in tiles: each wavefront takes a few rows of the tile into registers (two channels a lane), finds
// its own (A, H), and from those of the wavefronts before it, exchanged through LDS, the state that enters its rows.
// So every value is read once and written once.  Where sequences and channels are too few to fill the chip, the
// tiles of a sequence are cut into runs for several workgroups: a first launch leaves (A, H) of every run.
//
// Backward: with e_t = a_t (dh_t + e_{t+1}) -- what step t hands to the one before it, the same kind of recurrence from
// the other end -- d_t = dh_t + e_{t+1},  dx_t = (1 - a_t) d_t,  df_t = a_t (1 - a_t) d_t (h_{t-1} - x_t).
// The h_{t-1} are formed again, in fp32, from the state that the forward pass saved at the head of each tile.
#include "ops.h"

namespace lsam {
namespace {

constexpr int kRows = 8;             // rows of a tile that one wavefront takes
constexpr int kChannels = 128;       // of a workgroup: two for each lane
constexpr int kWaves = 8;            // of a workgroup; one where sequences are no longer than its rows
constexpr int kMaxSplits = 64;

struct Tensor { const void* p; int64_t stride, seq; };

struct RecurrenceParams {
  Tensor f, x, h, dh, df, dx;
  const int64_t* offsets;            // packed sequences: seqs + 1 row numbers, else null
  int64_t seq0, rows, D;             // rows of each sequence, or of all
  int64_t tiles_of_each;             // saved states of a sequence (not packed)
  int splits, slabs;
  const float* h0; float* last; float* states;
  const float* dlast; float* dh0;
  float* runs;                       // [seqs][splits][2][D]: A and H (or E) of every run
};

template <int DTYPE> struct Pair;
template <> struct Pair<LSAM_DTYPE_FP32> {
  typedef f32x2 raw;
  static __device__ __forceinline__ raw load(const float* p, int n) {
    if (n == 2) return *reinterpret_cast<const f32x2_any*>(p);
    return raw{n == 1 ? *p : 0.f, 0.f};
  }
  static __device__ __forceinline__ f32x2 wide(raw v) { return v; }
  static __device__ __forceinline__ void store(float* p, int n, f32x2 v) {
    if (n == 2) *reinterpret_cast<f32x2_any*>(p) = v;
    else if (n == 1) *p = v[0];
  }
};
template <> struct Pair<LSAM_DTYPE_BF16> {
  typedef u16x2 raw;
  static __device__ __forceinline__ raw load(const unsigned short* p, int n) {
    if (n == 2) return *reinterpret_cast<const u16x2_any*>(p);
    return raw{n == 1 ? *p : (unsigned short)0, 0};
  }
  static __device__ __forceinline__ f32x2 wide(raw v) { return f32x2{widen(v[0]), widen(v[1])}; }
  static __device__ __forceinline__ void store(unsigned short* p, int n, f32x2 v) {
    if (n == 2) *reinterpret_cast<u16x2_any*>(p) = u16x2{narrow(v[0]), narrow(v[1])};
    else if (n == 1) *p = narrow(v[0]);
  }
};

// a = sigmoid(f) and 1 - a, neither from the other: both keep their digits where they are small.
__device__ __forceinline__ void gates(float f, float& a, float& b) {
  const float e = __expf(-__builtin_fabsf(f)), r = __builtin_amdgcn_rcpf(1.f + e), small = e * r;
  a = f >= 0.f ? r : small;
  b = f >= 0.f ? small : r;
  if (f != f) a = b = f;
}

// Where a workgroup's sequence lies and which of its tiles are the workgroup's.
struct Place {
  int64_t seq, begin, len;      // begin: row number in packed tensors
  int64_t phase, state0;        // tile j: rows j R - phase ..; its saved state: states[state0 + j], j > 0
  int64_t tiles, first, end;
  int split;
  int64_t ch; int n;            // this lane's channels
  template <typename T>
  __device__ __forceinline__ T* at(const Tensor& t) const {
    return static_cast<T*>(const_cast<void*>(t.p)) + seq * t.seq + begin * t.stride + ch;
  }
};

template <int R>
__device__ __forceinline__ Place place(const RecurrenceParams& p) {
  Place w;
  const unsigned slab = blockIdx.x % (unsigned)p.slabs, rest = blockIdx.x / (unsigned)p.slabs;
  w.split = (int)(rest % (unsigned)p.splits);
  w.seq = p.seq0 + rest / (unsigned)p.splits;
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
  w.tiles = w.len > 0 ? (w.phase + w.len + R - 1) / R : 0;
  w.first = w.tiles * w.split / p.splits;
  w.end = w.tiles * (w.split + 1) / p.splits;
  const int64_t ch = (int64_t)slab * kChannels + (threadIdx.x & 63) * 2;
  w.n = p.D - ch >= 2 ? 2 : p.D - ch == 1 ? 1 : 0;
  w.ch = w.n ? ch : 0;
  return w;
}

typedef Pair<LSAM_DTYPE_FP32> State;

// RUNS: only (A, H) of the workgroup's run, for a launch that follows.
template <int DTYPE, int NW, bool RUNS>
__global__ __launch_bounds__(NW * 64) void recurrence_kernel(RecurrenceParams p) {
  typedef Pair<DTYPE> V;
  typedef typename Value<DTYPE>::T T;
  constexpr int R = NW * kRows;
  __shared__ f32x2 shA[2][NW][64], shH[2][NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place w = place<R>(p);
  const T* f = w.at<const T>(p.f);
  const T* x = w.at<const T>(p.x);
  T* h = RUNS ? nullptr : w.at<T>(p.h);
  f32x2 carry{0.f, 0.f}, whole{1.f, 1.f};
  if constexpr (!RUNS) {
    if (p.h0) carry = State::load(p.h0 + w.seq * p.D + w.ch, w.n);
    for (int q = 0; q < w.split; ++q) {
      const float* run = p.runs + (w.seq * p.splits + q) * 2 * p.D + w.ch;
      carry = State::load(run, w.n) * carry + State::load(run + p.D, w.n);
    }
  }
  typename V::raw rf[kRows], rx[kRows];
  auto fetch = [&](int64_t j) {
    const int64_t t0 = j * R - w.phase + wave * kRows;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int64_t t = t0 + i;
      const int n = j < w.end && t >= 0 && t < w.len ? w.n : 0;
      rf[i] = V::load(f + (n ? t * p.f.stride : 0), n);
      rx[i] = V::load(x + (n ? t * p.x.stride : 0), n);
    }
  };
  fetch(w.first);
  int b = 0;
  for (int64_t j = w.first; j < w.end; ++j) {
    const int64_t t0 = j * R - w.phase + wave * kRows;
    f32x2 a[kRows], v[kRows], A{1.f, 1.f}, H{0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const bool in = t0 + i >= 0 && t0 + i < w.len;
      const f32x2 wf = V::wide(rf[i]), wx = V::wide(rx[i]);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float g, k;
        gates(wf[c], g, k);
        a[i][c] = in ? g : 1.f;               // rows outside the sequence leave the state as it is
        v[i][c] = in ? k * wx[c] : 0.f;
      }
    }
    fetch(j + 1);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      A *= a[i];
      H = a[i] * H + v[i];
    }
    if constexpr (!RUNS)
      if (wave == 0 && p.states && j > 0) State::store(p.states + (w.state0 + j) * p.D + w.ch, w.n, carry);
    f32x2 s = carry;
    if constexpr (NW > 1) {
      shA[b][wave][lane] = A;
      shH[b][wave][lane] = H;
      __syncthreads();
#pragma unroll
      for (int q = 0; q < NW; ++q) {
        const f32x2 qa = shA[b][q][lane], qh = shH[b][q][lane];
        if (q == wave) s = carry;
        carry = qa * carry + qh;
        if constexpr (RUNS) whole *= qa;
      }
      b ^= 1;
    } else {
      carry = A * carry + H;
      if constexpr (RUNS) whole *= A;
    }
    if constexpr (!RUNS) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        s = a[i] * s + v[i];
        const int64_t t = t0 + i;
        if (t >= 0 && t < w.len) V::store(h + t * p.h.stride, w.n, s);
      }
    }
  }
  if (wave != 0) return;
  if constexpr (RUNS) {
    float* run = p.runs + (w.seq * p.splits + w.split) * 2 * p.D + w.ch;
    State::store(run, w.n, whole);
    State::store(run + p.D, w.n, carry);
  } else if (w.split == p.splits - 1 && p.last) {
    State::store(p.last + w.seq * p.D + w.ch, w.n, carry);
  }
}

// RUNS: only (A, E) of the workgroup's run.
template <int DTYPE, int NW, bool RUNS>
__global__ __launch_bounds__(NW * 64) void recurrence_grad_kernel(RecurrenceParams p) {
  typedef Pair<DTYPE> V;
  typedef typename Value<DTYPE>::T T;
  constexpr int R = NW * kRows;
  __shared__ f32x2 shA[2][NW][64], shE[2][NW][64], shH[2][NW][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place w = place<R>(p);
  const T* f = w.at<const T>(p.f);
  const T* x = RUNS ? nullptr : w.at<const T>(p.x);
  const T* dh = w.at<const T>(p.dh);
  T* df = RUNS ? nullptr : w.at<T>(p.df);
  T* dx = RUNS ? nullptr : w.at<T>(p.dx);
  f32x2 carry{0.f, 0.f}, whole{1.f, 1.f};
  if constexpr (!RUNS) {
    if (p.dlast) carry = State::load(p.dlast + w.seq * p.D + w.ch, w.n);
    for (int q = p.splits - 1; q > w.split; --q) {
      const float* run = p.runs + (w.seq * p.splits + q) * 2 * p.D + w.ch;
      carry = State::load(run, w.n) * carry + State::load(run + p.D, w.n);
    }
  }
  typename V::raw rf[kRows], rx[kRows], rd[kRows];
  f32x2 entry{0.f, 0.f};
  auto fetch = [&](int64_t j) {
    const int64_t t0 = j * R - w.phase + wave * kRows;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int64_t t = t0 + i;
      const int n = j >= w.first && t >= 0 && t < w.len ? w.n : 0;
      rf[i] = V::load(f + (n ? t * p.f.stride : 0), n);
      if constexpr (!RUNS) rx[i] = V::load(x + (n ? t * p.x.stride : 0), n);
      rd[i] = V::load(dh + (n ? t * p.dh.stride : 0), n);
    }
    if constexpr (!RUNS) {
      entry = f32x2{0.f, 0.f};
      if (j > 0) entry = State::load(p.states + (w.state0 + j) * p.D + w.ch, j >= w.first ? w.n : 0);
      else if (j == 0 && p.h0) entry = State::load(p.h0 + w.seq * p.D + w.ch, w.first == 0 ? w.n : 0);
    }
  };
  if (w.end > w.first) fetch(w.end - 1);
  int b = 0;
  for (int64_t j = w.end - 1; j >= w.first; --j) {
    const int64_t t0 = j * R - w.phase + wave * kRows;
    f32x2 a[kRows], k[kRows], xv[kRows], d[kRows], A{1.f, 1.f}, E{0.f, 0.f}, H{0.f, 0.f}, s = entry;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const bool in = t0 + i >= 0 && t0 + i < w.len;
      const f32x2 wf = V::wide(rf[i]);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float g, m;
        gates(wf[c], g, m);
        a[i][c] = in ? g : 1.f;
        k[i][c] = in ? m : 0.f;
      }
      if constexpr (!RUNS) xv[i] = V::wide(rx[i]);
      d[i] = V::wide(rd[i]);
    }
    fetch(j - 1);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      A *= a[i];
      if constexpr (!RUNS) H = a[i] * H + k[i] * xv[i];
    }
#pragma unroll
    for (int i = kRows - 1; i >= 0; --i) E = a[i] * (d[i] + E);
    f32x2 e = carry;
    if constexpr (NW > 1) {
      shA[b][wave][lane] = A;
      shE[b][wave][lane] = E;
      if constexpr (!RUNS) shH[b][wave][lane] = H;
      __syncthreads();
#pragma unroll
      for (int q = NW - 1; q >= 0; --q) {
        const f32x2 qa = shA[b][q][lane];
        if (q == wave) e = carry;
        carry = qa * carry + shE[b][q][lane];
        if constexpr (RUNS) whole *= qa;
      }
      if constexpr (!RUNS) {
#pragma unroll
        for (int q = 0; q < NW - 1; ++q)
          if (q < wave) s = shA[b][q][lane] * s + shH[b][q][lane];
      }
      b ^= 1;
    } else {
      carry = A * carry + E;
      if constexpr (RUNS) whole *= A;
    }
    if constexpr (!RUNS) {
      f32x2 before[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        before[i] = s;
        s = a[i] * s + k[i] * xv[i];
      }
#pragma unroll
      for (int i = kRows - 1; i >= 0; --i) {
        const f32x2 t_d = d[i] + e, kd = k[i] * t_d;
        const int64_t t = t0 + i;
        if (t >= 0 && t < w.len) {
          V::store(dx + t * p.dx.stride, w.n, kd);
          V::store(df + t * p.df.stride, w.n, a[i] * kd * (before[i] - xv[i]));
        }
        e = a[i] * t_d;
      }
    }
  }
  if (wave != 0) return;
  if constexpr (RUNS) {
    float* run = p.runs + (w.seq * p.splits + w.split) * 2 * p.D + w.ch;
    State::store(run, w.n, whole);
    State::store(run + p.D, w.n, carry);
  } else if (w.split == 0 && p.dh0) {
    State::store(p.dh0 + w.seq * p.D + w.ch, w.n, carry);
  }
}

// How a call is cut.  One wavefront where sequences are no longer than its rows (a step of generation).
struct Plan { int waves, splits, slabs; int64_t tiles_of_each, states; };
Plan plan(const lsam_recurrence_desc* d) {
  Plan c;
  const int64_t mean = d->packed ? (d->seqs ? (d->rows + d->seqs - 1) / d->seqs : 0) : d->rows;
  c.waves = mean <= kRows ? 1 : kWaves;
  const int64_t R = (int64_t)c.waves * kRows;
  c.slabs = (int)((d->dim + kChannels - 1) / kChannels);
  c.tiles_of_each = d->packed ? 0 : (d->rows + R - 1) / R;
  c.states = d->packed ? d->rows / R + 1 : d->seqs * c.tiles_of_each;
  // Runs: as many as give every unit two workgroups, of at least four tiles each.
  const int64_t groups = d->seqs * c.slabs, tiles = (d->rows + R - 1) / R;
  int64_t splits = groups > 0 && groups < 128 ? 512 / groups : 1;
  if (splits > tiles / 4) splits = tiles / 4;
  if (splits > kMaxSplits) splits = kMaxSplits;
  c.splits = splits < 1 ? 1 : (int)splits;
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

// The bytes that a tensor spans (-1: refused), sequences of an output apart from each other.
int64_t spans(const lsam_recurrence_desc* d, const lsam_rows& t, bool output) {
  const int64_t mats = d->packed ? 1 : d->seqs;
  if (output && !apart(mats, t.seq, d->rows, t.stride, d->dim)) return -1;
  return extent(mats, t.seq, d->rows, t.stride, d->dim, dtype_bytes(d->dtype));
}

struct Arg { const char* name; const void* p; int64_t bytes; int align; bool output; };
int check_args(const Arg* args, int n, const char* who) {
  for (int i = 0; i < n; ++i) {
    if (args[i].bytes < 0) return refuse(LSAM_EINVAL, "%s: a stride of %s is too small, or the array is too large", who, args[i].name);
    if (args[i].bytes && !args[i].p) return refuse(LSAM_EINVAL, "%s: %s is NULL", who, args[i].name);
    if (misaligned(args[i].p, args[i].align)) return refuse(LSAM_EINVAL, "%s: %s is not aligned to its values", who, args[i].name);
  }
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j)
      if (i != j && args[i].output && args[i].p && args[j].p && overlap(args[i].p, args[i].bytes, args[j].p, args[j].bytes))
        return refuse(LSAM_EINVAL, "%s: %s lies over %s", who, args[i].name, args[j].name);
  return LSAM_OK;
}

Tensor tensor(const void* p, const lsam_rows& r, bool packed) { return Tensor{p, r.stride, packed ? 0 : r.seq}; }

template <int DTYPE, int NW, bool GRAD>
void launch(RecurrenceParams p, int64_t seqs, hipStream_t s) {
  // a launch has less than 2^32 lanes: more sequences take further launches
  const int64_t most = ((1ll << 31) / (NW * 64)) / ((int64_t)p.splits * p.slabs);
  const int64_t step = most < 1 ? 1 : most;
  for (int64_t s0 = 0; s0 < seqs; s0 += step) {
    p.seq0 = s0;
    const unsigned grid = (unsigned)((seqs - s0 < step ? seqs - s0 : step) * p.splits * p.slabs);
    if constexpr (GRAD) {
      if (p.splits > 1) recurrence_grad_kernel<DTYPE, NW, true><<<grid, NW * 64, 0, s>>>(p);
      recurrence_grad_kernel<DTYPE, NW, false><<<grid, NW * 64, 0, s>>>(p);
    } else {
      if (p.splits > 1) recurrence_kernel<DTYPE, NW, true><<<grid, NW * 64, 0, s>>>(p);
      recurrence_kernel<DTYPE, NW, false><<<grid, NW * 64, 0, s>>>(p);
    }
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

int check_workspace(const lsam_recurrence_desc* d, const void* workspace, size_t bytes, const char* who) {
  const size_t need = lsam_recurrence_workspace_bytes(d);
  if (need && (!workspace || bytes < need))
    return refuse(LSAM_ENOMEM, "%s: the workspace has %zu bytes, %zu are needed", who, workspace ? bytes : 0, need);
  if (need && misaligned(workspace, 16)) return refuse(LSAM_EINVAL, "%s: the workspace must be 16-byte aligned", who);
  return LSAM_OK;
}

RecurrenceParams params(const lsam_recurrence_desc* d, const Plan& c, const int64_t* offsets, void* workspace) {
  RecurrenceParams p{};
  p.offsets = d->packed ? offsets : nullptr;
  p.rows = d->rows; p.D = d->dim;
  p.tiles_of_each = c.tiles_of_each;
  p.splits = c.splits; p.slabs = c.slabs;
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
  const int b = dtype_bytes(d->dtype);
  const int64_t state = d->seqs * d->dim * 4;
  const Arg args[] = {{"f", f, spans(d, d->f, false), b, false}, {"x", x, spans(d, d->x, false), b, false},
                      {"h", h, spans(d, d->h, true), b, true}, {"h0", h0, h0 ? state : 0, 4, false},
                      {"last", last, last ? state : 0, 4, true}, {"states", states, states ? c.states * d->dim * 4 : 0, 4, true},
                      {"offsets", d->packed ? offsets : nullptr, d->packed ? (d->seqs + 1) * 8 : 0, 8, false}};
  rc = check_args(args, sizeof args / sizeof args[0], "recurrence");
  if (rc != LSAM_OK) return rc;
  rc = check_workspace(d, workspace, workspace_bytes, "recurrence");
  if (rc != LSAM_OK) return rc;
  RecurrenceParams p = params(d, c, offsets, workspace);
  p.f = tensor(f, d->f, d->packed); p.x = tensor(x, d->x, d->packed); p.h = tensor(h, d->h, d->packed);
  p.h0 = h0; p.last = last; p.states = states;
  launch_any<false>(p, d, c.waves, static_cast<hipStream_t>(stream));
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
  const int b = dtype_bytes(d->dtype);
  const int64_t state = d->seqs * d->dim * 4;
  const Arg args[] = {{"f", f, spans(d, d->f, false), b, false}, {"x", x, spans(d, d->x, false), b, false},
                      {"dh", dh, spans(d, d->dh, false), b, false}, {"df", df, spans(d, d->df, true), b, true},
                      {"dx", dx, spans(d, d->dx, true), b, true}, {"h0", h0, h0 ? state : 0, 4, false},
                      {"dlast", dlast, dlast ? state : 0, 4, false}, {"dh0", dh0, dh0 ? state : 0, 4, true},
                      {"states", states, c.states * d->dim * 4, 4, false},
                      {"offsets", d->packed ? offsets : nullptr, d->packed ? (d->seqs + 1) * 8 : 0, 8, false}};
  rc = check_args(args, sizeof args / sizeof args[0], "recurrence_backward");
  if (rc != LSAM_OK) return rc;
  rc = check_workspace(d, workspace, workspace_bytes, "recurrence_backward");
  if (rc != LSAM_OK) return rc;
  RecurrenceParams p = params(d, c, offsets, workspace);
  p.f = tensor(f, d->f, d->packed); p.x = tensor(x, d->x, d->packed); p.dh = tensor(dh, d->dh, d->packed);
  p.df = tensor(df, d->df, d->packed); p.dx = tensor(dx, d->dx, d->packed);
  p.h0 = h0; p.states = const_cast<float*>(states); p.dlast = dlast; p.dh0 = dh0;
  launch_any<true>(p, d, c.waves, static_cast<hipStream_t>(stream));
  return launched();
}
