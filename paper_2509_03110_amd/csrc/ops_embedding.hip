// lsam_embedding, lsam_embedding_backward: rows of a table for tokens, and the sum of each token's rows of a gradient.
//
//   lookup_kernel   y = scale E[token]: sixteen bytes of y a lane
//   order_kernel    the places of a replica's tokens, sorted by token and within a token by place, with no atomics: a workgroup owns
//                   a range of tokens, walks over the places and keeps what is in its range.  Where places are many they are cut
//                   into parts for several workgroups, and
//   count_kernel    says before how often each token occurs in each part
//   sums_kernel     a wavefront takes 64 sorted places and 256 columns; a token whose places all lie there is finished, of
//                   others it leaves partial sums; further wavefronts write the zeros of tokens that do not occur
//   join_kernel     partial sums of tokens that go on past an edge of 64 places
#include "ops.h"

namespace lsam {
namespace {

constexpr int kOrderWaves = 16;
constexpr int kMaxRange = 512;         // tokens of a workgroup of order_kernel: [range][wavefronts] counters in LDS, 32 KiB
constexpr int kAhead = 8;              // loads of 64 tokens on their way
constexpr int kPlaces = 64;            // sorted places of a wavefront of sums_kernel, one for each lane
constexpr int kSlab = 256;             // columns of a wavefront, four a lane
constexpr int kZeroRows = 16;          // rows of the table that a wavefront looks at for tokens that do not occur
constexpr int kJoinWaves = 8;

struct EmbeddingParams {
  const int32_t* tokens; const void* table; void* y;
  const void* dy; float* dtable;
  int64_t rows, vocab, dim, token_replica;
  int64_t table_stride, table_replica, y_stride, y_replica, dy_stride, dy_replica, dtable_stride, dtable_replica;
  float scale;
  int32_t replica0;                    // first replica of this launch
  int64_t row0, chunk0;                // first row of the launch (lookup; zeros of sums_kernel), first chunk (sums, join)
  unsigned units, zeros;               // lanes with work (lookup); wavefronts that sum, or join, and that write zeros
  unsigned pieces;                     // of a lane's columns in a row (lookup), of kSlab (sums, join)
  int64_t chunks;                      // of kPlaces places
  unsigned range, ranges, parts;       // order_kernel: tokens of a workgroup, workgroups for all tokens, parts of the places
  int64_t part;                        // places of a part
  uint32_t* count; uint32_t* total;    // [replicas][vocab][parts], [replicas][ranges][parts]
  int32_t* order; int32_t* start;      // [replicas][rows], [replicas][vocab + 1]
  float* partial;                      // [replicas][chunks][2][dim]: of the token that comes from the chunk before, that goes on into the next
};

// Numbers of y that a lane writes.
template <int DTYPE> constexpr int kLookup = DTYPE == LSAM_DTYPE_BF16 ? 8 : 4;

// Four columns of a row from `col` on, zeros behind the row's end.
template <int DTYPE>
__device__ __forceinline__ f32x4 load4(const typename Value<DTYPE>::T* p, int n) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (n == 4) {
    if constexpr (DTYPE == LSAM_DTYPE_FP32) {
      v = *reinterpret_cast<const f32x4_any*>(p);
    } else {
      const u16x4 w = *reinterpret_cast<const u16x4_any*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = widen(w[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) v[e] = Value<DTYPE>::get(p + e);
  }
  return v;
}
__device__ __forceinline__ void store4(float* p, f32x4 v, int n) {
  if (n == 4) {
    *reinterpret_cast<f32x4_any*>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = v[e];
  }
}

// One load of a token before the row's address is known, so bound by latency where rows are few.  Where there are many a lane has UNITS units, the
// workgroup's threads apart, whose loads do not wait for each other.
template <int TABLE, int DTYPE, int UNITS>
__global__ __launch_bounds__(256) void lookup_kernel(EmbeddingParams p) {
  typedef typename Value<TABLE>::T T;
  typedef typename Value<DTYPE>::T Y;
  constexpr int N = kLookup<DTYPE>;
  const int64_t replica = p.replica0 + blockIdx.y;
  const unsigned first = blockIdx.x * (256 * UNITS) + threadIdx.x;
  int64_t row[UNITS];
  int col[UNITS];
  int32_t token[UNITS];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const unsigned unit = first + i * 256 < p.units ? first + i * 256 : p.units - 1, local = unit / p.pieces;
    col[i] = (int)(unit - local * p.pieces) * N;
    row[i] = p.row0 + local;
    token[i] = p.tokens[replica * p.token_replica + row[i]];
  }
  float v[UNITS][N];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const bool there = token[i] >= 0 && token[i] < p.vocab;
    const T* src = static_cast<const T*>(p.table) + replica * p.table_replica + (there ? token[i] : 0) * p.table_stride + col[i];
    if (col[i] + N <= p.dim) {
      if constexpr (N == 8) {
        Value<TABLE>::load8(src, v[i]);
      } else {
        const f32x4 w = load4<TABLE>(src, 4);
#pragma unroll
        for (int e = 0; e < N; ++e) v[i][e] = w[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[i][e] = col[i] + e < p.dim ? Value<TABLE>::get(src + e) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) v[i][e] = there ? v[i][e] * p.scale : 0.f;
  }
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    if (first + i * 256 >= p.units) return;
    Y* dst = static_cast<Y*>(p.y) + replica * p.y_replica + row[i] * p.y_stride + col[i];
    if (col[i] + N <= p.dim) {
      if constexpr (N == 8) Value<DTYPE>::store8(dst, v[i]);
      else *reinterpret_cast<f32x4_any*>(dst) = f32x4{v[i][0], v[i][1], v[i][2], v[i][3]};
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (col[i] + e < p.dim) Value<DTYPE>::put(dst + e, v[i][e]);
    }
  }
}

// Calls f(token, lanes that hold it) for every token of the range that the wavefront holds.
template <typename F>
__device__ __forceinline__ void each_token(int32_t token, bool mine, F f) {
  unsigned long long left = __ballot(mine);
  while (left) {
    const int32_t t = __builtin_amdgcn_readlane(token, __builtin_ctzll(left));
    const unsigned long long same = __ballot(mine && token == t);
    f(t, same);
    left &= ~same;
  }
}

// A wavefront's run of the places of a workgroup's part: f(tokens, first place of them), 64 tokens in the lanes, kAhead times at once.
template <typename F>
__device__ __forceinline__ void each_run(const EmbeddingParams& p, const int32_t* tokens, int part, int wave, F f) {
  const int lane = threadIdx.x & 63;
  const int64_t begin = part * p.part, end = begin + p.part < p.rows ? begin + p.part : p.rows;
  const int64_t steps = (end - begin + 63) / 64, each = (steps + kOrderWaves - 1) / kOrderWaves;
  const int64_t first = begin + wave * each * 64, last = first + each * 64 < end ? first + each * 64 : end;
  for (int64_t at = first; at < last; at += 64 * kAhead) {
    int32_t t[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t row = at + i * 64 + lane;
      t[i] = row < last ? tokens[row] : -1;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (at + i * 64 < last) f(t[i], at + i * 64);
  }
}
// A range of tokens, and the counters [range][wavefronts] of a workgroup's part, one column for each wavefront; all its lanes update one alike.
struct Range { int32_t lo, hi; };
__device__ __forceinline__ Range range_of(const EmbeddingParams& p) {
  const int32_t lo = (int32_t)(blockIdx.x * p.range);
  return Range{lo, (int32_t)(lo + p.range < p.vocab ? lo + p.range : p.vocab)};
}
__device__ __forceinline__ uint32_t count_tokens(const EmbeddingParams& p, const int32_t* tokens, const Range& r, int part, int wave, uint32_t* counts) {
  for (int i = threadIdx.x; i < (r.hi - r.lo) * kOrderWaves; i += kOrderWaves * 64) counts[i] = 0;
  __syncthreads();
  uint32_t fewer = 0;                                      // tokens of lower ranges
  each_run(p, tokens, part, wave, [&](int32_t t, int64_t) {
    fewer += (uint32_t)__popcll(__ballot(t >= 0 && t < r.lo));
    each_token(t, t >= r.lo && t < r.hi, [&](int32_t token, unsigned long long same) { counts[(token - r.lo) * kOrderWaves + wave] += (uint32_t)__popcll(same); });
  });
  __syncthreads();
  return fewer;
}
__device__ __forceinline__ uint32_t of_token(const uint32_t* counts, int token) {
  uint32_t n = 0;
#pragma unroll
  for (int w = 0; w < kOrderWaves; ++w) n += counts[token * kOrderWaves + w];
  return n;
}
// Sum over the workgroup's threads before this one, and of all.
__device__ __forceinline__ uint32_t before_thread(uint32_t mine, uint32_t& all) {
  __shared__ uint32_t sums[kOrderWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t before = mine;                                  // with those of lower lanes
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t other = __shfl_up(before, d);
    if (lane >= d) before += other;
  }
  if (lane == 63) sums[wave] = before;
  __syncthreads();
  before -= mine;
  all = 0;
  for (int w = 0; w < kOrderWaves; ++w) {
    if (w < wave) before += sums[w];
    all += sums[w];
  }
  __syncthreads();
  return before;
}

__global__ __launch_bounds__(kOrderWaves * 64) void count_kernel(EmbeddingParams p) {
  __shared__ uint32_t counts[kMaxRange * kOrderWaves];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = blockIdx.y;
  const int64_t replica = p.replica0 + blockIdx.z;
  const Range r = range_of(p);
  count_tokens(p, p.tokens + replica * p.token_replica, r, part, wave, counts);
  const uint32_t n = tid < r.hi - r.lo ? of_token(counts, tid) : 0;
  if (tid < r.hi - r.lo) p.count[(replica * p.vocab + r.lo + tid) * p.parts + part] = n;
  uint32_t all;
  before_thread(n, all);
  if (tid == 0) p.total[(replica * p.ranges + blockIdx.x) * p.parts + part] = all;
}

// Each wavefront owns a run of places and a column of counters, so that places keep their order: counted first, then, from where each token's
// places of the wavefront begin, put there.  Tokens of other ranges cost a load and two comparisons.  131072 places of 1000 tokens: 64 us
// with all places for each of 250 workgroups, 18 and 8 for the counts with 16 parts of them; 4 x 4096 places of 32003 tokens 9 us, most of it latency.
__global__ __launch_bounds__(kOrderWaves * 64) void order_kernel(EmbeddingParams p) {
  __shared__ uint32_t counts[kMaxRange * kOrderWaves], below[kOrderWaves];
  static_assert(kMaxRange <= kOrderWaves * 64, "a token a thread");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), part = blockIdx.y;
  const int64_t replica = p.replica0 + blockIdx.z;
  const int32_t* tokens = p.tokens + replica * p.token_replica;
  int32_t* order = p.order + replica * p.rows;
  const Range r = range_of(p);
  uint32_t fewer = count_tokens(p, tokens, r, part, wave, counts);
  uint32_t base = 0, mine = 0, earlier = 0;                // places of lower ranges; a token's, one a thread, and those of them in earlier parts
  if (p.parts > 1) {
    uint32_t lower = 0;
    for (int64_t i = tid; i < (int64_t)blockIdx.x * p.parts; i += kOrderWaves * 64) lower += p.total[replica * p.ranges * p.parts + i];
    before_thread(lower, base);
    if (tid < r.hi - r.lo) {
      const uint32_t* of = p.count + (replica * p.vocab + r.lo + tid) * p.parts;
      for (unsigned i = 0; i < p.parts; ++i) {
        if ((int)i < part) earlier += of[i];
        mine += of[i];
      }
    }
  } else {
    if (lane == 0) below[wave] = fewer;
    __syncthreads();
    for (int w = 0; w < kOrderWaves; ++w) base += below[w];
    if (tid < r.hi - r.lo) mine = of_token(counts, tid);
  }
  uint32_t all;
  uint32_t at = base + before_thread(mine, all);
  int32_t* start = p.start + replica * (p.vocab + 1);
  if (tid < r.hi - r.lo) {
    if (part == 0) start[r.lo + tid] = (int32_t)at;
    at += earlier;
#pragma unroll
    for (int w = 0; w < kOrderWaves; ++w) {
      const uint32_t c = counts[tid * kOrderWaves + w];
      counts[tid * kOrderWaves + w] = at;
      at += c;
    }
  }
  if (part == 0 && r.hi == p.vocab && tid == 0) start[p.vocab] = (int32_t)(base + all);
  __syncthreads();
  each_run(p, tokens, part, wave, [&](int32_t t, int64_t row0) {
    each_token(t, t >= r.lo && t < r.hi, [&](int32_t token, unsigned long long same) {
      uint32_t* c = &counts[(token - r.lo) * kOrderWaves + wave];
      const uint32_t place = *c;
      if (same >> lane & 1) order[place + (uint32_t)__popcll(same & ((1ull << lane) - 1))] = (int32_t)(row0 + lane);
      *c = place + (uint32_t)__popcll(same);
    });
  });
}

// The same for what is not read again soon: it does not take the place of other lines in the caches.
__device__ __forceinline__ void store4_past(float* p, f32x4 v, int n) {
  if (n == 4) {
    __builtin_nontemporal_store(v, reinterpret_cast<f32x4_any*>(p));
  } else {
    store4(p, v, n);
  }
}

// The first p.units wavefronts of a replica sum, p.zeros more write zeros.  Bound by memory: 131072 rows of 777 numbers of fp32, read in the order of their
// tokens, take 126 us (3.3 TB/s); 4 x 4096 rows of 1024 with tables of 32003 rows, which are written whole, 105 us (5.3 TB/s).
template <int DTYPE>
__global__ __launch_bounds__(256) void sums_kernel(EmbeddingParams p) {
  typedef typename Value<DTYPE>::T T;
  const int lane = threadIdx.x & 63;
  const int64_t replica = p.replica0 + blockIdx.y;
  unsigned unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t* start = p.start + replica * (p.vocab + 1);
  float* dtable = p.dtable + replica * p.dtable_replica;
  if (unit >= p.units) {
    unit -= p.units;
    if (unit >= p.zeros) return;
    const int64_t row0 = p.row0 + (int64_t)unit * kZeroRows, at = row0 + lane;
    unsigned long long left = __ballot(lane < kZeroRows && at < p.vocab && start[at < p.vocab ? at : 0] == start[at < p.vocab ? at + 1 : 0]);
    for (; left; left &= left - 1) {
      float* row = dtable + (row0 + __builtin_ctzll(left)) * p.dtable_stride;
      for (int64_t col = lane * 4; col < p.dim; col += kSlab) store4_past(row + col, f32x4{0.f, 0.f, 0.f, 0.f}, (int)(p.dim - col < 4 ? p.dim - col : 4));
    }
    return;
  }
  const int64_t chunk = p.chunk0 + unit / p.pieces, col = (int64_t)(unit % p.pieces) * kSlab + lane * 4;
  const int64_t at = chunk * kPlaces, all = start[p.vocab];
  if (at >= all) return;
  const int n = (int)(p.dim - col < 4 ? p.dim - col : 4);                   // none of a lane behind the row's end
  const int32_t* order = p.order + replica * p.rows;
  const int32_t* tokens = p.tokens + replica * p.token_replica;
  const int places = (int)(all - at < kPlaces ? all - at : kPlaces);
  const int32_t row = order[at + (lane < places ? lane : places - 1)], token = tokens[row];
  const int32_t prev = at > 0 ? tokens[order[at - 1]] : -1, next = at + places < all ? tokens[order[at + places]] : -1;
  const int32_t left = __shfl_up(token, 1);
  const unsigned long long heads = __ballot(lane > 0 && lane < places && token != left);   // a token begins there
  const T* dy = static_cast<const T*>(p.dy) + replica * p.dy_replica + (n > 0 ? col : 0);
  float* partial = p.partial + (replica * p.chunks + chunk) * 2 * p.dim + col;
  bool open = __builtin_amdgcn_readfirstlane(token) == prev;                // the first token comes from the chunk before
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  auto leave = [&](int place, bool more) {                                  // the token that ends at `place`, or goes on
    if (n > 0) {
      if (open) store4(partial, acc, n);
      else if (more) store4(partial + p.dim, acc, n);
      else store4(dtable + __builtin_amdgcn_readlane(token, place) * p.dtable_stride + col, acc * p.scale, n);
    }
    open = false;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  for (int i0 = 0; i0 < places; i0 += 8) {
    f32x4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int place = i0 + i < places ? i0 + i : places - 1;
      v[i] = load4<DTYPE>(dy + __builtin_amdgcn_readlane(row, place) * p.dy_stride, n);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i0 + i >= places) break;
      if (heads >> (i0 + i) & 1) leave(i0 + i - 1, false);
      acc += v[i];
    }
  }
  leave(places - 1, __builtin_amdgcn_readlane(token, places - 1) == next);
}

// A wavefront for each chunk, and kSlab columns, in which a token begins that goes on into the next: it adds the token's partial sums, or, where
// they are more than kAlone, the workgroup's wavefronts add runs of them, which are added in their order.  A workgroup's units lie far apart, since
// many partial sums of a token are those of neighbours: 131072 places of 1000 tokens take 13 us, 28 with neighbours and 19 with a workgroup for each unit.
constexpr int kAlone = 8;
struct Joined { int64_t chunk, col, all; int32_t token; int n; };            // all: chunks behind this one; 0: nothing to join
__device__ __forceinline__ Joined joined(const EmbeddingParams& p, unsigned unit, int64_t replica, int lane) {
  Joined j{p.chunk0 + unit / p.pieces, (int64_t)(unit % p.pieces) * kSlab + lane * 4, 0, 0, 0};
  const int32_t* start = p.start + replica * (p.vocab + 1);
  const int64_t edge = (j.chunk + 1) * kPlaces;
  if (unit >= p.units || edge >= start[p.vocab]) return j;
  j.token = p.tokens[replica * p.token_replica + p.order[replica * p.rows + edge]];
  const int64_t begin = start[j.token], end = start[j.token + 1];
  if (begin < edge && begin >= edge - kPlaces) j.all = (end - 1) / kPlaces - j.chunk;
  j.n = (int)(p.dim - j.col < 4 ? p.dim - j.col : 4);
  return j;
}
// Partial sums of the token's chunks from + 1 .. to behind the first.
__device__ __forceinline__ f32x4 add_partial(const float* first, int64_t step, int64_t from, int64_t to, int n, f32x4 acc) {
  for (int64_t c = from; c < to; c += kAlone) {
    f32x4 v[kAlone];
#pragma unroll
    for (int i = 0; i < kAlone; ++i) v[i] = load4<LSAM_DTYPE_FP32>(first + ((c + i < to ? c + i : to - 1) + 1) * step, n);
#pragma unroll
    for (int i = 0; i < kAlone; ++i)
      if (c + i < to) acc += v[i];
  }
  return acc;
}
__global__ __launch_bounds__(kJoinWaves * 64) void join_kernel(EmbeddingParams p) {
  __shared__ f32x4 part[kJoinWaves][64];
  __shared__ bool together[kJoinWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t replica = p.replica0 + blockIdx.y, step = 2 * p.dim;
  const auto first_of = [&](const Joined& j) { return p.partial + (replica * p.chunks + j.chunk) * step + (j.n > 0 ? j.col : 0); };
  const auto store = [&](const Joined& j, f32x4 acc) { store4(p.dtable + replica * p.dtable_replica + j.token * p.dtable_stride + j.col, acc * p.scale, j.n); };
  const Joined mine = joined(p, wave * gridDim.x + blockIdx.x, replica, lane);
  if (lane == 0) together[wave] = mine.all > kAlone;
  if (mine.all > 0 && mine.all <= kAlone) {
    const float* first = first_of(mine);
    const f32x4 acc = add_partial(first, step, 0, mine.all, mine.n, load4<LSAM_DTYPE_FP32>(first + p.dim, mine.n));
    if (mine.n > 0) store(mine, acc);
  }
  __syncthreads();
  for (int u = 0; u < kJoinWaves; ++u) {
    if (!together[u]) continue;
    const Joined j = joined(p, u * gridDim.x + blockIdx.x, replica, lane);
    const int64_t each = (j.all + kJoinWaves - 1) / kJoinWaves, from = wave * each < j.all ? wave * each : j.all, to = from + each < j.all ? from + each : j.all;
    const float* first = first_of(j);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (wave == 0) acc = load4<LSAM_DTYPE_FP32>(first + p.dim, j.n);
    part[wave][lane] = add_partial(first, step, from, to, j.n, acc);
    __syncthreads();
    if (wave == 0 && j.n > 0) {
      acc = part[0][lane];
      for (int w = 1; w < kJoinWaves; ++w) acc += part[w][lane];
      store(j, acc);
    }
    __syncthreads();
  }
}

struct Plan { int ranges, parts; unsigned range; int64_t part, chunks; size_t start_at, count_at, total_at, partial_at, bytes; };
// Ranges of tokens and parts of the places: about as many workgroups as there are units, each of kPart places where the counts of all
// parts are not much to read.
constexpr int kPart = 8192;
constexpr int64_t kMaxCounts = 1 << 22;
Plan plan(const lsam_embedding_desc* d) {
  Plan c;
  const int64_t replicas = d->replicas > 0 ? d->replicas : 1;
  int64_t parts = (d->rows + kPart - 1) / kPart;
  parts = parts < kMaxCounts / d->vocab ? parts : kMaxCounts / d->vocab;
  parts = parts < 1 ? 1 : parts > 64 ? 64 : parts;
  c.part = (d->rows + parts - 1) / parts;
  c.parts = (int)(c.part > 0 ? (d->rows + c.part - 1) / c.part : 1);
  int64_t want = (256 + replicas * c.parts - 1) / (replicas * c.parts);
  const int64_t least = (d->vocab + kMaxRange - 1) / kMaxRange;
  want = want < least ? least : want > d->vocab ? d->vocab : want;
  c.range = (unsigned)((d->vocab + want - 1) / want);
  c.ranges = (int)((d->vocab + c.range - 1) / c.range);
  c.chunks = (d->rows + kPlaces - 1) / kPlaces;
  const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
  c.start_at = up((size_t)d->replicas * d->rows * 4);
  c.count_at = c.start_at + up((size_t)d->replicas * (d->vocab + 1) * 4);
  c.total_at = c.count_at + (c.parts > 1 ? up((size_t)d->replicas * d->vocab * c.parts * 4) : 0);
  c.partial_at = c.total_at + (c.parts > 1 ? up((size_t)d->replicas * c.ranges * c.parts * 4) : 0);
  c.bytes = c.partial_at + (size_t)d->replicas * c.chunks * 2 * d->dim * 4;
  return c;
}

int check(const lsam_embedding_desc* d, const char* who) {
  if (!d) return refuse(LSAM_EINVAL, "%s: the descriptor is NULL", who);
  if (!known_dtype(d->dtype) || !known_dtype(d->table_dtype)) return refuse(LSAM_EINVAL, "%s: dtype %d, %d: LSAM_DTYPE_* are wanted", who, d->dtype, d->table_dtype);
  if (d->replicas < 0 || d->replicas > 65535) return refuse(LSAM_EINVAL, "%s: replicas must be in 0..65535", who);
  if (d->rows < 0 || d->rows >= 1ll << 31) return refuse(LSAM_EINVAL, "%s: rows must be in 0..2^31-1", who);
  if (d->vocab < 1 || d->vocab > LSAM_EMBEDDING_MAX_VOCAB) return refuse(LSAM_EINVAL, "%s: vocab must be in 1..%d", who, LSAM_EMBEDDING_MAX_VOCAB);
  if (d->dim < 1 || d->dim > 1 << 24) return refuse(LSAM_EINVAL, "%s: dim must be in 1..2^24", who);
  if ((__int128)d->replicas * (d->rows > d->vocab ? d->rows : d->vocab) * d->dim >= (__int128)1 << 44)
    return refuse(LSAM_EINVAL, "%s: the arrays are too large", who);
  return LSAM_OK;
}

EmbeddingParams params(const lsam_embedding_desc* d, const int32_t* tokens) {
  EmbeddingParams p{};
  p.tokens = tokens;
  p.rows = d->rows; p.vocab = d->vocab; p.dim = d->dim; p.token_replica = d->token_replica; p.scale = d->scale;
  return p;
}

// Units of a lane where they are many: 131072 x 777 numbers of fp32 (25.6 M units) take 110 us with one, 99 with two, 85 with four and 95 with eight; 4 x 4096 x
// 1024 of bf16 (2.1 M) 12.7 with one, 13.5 with four.
constexpr int kUnits = 4;
constexpr unsigned kMany = 1 << 22;
template <int TABLE, int DTYPE>
void lookup(const EmbeddingParams& p, unsigned replicas, hipStream_t s) {
  if (p.units * (uint64_t)replicas >= kMany) lookup_kernel<TABLE, DTYPE, kUnits><<<dim3((p.units + 256 * kUnits - 1) / (256 * kUnits), replicas), 256, 0, s>>>(p);
  else lookup_kernel<TABLE, DTYPE, 1><<<dim3((p.units + 255) / 256, replicas), 256, 0, s>>>(p);
}
template <int TABLE>
void lookup(const EmbeddingParams& p, int dtype, unsigned replicas, hipStream_t s) {
  if (dtype == LSAM_DTYPE_BF16) lookup<TABLE, LSAM_DTYPE_BF16>(p, replicas, s);
  else lookup<TABLE, LSAM_DTYPE_FP32>(p, replicas, s);
}

}  // namespace
}  // namespace lsam

using namespace lsam;

extern "C" int lsam_embedding(const lsam_embedding_desc* d, const int32_t* tokens, const void* table, void* y, void* stream) {
  int rc = check(d, "embedding");
  if (rc != LSAM_OK) return rc;
  if (d->replicas == 0 || d->rows == 0) return LSAM_OK;
  Arg args[] = {matrices("tokens", tokens, 1, 0, d->replicas, d->token_replica, d->rows, 4, false),
                matrices("table", table, d->replicas, d->table_replica, d->vocab, d->table_stride, d->dim, dtype_bytes(d->table_dtype), false),
                matrices("y", y, d->replicas, d->y_replica, d->rows, d->y_stride, d->dim, dtype_bytes(d->dtype), true)};
  constexpr int n = sizeof args / sizeof args[0];
  if (d->token_replica >= 0 && d->token_replica < d->rows)    // replicas may share tokens, or read parts that overlap
    args[0] = matrices("tokens", tokens, d->replicas, d->token_replica, 1, 0, d->rows, 4, false);
  if (!apart(d->replicas, d->y_replica, d->rows, d->y_stride, d->dim)) return refuse(LSAM_EINVAL, "embedding: the replicas of y lie over each other");
  rc = check_values(args, n, "embedding");
  if (rc == LSAM_OK) rc = check_apart(args, n, "embedding");
  if (rc != LSAM_OK) return rc;
  EmbeddingParams p = params(d, tokens);
  p.table = table; p.y = y;
  p.table_stride = d->table_stride; p.table_replica = d->table_replica; p.y_stride = d->y_stride; p.y_replica = d->y_replica;
  const int each = d->dtype == LSAM_DTYPE_BF16 ? kLookup<LSAM_DTYPE_BF16> : kLookup<LSAM_DTYPE_FP32>;
  p.pieces = (unsigned)((d->dim + each - 1) / each);
  // launches of less than 2^32 lanes
  const int64_t most = (1 << 30) / p.pieces;
  const unsigned K = (unsigned)d->replicas;
  for (int64_t r0 = 0; r0 < d->rows; r0 += most) {
    p.row0 = r0;
    p.units = (unsigned)((d->rows - r0 < most ? d->rows - r0 : most) * p.pieces);
    const unsigned blocks = (p.units + 255) / 256, together = (1u << 23) / blocks < 65535 ? (1u << 23) / blocks : 65535;
    for (unsigned k = 0; k < K; k += together) {
      p.replica0 = (int32_t)k;
      const unsigned n = K - k < together ? K - k : together;
      if (d->table_dtype == LSAM_DTYPE_BF16) lookup<LSAM_DTYPE_BF16>(p, d->dtype, n, static_cast<hipStream_t>(stream));
      else lookup<LSAM_DTYPE_FP32>(p, d->dtype, n, static_cast<hipStream_t>(stream));
    }
  }
  return launched();
}

extern "C" size_t lsam_embedding_workspace_bytes(const lsam_embedding_desc* d) {
  if (check(d, "embedding") != LSAM_OK) return 0;
  return plan(d).bytes;
}

extern "C" int lsam_embedding_backward(const lsam_embedding_desc* d, const int32_t* tokens, const void* dy, float* dtable, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  const char* who = "embedding_backward";
  int rc = check(d, who);
  if (rc != LSAM_OK) return rc;
  if (d->replicas == 0) return LSAM_OK;
  const Plan c = plan(d);
  Arg args[] = {matrices("tokens", tokens, 1, 0, d->replicas, d->token_replica, d->rows, 4, false),
                matrices("dy", dy, d->replicas, d->dy_replica, d->rows, d->dy_stride, d->dim, dtype_bytes(d->dtype), false),
                matrices("dtable", dtable, d->replicas, d->dtable_replica, d->vocab, d->dtable_stride, d->dim, 4, true)};
  constexpr int n = sizeof args / sizeof args[0];
  if (d->token_replica >= 0 && d->token_replica < d->rows)
    args[0] = matrices("tokens", tokens, d->replicas, d->token_replica, 1, 0, d->rows, 4, false);
  if (!apart(d->replicas, d->dtable_replica, d->vocab, d->dtable_stride, d->dim)) return refuse(LSAM_EINVAL, "%s: the replicas of dtable lie over each other", who);
  rc = check_values(args, n, who);
  if (rc == LSAM_OK) rc = check_apart(args, n, who);
  if (rc == LSAM_OK) rc = check_workspace(args, n, workspace, workspace_bytes, c.bytes, 16, who);
  if (rc != LSAM_OK) return rc;
  EmbeddingParams p = params(d, tokens);
  p.dy = dy; p.dtable = dtable;
  p.dy_stride = d->dy_stride; p.dy_replica = d->dy_replica; p.dtable_stride = d->dtable_stride; p.dtable_replica = d->dtable_replica;
  p.order = static_cast<int32_t*>(workspace);
  p.start = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + c.start_at);
  p.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + c.partial_at);
  p.count = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + c.count_at);
  p.total = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + c.total_at);
  p.range = c.range; p.ranges = (unsigned)c.ranges; p.parts = (unsigned)c.parts; p.part = c.part;
  p.chunks = c.chunks;
  p.pieces = (unsigned)((d->dim + kSlab - 1) / kSlab);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const unsigned K = (unsigned)d->replicas;
  // launches of less than 2^32 lanes
  const int64_t fit = (1 << 21) / ((int64_t)c.ranges * c.parts);
  const unsigned apiece = (unsigned)(fit < 1 ? 1 : fit < 65535 ? fit : 65535);
  for (unsigned k = 0; k < K; k += apiece) {
    p.replica0 = (int32_t)k;
    const dim3 grid((unsigned)c.ranges, (unsigned)c.parts, K - k < apiece ? K - k : apiece);
    if (c.parts > 1) count_kernel<<<grid, kOrderWaves * 64, 0, s>>>(p);
    order_kernel<<<grid, kOrderWaves * 64, 0, s>>>(p);
  }
  // a wavefront for each chunk and piece of columns to be summed, then for each kZeroRows rows of the table
  const int64_t most = (1 << 24) / p.pieces, most_rows = (int64_t)kZeroRows << 24;
  for (int64_t c0 = 0, r0 = 0; c0 < c.chunks || r0 < d->vocab;) {
    const int64_t nc = c.chunks - c0 < most ? c.chunks - c0 : most, nr = d->vocab - r0 < most_rows ? d->vocab - r0 : most_rows;
    p.chunk0 = c0; p.row0 = r0;
    p.units = (unsigned)(nc * p.pieces); p.zeros = (unsigned)((nr + kZeroRows - 1) / kZeroRows);
    const unsigned blocks = (p.units + p.zeros + 3) / 4, together = (1u << 23) / blocks < 65535 ? (1u << 23) / blocks : 65535;
    for (unsigned k = 0; k < K; k += together) {
      p.replica0 = (int32_t)k;
      const dim3 grid(blocks, K - k < together ? K - k : together);
      if (d->dtype == LSAM_DTYPE_BF16) sums_kernel<LSAM_DTYPE_BF16><<<grid, 256, 0, s>>>(p);
      else sums_kernel<LSAM_DTYPE_FP32><<<grid, 256, 0, s>>>(p);
    }
    c0 += nc;
    r0 += nr;
  }
  const int64_t most_joined = (1 << 24) / p.pieces;
  for (int64_t c0 = 0; c0 + 1 < c.chunks; c0 += most_joined) {
    p.chunk0 = c0;
    p.units = (unsigned)((c.chunks - 1 - c0 < most_joined ? c.chunks - 1 - c0 : most_joined) * p.pieces);
    const unsigned blocks = (p.units + kJoinWaves - 1) / kJoinWaves;
    const unsigned together = (1u << 22) / blocks < 65535 ? (1u << 22) / blocks : 65535;
    for (unsigned k = 0; k < K; k += together) {
      p.replica0 = (int32_t)k;
      join_kernel<<<dim3(blocks, K - k < together ? K - k : together), kJoinWaves * 64, 0, s>>>(p);
    }
  }
  return launched();
}
