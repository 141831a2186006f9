// The search for a row's sequence in csrc/attention.h, as it stands there (sequences.inc), with a wavefront's 64 lanes as fibers on the CPU: each
// runs up to what lanes exchange, and on once all are there.  Cases come on standard input and are held to a search through all offsets.
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <sys/mman.h>
#include <ucontext.h>

#include <vector>

#define __device__
#define __forceinline__ inline
static struct { unsigned x; } threadIdx;

static const int kLanes = 64;
static const size_t kStack = 1 << 16;
static ucontext_t scheduler, fibers[kLanes];
static int64_t slots[2][kLanes];
static int turns[kLanes];
static bool done[kLanes];
static std::vector<char> stacks(kLanes * kStack);

// Every lane's value; all of them are there on return.
static const int64_t* exchange(int64_t value) {
  const unsigned lane = threadIdx.x;
  const int side = turns[lane]++ & 1;
  slots[side][lane] = value;
  swapcontext(&fibers[lane], &scheduler);
  return slots[side];
}
static unsigned long long __ballot(bool v) {
  const int64_t* all = exchange(v);
  unsigned long long m = 0;
  for (int i = 0; i < kLanes; ++i) m |= (unsigned long long)(all[i] != 0) << i;
  return m;
}
static int __popcll(unsigned long long v) { return __builtin_popcountll(v); }
static int __builtin_amdgcn_readlane(int v, int lane) {
  if (lane < 0 || lane >= kLanes) abort();
  return (int)exchange(v)[lane];
}
static int __builtin_amdgcn_readfirstlane(int v) { return (int)exchange(v)[0]; }
static int __builtin_amdgcn_ds_bpermute(int address, int v) { return (int)exchange(v)[address >> 2 & 63]; }

#include "sequences.inc"

struct Case { Sequences q; int tile, top, first, period; };                // rows of the lanes: first + lane % period
static Case now;
static Span spans[kLanes];
static void lane_main(int lane) {
  const int bottom = now.top + now.tile <= now.q.rows ? now.top + now.tile - 1 : now.q.rows - 1;
  spans[lane] = span_of(now.q, now.first + lane % now.period, now.top, bottom);
  done[lane] = true;
  swapcontext(&fibers[lane], &scheduler);
}
static void run() {
  for (int i = 0; i < kLanes; ++i) {
    turns[i] = 0;
    done[i] = false;
    getcontext(&fibers[i]);
    fibers[i].uc_stack.ss_sp = &stacks[i * kStack];
    fibers[i].uc_stack.ss_size = kStack;
    fibers[i].uc_link = nullptr;
    makecontext(&fibers[i], (void (*)())lane_main, 1, i);
  }
  for (int left = kLanes; left;)
    for (int i = 0; i < kLanes; ++i) {
      if (done[i]) { fprintf(stderr, "a lane ended before the others\n"); exit(1); }
      threadIdx.x = i;
      swapcontext(&scheduler, &fibers[i]);
      left -= done[i];
    }
}

static int64_t inside(int64_t v, int rows) { return v < 0 ? 0 : v < rows ? v : rows; }
// The sequence of a row by looking at all from `from` on (those before are empty).
static bool sequence(const Sequences& q, int64_t from, int row, int& begin, int& end) {
  for (int64_t s = from; s < q.n; ++s) {
    const int64_t b = inside(q.offsets[s], q.rows), e = inside(q.offsets[s + 1], q.rows);
    if (b <= row && row < e) { begin = (int)b; end = (int)e; return true; }
  }
  return false;
}
// Every tile of the sizes that kernels have, and every row of a wavefront in it.
static int check(const Sequences& q, int64_t from, const char* name) {
  static const int tiles[3] = {128, 32, 8};
  for (int tile : tiles)
    for (int top = 0; top < q.rows; top += tile)
      for (int first = top; first < top + tile; first += 32) {
        now = Case{q, tile, top, first, tile < 32 ? tile : 32};
        run();
        const int bottom = top + tile <= q.rows ? top + tile - 1 : q.rows - 1;
        int top_begin = top, bottom_end = bottom + 1, none;
        sequence(q, from, top, top_begin, none);
        sequence(q, from, bottom, none, bottom_end);
        for (int i = 0; i < kLanes; ++i) {
          const int row = now.first + i % now.period;
          int begin = 0, end = 0;
          sequence(q, from, row, begin, end);
          const Span& s = spans[i];
          if (s.begin != begin || s.end != end || s.top_begin != top_begin || s.bottom_end != bottom_end) {
            printf("%s: tile of %d rows from %d on, row %d of %d: %d..%d, %d %d; %d..%d, %d %d are wanted\n", name, tile, top, row, q.rows, s.begin, s.end,
                   s.top_begin, s.bottom_end, begin, end, top_begin, bottom_end);
            return 1;
          }
        }
      }
  return 0;
}

// list: lines "rows n offsets[0] .. offsets[n]".  many: lines "rows n tail": n sequences, of which the last `tail` have rows / tail rows each and those
// before have none; only the pages that are written, or read as zeros, are there.
int main(int argc, char** argv) {
  long long rows, n, tail;
  int cases = 0;
  const bool many = argc > 1 && argv[1][0] == 'm';
  while (scanf("%lld %lld", &rows, &n) == 2) {
    char name[64];
    snprintf(name, sizeof name, "case %d, %lld sequences", cases++, n);
    if (!many) {
      std::vector<int64_t> at(n + 1);
      for (auto& v : at) {
        long long x;
        if (scanf("%lld", &x) != 1) return 2;
        v = x;
      }
      if (check(Sequences{at.data(), (int)n, (int)rows}, 0, name)) return 1;
    } else {
      if (scanf("%lld", &tail) != 1) return 2;
      const size_t bytes = (size_t)(n + 1) * 8;
      void* p = mmap(nullptr, bytes, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
      if (p == MAP_FAILED) return 2;
      int64_t* at = static_cast<int64_t*>(p);
      for (long long i = 0; i <= tail; ++i) at[n - tail + i] = rows * i / tail;
      if (check(Sequences{at, (int)n, (int)rows}, n - tail, name)) return 1;
      munmap(p, bytes);
    }
  }
  printf("%d cases\n", cases);
  return 0;
}
