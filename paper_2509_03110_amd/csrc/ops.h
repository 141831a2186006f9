// What the operators of include/lsam_ops.h share: checks of arguments on the host, and loads and stores of
// values of either type from rows that are aligned to one value only.
#pragma once
#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/lsam_ops.h"

namespace lsam {

void set_last_error(const char* msg);

// `code` with a message for lsam_last_error().
__attribute__((format(printf, 2, 3))) inline int refuse(int code, const char* fmt, ...) {
  char msg[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(msg, sizeof msg, fmt, ap);
  va_end(ap);
  set_last_error(msg);
  return code;
}

inline int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LSAM_OK : refuse(LSAM_EHIP, "%s", hipGetErrorString(e));
}

inline int dtype_bytes(int32_t dtype) { return dtype == LSAM_DTYPE_BF16 ? 2 : 4; }
inline bool known_dtype(int32_t dtype) { return dtype == LSAM_DTYPE_FP32 || dtype == LSAM_DTYPE_BF16; }

// Bytes from the first to behind the last value of `mats` times `rows` rows of `cols` values; -1 where a stride is
// negative, rows overlap, or the last value lies beyond what an address can say.
inline int64_t extent(int64_t mats, int64_t mat_stride, int64_t rows, int64_t stride, int64_t cols, int bytes) {
  if (mats <= 0 || rows <= 0 || cols <= 0) return 0;
  if ((rows > 1 && stride < cols) || (mats > 1 && mat_stride < 0)) return -1;
  const __int128 n = ((__int128)(mats - 1) * (mats > 1 ? mat_stride : 0) + (__int128)(rows - 1) * (rows > 1 ? stride : 0) + cols) * bytes;
  return n < ((__int128)1 << 46) ? (int64_t)n : -1;
}
// Whether the matrices of an output lie apart: one behind the other, or row by row side by side.
inline bool apart(int64_t mats, int64_t mat_stride, int64_t rows, int64_t stride, int64_t cols) {
  if (mats <= 1 || rows <= 0 || cols <= 0) return true;
  const __int128 matrix = (__int128)(rows - 1) * (rows > 1 ? stride : 0) + cols, row = (__int128)(mats - 1) * mat_stride + cols;
  return mat_stride >= cols && ((__int128)mat_stride >= matrix || rows == 1 || (__int128)stride >= row);
}
inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}
inline bool misaligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// An argument: `bytes` from the first to behind the last value, in blocks of `one` bytes whose starts are multiples of `step` apart
// (0: it is one block), the rows of a part of wider rows, say; and, coarser, in blocks of `many` bytes `far` apart, as the
// factors of one vector per replica are.
struct Arg {
  const char* name; const void* p; int64_t bytes; int align; bool output;
  int64_t one = 0, step = 0, many = 0, far = 0;
};
inline int64_t common(int64_t a, int64_t b) {
  while (b) { const int64_t r = a % b; a = b; b = r; }
  return a;
}
// The same for `mats` matrices of `rows` rows, from their first to behind their last value.
inline Arg matrices(const char* name, const void* p, int64_t mats, int64_t mat_stride, int64_t rows, int64_t stride, int64_t cols, int bytes,
                    bool output) {
  Arg a{name, p, extent(mats, mat_stride, rows, stride, cols, bytes), bytes, output};
  if (a.bytes <= 0) return a;
  const int64_t apart = mats > 1 ? mat_stride * bytes : 0;
  a.one = cols * bytes;
  a.step = common(apart, rows > 1 ? stride * bytes : 0);
  a.many = extent(1, 0, rows, stride, cols, bytes);
  a.far = apart;
  return a;
}
// Whether two arguments have a byte in common; where blocks of different strides go through each other, whether they might.
inline bool meet(const Arg& a, const Arg& b) {
  if (!a.p || !b.p || !overlap(a.p, a.bytes, b.p, b.bytes)) return false;
  // blocks of both in turn: all of a's begin at the same place of every g bytes, all of b's at another, and none reaches the other's
  const int64_t size[2][2] = {{a.one, a.many}, {b.one, b.many}}, step[2][2] = {{a.step, a.far}, {b.step, b.far}};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j) {
      const int64_t g = common(step[0][i], step[1][j]), m = size[0][i], n = size[1][j];
      if (!g || !m || !n) continue;
      const int64_t off = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)) % g;
      const int64_t at = off < 0 ? off + g : off;
      if (at >= m && at + n <= g) return false;
    }
  return true;
}
// That arguments are there, aligned and not too large.
inline int check_values(const Arg* args, int n, const char* who) {
  for (int i = 0; i < n; ++i) {
    if (args[i].bytes < 0) return refuse(LSAM_EINVAL, "%s: a stride of %s is too small, or the array is too large", who, args[i].name);
    if (args[i].bytes && !args[i].p) return refuse(LSAM_EINVAL, "%s: %s is NULL", who, args[i].name);
    if (misaligned(args[i].p, args[i].align)) return refuse(LSAM_EINVAL, "%s: %s is not aligned to its values", who, args[i].name);
  }
  return LSAM_OK;
}
// That no output lies over another argument.
inline int check_apart(const Arg* args, int n, const char* who) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < n; ++j)
      if (i != j && args[i].output && meet(args[i], args[j]))
        return refuse(LSAM_EINVAL, "%s: %s lies over %s", who, args[i].name, args[j].name);
  return LSAM_OK;
}
// That the workspace is large enough, aligned, and apart from the arguments.
inline int check_workspace(const Arg* args, int n, const void* workspace, size_t bytes, size_t need, int align, const char* who) {
  if (!need) return LSAM_OK;
  if (!workspace || bytes < need)
    return refuse(LSAM_ENOMEM, "%s: the workspace has %zu bytes, %zu are needed", who, workspace ? bytes : 0, need);
  if (misaligned(workspace, align)) return refuse(LSAM_EINVAL, "%s: the workspace must be %d-byte aligned", who, align);
  for (int i = 0; i < n; ++i)
    if (meet(Arg{"", workspace, (int64_t)need, align, true}, args[i]))
      return refuse(LSAM_EINVAL, "%s: the workspace lies over %s", who, args[i].name);
  return LSAM_OK;
}

#if defined(__HIPCC__)

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Global memory takes wide accesses at any address that a value may have.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u16x8 u16x8_any __attribute__((aligned(2)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));

__device__ __forceinline__ float widen(unsigned short b) { return __builtin_bit_cast(float, (unsigned)b << 16); }
__device__ __forceinline__ unsigned short narrow(float f) { return __builtin_bit_cast(unsigned short, static_cast<__bf16>(f)); }

template <int DTYPE> struct Value;
template <> struct Value<LSAM_DTYPE_FP32> {
  typedef float T;
  static __device__ __forceinline__ float get(const T* p) { return *p; }
  static __device__ __forceinline__ void put(T* p, float v) { *p = v; }
  static __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  }
  static __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    *reinterpret_cast<f32x4_any*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_any*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
};
template <> struct Value<LSAM_DTYPE_BF16> {
  typedef unsigned short T;
  static __device__ __forceinline__ float get(const T* p) { return widen(*p); }
  static __device__ __forceinline__ void put(T* p, float v) { *p = narrow(v); }
  static __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
    const u16x8 a = *reinterpret_cast<const u16x8_any*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = widen(a[e]);
  }
  static __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    u16x8 a;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = narrow(v[e]);
    *reinterpret_cast<u16x8_any*>(p) = a;
  }
};

#endif

}  // namespace lsam
