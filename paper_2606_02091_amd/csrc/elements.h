// Shared by the training step's kernels and their entry points: elements in 16-byte accesses, conversions, launches by type, and
// the host's checks of arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "device_common.h"
#include "dflare.h"

namespace dflare {

namespace {

constexpr int kT = 256;  // threads per work-group

typedef __bf16 bf16x2_v __attribute__((ext_vector_type(2)));
typedef float f32x2_v __attribute__((ext_vector_type(2)));
struct bf16_t {
  uint16_t b;
};

// The elements of one 16-byte access, as floats.  Conversions to bf16 round to nearest even and keep NaN.
template <typename T>
constexpr int kVec = 16 / sizeof(T);
__device__ __forceinline__ void unpack(u32x4 v, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(v[e] << 16);
    x[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack(u32x4 v, float (&x)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = __uint_as_float(v[e]);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_v{a, b}), bf16x2_v));
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8]) {
  return u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
}
__device__ __forceinline__ u32x4 pack(const float (&x)[4]) {
  return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
__device__ __forceinline__ float to_f(bf16_t v) { return __uint_as_float((uint32_t)v.b << 16); }
__device__ __forceinline__ float to_f(float v) { return v; }
template <typename T>
__device__ __forceinline__ T from_f(float v) {
  if constexpr (std::is_same_v<T, float>) return v;
  else return T{(uint16_t)pack2(v, 0.f)};
}
// the value as it is stored
template <typename T>
__device__ __forceinline__ float rounded(float v) {
  return to_f(from_f<T>(v));
}

// 16 bytes at an address that is a multiple of A
template <int A>
struct __attribute__((packed, aligned(A))) Piece {
  u32x4 v;
};
// VE elements at p: one 16-byte access where VE is kVec<T> (at any element unless ALIGNED), single ones otherwise
template <typename T, int VE, bool ALIGNED = true>
__device__ __forceinline__ void load_n(const T* p, float (&x)[VE]) {
  if constexpr (VE == kVec<T>) unpack(reinterpret_cast<const Piece<ALIGNED ? 16 : sizeof(T)>*>(p)->v, x);
  else {
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = to_f(p[e]);
  }
}
template <typename T, int VE, bool ALIGNED = true>
__device__ __forceinline__ void store_n(T* p, const float (&x)[VE]) {
  if constexpr (VE == kVec<T>) reinterpret_cast<Piece<ALIGNED ? 16 : sizeof(T)>*>(p)->v = pack(x);
  else {
#pragma unroll
    for (int e = 0; e < VE; ++e) p[e] = from_f<T>(x[e]);
  }
}

// VE elements as they lie in memory
template <typename T, int VE, bool ALIGNED>
struct Raw {
  std::conditional_t<VE == kVec<T>, u32x4, T> v;
  __device__ __forceinline__ void load(const T* p) {
    static_assert(VE == kVec<T> || VE == 1);
    if constexpr (VE == 1) v = *p;
    else v = reinterpret_cast<const Piece<ALIGNED ? 16 : sizeof(T)>*>(p)->v;
  }
  __device__ __forceinline__ void get(float (&x)[VE]) const {
    if constexpr (VE == 1) x[0] = to_f(v);
    else unpack(v, x);
  }
};

// A factor 2^e m, m in [0.5, 1]: as one fp32 number it loses its digits where max_norm / norm is below fp32's normal range
// (finite gradients of 1e38)
struct Factor {
  float m;
  int e;
  __device__ __forceinline__ float of(float x) const { return __builtin_amdgcn_ldexpf(x * m, e); }
};

// ---- host side ----

// DFLARE_OK where `stream` (NULL: the default one) belongs to the current device
int stream_ok(void* stream) {
  if (!stream) return DFLARE_OK;
  int dev = -1, sdev = -1;
  if (hipGetDevice(&dev) != hipSuccess || hipStreamGetDevice((hipStream_t)stream, &sdev) != hipSuccess)
    return DFLARE_ERR_HIP;
  return dev == sdev ? DFLARE_OK : DFLARE_ERR_INVALID_ARG;
}
int launched() { return hipGetLastError() == hipSuccess ? DFLARE_OK : DFLARE_ERR_HIP; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
int size_of(int dtype) { return dtype == DFLARE_F32 ? 4 : dtype == DFLARE_BF16 ? 2 : 0; }

constexpr int kGroupsOfLaunch = 1 << 21;  // (a launch has less than 2^32 threads)

template <typename F>
void by_type(int dtype, F&& f) {
  if (dtype == DFLARE_F32) f(float{});
  else f(bf16_t{});
}
template <int N>
using int_c = std::integral_constant<int, N>;
bool misplaced(const void* p, int size) { return ((uintptr_t)p & (size - 1)) != 0; }

// a and b, of the same size, are one tensor or lie apart (or one is NULL)
bool same_or_apart(const void* a, const void* b, size_t bytes) { return a == b || !overlap(a, bytes, b, bytes); }

// The bytes of a rotary tensor: runs of `run` bytes at p + i s[0] + j s[1], i < n[0], j < n[1]
struct Runs {
  __int128 p, s[2];
  long n[2], run;
  Runs(const void* at, long row, long head, int rows, int heads, int hd, int size)
      : p((uintptr_t)at), s{(__int128)row * size, (__int128)head * size}, n{rows, heads}, run((long)hd * size) {
    for (int k = 0; k < 2; ++k) {
      if (n[k] == 1) s[k] = 0;
      if (s[k] < 0) {  // the same runs from the other end
        p += s[k] * (n[k] - 1);
        s[k] = -s[k];
      }
    }
  }
  bool empty() const { return !n[0] || !n[1]; }
  // no two runs overlap: one stride clears the runs, the other clears the whole of these
  bool distinct() const {
    auto nested = [&](int in, int out) {
      return (n[in] == 1 || s[in] >= run) && (n[out] == 1 || s[out] >= s[in] * (n[in] - 1) + run);
    };
    return nested(0, 1) || nested(1, 0);
  }
  // bytes from p to the end of the last run, without the strides that are multiples of m (0: with all)
  __int128 extent(__int128 m) const {
    __int128 e = run;
    for (int k = 0; k < 2; ++k)
      if (!m || s[k] % m) e += s[k] * (n[k] - 1);
    return e;
  }
};
// Their strides show that a and b have no byte in common: by their ends, or because they lie in different parts of
// every period of one of the strides (queries and keys of one buffer).
bool runs_apart(const Runs& a, const Runs& b) {
  if (a.empty() || b.empty()) return true;
  if (a.p + a.extent(0) <= b.p || b.p + b.extent(0) <= a.p) return true;
  for (const __int128 m : {a.s[0], a.s[1], b.s[0], b.s[1]}) {
    if (!m) continue;
    const __int128 to_b = ((b.p - a.p) % m + m) % m;
    if (a.extent(m) <= to_b && to_b + b.extent(m) <= m) return true;
  }
  return false;
}

}  // namespace

}  // namespace dflare
