// Row-wise and element-wise kernels of a draft layer's training step, and their C-ABI entry points:
//   * rotary positions of queries and keys (half and interleaved pairs, part of the head), and the
//     inverse rotation, which is the gradient;
//   * RMSNorm and LayerNorm with an optional residual sum, forward and backward;
//   * the global norm of many gradient tensors, and their clipping.
// All of them are bound by memory, and by launch latency where they are small.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <type_traits>
#include <vector>

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

// ---- rotary positions: pair m of a row at position p turns by p f_m.  A work-group takes RW rows: it puts their
// cosines and sines into LDS (once for all heads) and then walks (row, head, item); an item is the pairs
// of one 16-byte access (half layout: of the two accesses rot / 2 apart), or VE elements past the rotated
// part, which are copied.  The angle is formed and reduced to turns in 64 bits: p f_m in 32 would be off by
// 0.06 radians at position 1,000,000.  8,192 rows of 32 + 8 heads x 128: 33 us, 5.0 TB/s. ----
struct RopeSide {
  const void* x;
  void* y;
  long x_row, x_head, y_row, y_head;
  int heads;
};
struct RopeArgs {
  RopeSide t[2];
  const int32_t* positions;
  const double* freq;
  int rows, B, hd, rot, RW, group0;  // group0: first work-group of the launch
  float scale, sign;
};

template <typename T, int VE, bool HALF>
__global__ __launch_bounds__(kT) void k_rope(RopeArgs a) {
  extern __shared__ float tab[];  // [RW][rot / 2] cosines, then sines
  const int half = a.rot / 2;
  const int row0 = (a.group0 + (int)blockIdx.x) * a.RW, nr = min(a.RW, a.rows - row0);
  float *tc = tab, *ts = tab + a.RW * half;
  for (int i = threadIdx.x; i < nr * half; i += kT) {
    const int r = i / half, m = i - r * half, row = row0 + r;
    const double p = a.positions ? (double)a.positions[row / a.B] + row % a.B : (double)row;
    double t = p * a.freq[m] * 0.15915494309189535;  // turns: / 2 pi
    t -= rint(t);
    float s, c;
    sincospif((float)(2.0 * t), &s, &c);
    tc[i] = c * a.scale;
    ts[i] = s * a.scale * a.sign;
  }
  __syncthreads();
  constexpr int PV = HALF || VE == 1 ? VE : VE / 2;  // pairs of an item
  const int turn = half / PV, items = turn + (a.hd - a.rot) / VE;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const RopeSide& t = a.t[k];
    const int n = nr * t.heads * items;
    for (int i = threadIdx.x; i < n; i += kT) {
      const int s = i / items, it = i - s * items, r = s / t.heads, h = s - r * t.heads;
      const T* x = (const T*)t.x + (long)(row0 + r) * t.x_row + h * t.x_head;
      T* y = (T*)t.y + (row0 + r) * t.y_row + h * t.y_head;
      if (it >= turn) {
        if (x != y) {
          const int at = a.rot + (it - turn) * VE;
          float v[VE];
          load_n<T, VE>(x + at, v);
          store_n<T, VE>(y + at, v);
        }
        continue;
      }
      const int m = it * PV;
      const float *pc = tc + r * half + m, *ps = ts + r * half + m;
      if constexpr (HALF) {
        float u[VE], v[VE], p[VE], q[VE];
        load_n<T, VE>(x + m, u);
        load_n<T, VE>(x + m + half, v);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          p[e] = u[e] * pc[e] - v[e] * ps[e];
          q[e] = v[e] * pc[e] + u[e] * ps[e];
        }
        store_n<T, VE>(y + m, p);
        store_n<T, VE>(y + m + half, q);
      } else {
        constexpr int W = VE == 1 ? 2 : VE;
        float u[W], p[W];
        load_n<T, W>(x + 2 * m, u);
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          p[2 * e] = u[2 * e] * pc[e] - u[2 * e + 1] * ps[e];
          p[2 * e + 1] = u[2 * e + 1] * pc[e] + u[2 * e] * ps[e];
        }
        store_n<T, W>(y + 2 * m, p);
      }
    }
  }
}

// ---- norms.  8,192 x 4,096 bf16 with a residual: forward 45 us (268 MB), backward 52 (268 MB and the partials): memory.
// Few rows: latency, 4 us a launch.  WPR waves hold a row in registers, S pieces of VE elements per thread (piece k T + t for thread t
// of the row's T), so that a row is read once and mean and variance are sums over held values.  Rows that do not start or
// end on 16-byte boundaries are read and written in 16-byte pieces all the same; a piece that would pass the
// row's end is the row's last 16 bytes, of which the elements of the piece before take no part (869 x 6,047 bf16, both
// passes: 31 us; by single values 146). ----
struct NormArgs {
  const void *x, *res, *gain, *bias, *dy, *dsum;
  void *sum, *y, *dx;
  const float *mean_in, *rstd_in;
  float *mean, *rstd, *part;
  int rows, H, row0;  // row0: first row of the launch (forward)
  float eps;
};

// threads of a work-group: one row of WPR waves, or four rows of one
template <int WPR>
constexpr int norm_threads = WPR == 1 ? kT : 64 * WPR;

// sum over the row's threads, the same value in each of them (fixed order)
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if constexpr (WPR > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int k = 1; k < WPR; ++k) v += red[k];
  }
  return v;
}

// Piece k of thread t: its first element c, where it lies, and which of its elements it stands for
template <typename T, int VE, bool ALIGNED>
struct RowPiece {
  unsigned c, at, H;
  __device__ __forceinline__ RowPiece(unsigned i, unsigned H_) : c(i * VE), at(min(i * VE, H_ - VE)), H(H_) {}
  __device__ __forceinline__ bool any() const { return c < H; }
  __device__ __forceinline__ bool has(int e) const { return ALIGNED ? c < H : at + e >= c; }
  __device__ __forceinline__ void store(T* row, const float (&x)[VE]) const {
    if (ALIGNED || c + VE <= H) return store_n<T, VE, ALIGNED>(row + c, x);
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (has(e)) row[at + e] = from_f<T>(x[e]);
  }
};

template <typename T, int VE, bool AL, int WPR, int S, bool LAYER>
__global__ __launch_bounds__(norm_threads<WPR>) void k_norm_fwd(NormArgs a) {
  __shared__ float red[16];
  constexpr int TR = 64 * WPR;
  const unsigned t = WPR == 1 ? threadIdx.x % TR : threadIdx.x;
  const long row = a.row0 + (WPR == 1 ? blockIdx.x * 4l + threadIdx.x / TR : (long)blockIdx.x);
  if (WPR == 1 && row >= a.rows) return;  // (WPR > 1: one row per work-group, all of them in range)
  const unsigned H = a.H;
  const long at = row * H;
  const T *x = (const T*)a.x + at, *res = (const T*)a.res + at, *gain = (const T*)a.gain, *bias = (const T*)a.bias;
  T *sum = (T*)a.sum + at, *y = (T*)a.y + at;
  auto piece = [&](int k) { return RowPiece<T, VE, AL>(k * TR + t, H); };
  float h[S][VE];
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const auto p = piece(k);
    load_n<T, VE, AL>(x + p.at, h[k]);
#pragma unroll
    for (int e = 0; e < VE; ++e) h[k][e] = p.has(e) ? h[k][e] : 0.f;
  }
  if (a.res) {
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const auto p = piece(k);
      float r[VE];
      load_n<T, VE, AL>(res + p.at, r);
#pragma unroll
      for (int e = 0; e < VE; ++e) h[k][e] = p.has(e) ? rounded<T>(h[k][e] + r[e]) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const auto p = piece(k);
      if (p.any()) p.store(sum, h[k]);
    }
  }
  float mu = 0.f;
  if constexpr (LAYER) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < S; ++k)
#pragma unroll
      for (int e = 0; e < VE; ++e) s += h[k][e];
    mu = row_sum<WPR>(s, red) / (float)H;  // (divided, not scaled: exact for constant rows)
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const auto p = piece(k);
#pragma unroll
      for (int e = 0; e < VE; ++e) h[k][e] = p.has(e) ? h[k][e] - mu : 0.f;
    }
  }
  float q = 0.f;
#pragma unroll
  for (int k = 0; k < S; ++k)
#pragma unroll
    for (int e = 0; e < VE; ++e) q = fmaf(h[k][e], h[k][e], q);
  const float rstd = 1.f / sqrtf(row_sum<WPR>(q, red) / (float)H + a.eps);
  if (t == 0) {
    a.rstd[row] = rstd;
    if constexpr (LAYER) a.mean[row] = mu;
  }
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const auto p = piece(k);
    if (!p.any()) continue;
    float g[VE], b[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      g[e] = 1.f;
      b[e] = 0.f;
    }
    if (a.gain) load_n<T, VE, AL>(gain + p.at, g);
    if (LAYER && a.bias) load_n<T, VE, AL>(bias + p.at, b);
#pragma unroll
    for (int e = 0; e < VE; ++e) h[k][e] = fmaf(h[k][e] * rstd, g[e], b[e]);
    p.store(y, h[k]);
  }
}

// Backward: dx of every row, and per work-group the sums over its rows of dy xhat and dy (part[work-group][1 or 2][H]),
// which k_norm_cols adds up in a fixed order.
template <typename T, int VE, bool AL, int WPR, int S, bool LAYER>
__global__ __launch_bounds__(norm_threads<WPR>) void k_norm_bwd(NormArgs a) {
  __shared__ float red[16];
  constexpr int TR = 64 * WPR, RG = norm_threads<WPR> / TR;
  const unsigned t = WPR == 1 ? threadIdx.x % TR : threadIdx.x;
  const int sub = WPR == 1 ? threadIdx.x / TR : 0;
  const unsigned H = a.H;
  const T* gain = (const T*)a.gain;
  float dg[S][VE], db[LAYER ? S : 1][VE];
#pragma unroll
  for (int k = 0; k < S; ++k)
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      dg[k][e] = 0.f;
      db[LAYER ? k : 0][e] = 0.f;
    }
  // a row's values as they lie in memory, loaded (where registers allow it) while the row before is worked on
  constexpr bool AHEAD = WPR <= 4 && S * VE <= 16;
  const int stride = gridDim.x * RG;
  auto piece = [&](int k) { return RowPiece<T, VE, AL>(k * TR + t, H); };
  Raw<T, VE, AL> nx[S], nd[S], ns[S] = {};
  auto fetch = [&](long row) {
    const long at = min(row, a.rows - 1l) * H;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const unsigned c = piece(k).at;
      nx[k].load((const T*)a.x + at + c);
      nd[k].load((const T*)a.dy + at + c);
      if (a.dsum) ns[k].load((const T*)a.dsum + at + c);
    }
  };
  if constexpr (AHEAD) fetch(blockIdx.x * RG + sub);
  for (long row = blockIdx.x * RG + sub; row < a.rows; row += stride) {
    if constexpr (!AHEAD) fetch(row);
    T* dx = (T*)a.dx + row * H;
    const float rstd = a.rstd_in[row], mu = LAYER ? a.mean_in[row] : 0.f;
    float xh[S][VE], d[S][VE];
    Raw<T, VE, AL> rs[S];
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const auto p = piece(k);
      nx[k].get(xh[k]);
      nd[k].get(d[k]);
      rs[k] = ns[k];
#pragma unroll
      for (int e = 0; e < VE; ++e) {  // (past the row no part in the sums)
        xh[k][e] = p.has(e) ? xh[k][e] : mu;
        d[k][e] = p.has(e) ? d[k][e] : 0.f;
      }
    }
    if constexpr (AHEAD) fetch(row + stride);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      float g[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) g[e] = 1.f;
      if (gain) load_n<T, VE, AL>(gain + piece(k).at, g);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        xh[k][e] = (xh[k][e] - mu) * rstd;
        dg[k][e] = fmaf(d[k][e], xh[k][e], dg[k][e]);
        if constexpr (LAYER) db[k][e] += d[k][e];
        d[k][e] *= g[e];
        if constexpr (LAYER) s1 += d[k][e];
        s2 = fmaf(d[k][e], xh[k][e], s2);
      }
    }
    if constexpr (LAYER) s1 = row_sum<WPR>(s1, red) / (float)H;
    s2 = row_sum<WPR>(s2, red) / (float)H;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const auto p = piece(k);
      if (!p.any()) continue;
      float r[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) r[e] = 0.f;
      if (a.dsum) rs[k].get(r);
#pragma unroll
      for (int e = 0; e < VE; ++e) r[e] += rstd * ((LAYER ? d[k][e] - s1 : d[k][e]) - xh[k][e] * s2);
      p.store(dx, r);
    }
  }
  float* part = a.part + ((long)blockIdx.x * RG + sub) * (LAYER ? 2 : 1) * H;
#pragma unroll
  for (int k = 0; k < S; ++k) {
    const auto p = piece(k);
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (p.has(e)) {
        part[p.at + e] = dg[k][e];
        if constexpr (LAYER) part[H + p.at + e] = db[k][e];
      }
  }
}

// out[c] = sum over the parts of column c (16 groups of parts, then these in order); n = H or 2 H columns, of
// which the second H go to dbias
__global__ __launch_bounds__(kT) void k_norm_cols(const float* part, int parts, int n, int H, float* dgain, float* dbias) {
  __shared__ float s[16][17];
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, c = blockIdx.x * 16 + l;
  float v = 0.f;
  if (c < n) {
#pragma unroll 16
    for (int p = g; p < parts; p += 16) v += part[(long)p * n + c];
  }
  s[g][l] = v;
  __syncthreads();
  if (g == 0 && c < n) {
    for (int k = 1; k < 16; ++k) v += s[k][l];
    if (c < H) dgain[c] = v;
    else if (dbias) dbias[c - H] = v;
  }
}

// ---- gradients.  The tensors of a launch are in its arguments; each is cut into chunks of kChunk 16-byte
// pieces counted from its first aligned element, and a work-group takes a contiguous range of the chunks.
// Squares are formed and summed in 64 bits, in an order that the sizes alone set.  1.6 G bf16 values: norm 534 us (6.0 TB/s),
// clipping 1,290 (5.0 TB/s, a copy's rate); 301 small tensors: launches of 5-7 us. ----
constexpr int kChunk = 2048;  // 16-byte pieces of a chunk
constexpr int kGradGroups = 2048;
// A table of up to N tensors, as many as a launch's arguments (4 KB) hold: 230 that are read or scaled in place,
// 160 with outputs of their own.
template <bool OUT>
struct GradTab {
  static constexpr int N = OUT ? 160 : 230;
  const void* p[N];
  void* out[OUT ? N : 1];
  uint32_t n[N];     // elements, the low 32 bits
  int first[N + 1];  // chunks before the tensor
  uint8_t tag[N];    // 1: fp32; the high bits of n above
  int count;
  __device__ __forceinline__ bool f32(int i) const { return tag[i] & 1; }
  __device__ __forceinline__ long size(int i) const { return (long)n[i] | (long)(tag[i] >> 1) << 32; }
  __device__ __forceinline__ void* to(int i) const { return OUT ? out[i] : const_cast<void*>(p[i]); }
};
static_assert(sizeof(GradTab<true>) <= 4048 && sizeof(GradTab<false>) <= 4048, "kernel arguments");

// f(tensor, first element, end) for every range of the work-group's chunks
template <typename TAB, typename F>
__device__ __forceinline__ void grad_walk(const TAB& tab, F&& f) {
  const long total = tab.first[tab.count];
  int c = (int)(total * blockIdx.x / gridDim.x);
  const int end = (int)(total * (blockIdx.x + 1) / gridDim.x);
  if (c >= end) return;
  int lo = 0, hi = tab.count - 1;  // the last tensor whose first chunk is not after c
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (tab.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  for (; c < end; ++c) {
    while (tab.first[lo + 1] <= c) ++lo;
    f(lo, c - tab.first[lo]);
  }
}
__device__ __forceinline__ int lead(const void* p, int size) {  // elements before the first 16-byte boundary
  return (int)((0u - (unsigned)(uintptr_t)p) & 15u) / size;
}

template <typename T>
__device__ __forceinline__ double chunk_sumsq(const T* p, long n, int c) {
  constexpr int VE = kVec<T>;
  const long head = min((long)lead(p, sizeof(T)), n), np = (n - head) / VE;
  const long e0 = (long)c * kChunk, e1 = min(e0 + kChunk, np);
  double s0 = 0.0, s1 = 0.0;
  auto one = [&](float x) { s0 = fma((double)x, (double)x, s0); };
  if (c == 0 && (int)threadIdx.x < head) one(to_f(p[threadIdx.x]));
  const long tail0 = head + np * VE;
  if (e0 + kChunk >= np && tail0 + threadIdx.x < n) one(to_f(p[tail0 + threadIdx.x]));
#pragma unroll 4
  for (long e = e0 + threadIdx.x; e < e1; e += kT) {
    float x[VE];
    load_n<T, VE>(p + head + e * VE, x);
#pragma unroll
    for (int k = 0; k < VE; k += 2) {
      s0 = fma((double)x[k], (double)x[k], s0);
      s1 = fma((double)x[k + 1], (double)x[k + 1], s1);
    }
  }
  return s0 + s1;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kT) void k_grad_sumsq(GradTab<false> tab, double* part) {
  __shared__ double red[4];
  double s = 0.0;
  grad_walk(tab, [&](int i, int c) {
    s += tab.f32(i) ? chunk_sumsq((const float*)tab.p[i], tab.size(i), c) : chunk_sumsq((const bf16_t*)tab.p[i], tab.size(i), c);
  });
  s = block_sum(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(kT) void k_grad_norm(const double* part, int n, double* sumsq, float* norm) {
  __shared__ double red[4];
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kT) s += part[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) {
    sumsq[0] = s;
    if (norm) norm[0] = (float)sqrt(s);
  }
}

// A factor 2^e m, m in [0.5, 1]: as one fp32 number it loses its digits where max_norm / norm is below fp32's normal range
// (finite gradients of 1e38)
struct Factor {
  float m;
  int e;
  __device__ __forceinline__ float of(float x) const { return __builtin_amdgcn_ldexpf(x * m, e); }
};

// (Streamed stores: 2% faster than others into tensors of their own at 3.2 GB; in place the same within 2% from 4 MB to 3.2 GB, and so
// is a pass that reads the values afterwards.)
template <typename T>
__device__ __forceinline__ void chunk_scale(const T* p, T* o, long n, int c, Factor f) {
  constexpr int VE = kVec<T>;
  const long head = min((long)lead(p, sizeof(T)), n), np = (n - head) / VE;
  const long e0 = (long)c * kChunk, e1 = min(e0 + kChunk, np);
  if (c == 0 && (int)threadIdx.x < head) o[threadIdx.x] = from_f<T>(f.of(to_f(p[threadIdx.x])));
  const long tail = head + np * VE + threadIdx.x;
  if (e0 + kChunk >= np && tail < n) o[tail] = from_f<T>(f.of(to_f(p[tail])));
  if ((((uintptr_t)p ^ (uintptr_t)o) & 15) == 0) {
#pragma unroll 4
    for (long e = e0 + threadIdx.x; e < e1; e += kT) {
      float x[VE];
      load_n<T, VE>(p + head + e * VE, x);
#pragma unroll
      for (int k = 0; k < VE; ++k) x[k] = f.of(x[k]);
      __builtin_nontemporal_store(pack(x), reinterpret_cast<u32x4*>(o + head + e * VE));
    }
  } else {
    for (long e = head + e0 * VE + threadIdx.x; e < head + e1 * VE; e += kT) o[e] = from_f<T>(f.of(to_f(p[e])));
  }
}

// g max_norm / norm where the norm is above max_norm, g otherwise and where the norm is not finite
template <bool OUT>
__global__ __launch_bounds__(kT) void k_grad_clip(GradTab<OUT> tab, const double* sumsq, float max_norm) {
  const double norm = sqrt(sumsq[0]);
  const bool clip = norm > (double)max_norm && norm < (double)INFINITY;
  if (!clip && !OUT) return;
  Factor f{1.f, 0};
  if (clip) f.m = (float)frexp((double)max_norm / norm, &f.e);
  grad_walk(tab, [&](int i, int c) {
    if (!clip && tab.p[i] == tab.to(i)) return;
    if (tab.f32(i)) chunk_scale((const float*)tab.p[i], (float*)tab.to(i), tab.size(i), c, f);
    else chunk_scale((const bf16_t*)tab.p[i], (bf16_t*)tab.to(i), tab.size(i), c, f);
  });
}

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

constexpr int kNormMaxH = 16384;
// f(VE, aligned, WPR, S) of a norm over rows of H
template <typename T, typename F>
void norm_shape(int H, bool aligned, F&& f) {
  constexpr int V = kVec<T>;
  if (H < V) return f(int_c<1>{}, std::true_type{}, int_c<1>{}, int_c<1>{});
  auto sized = [&](auto al) {
    if (H <= 64 * V) f(int_c<V>{}, al, int_c<1>{}, int_c<1>{});
    else if (H <= 128 * V) f(int_c<V>{}, al, int_c<1>{}, int_c<2>{});
    else if (H <= 512 * V) f(int_c<V>{}, al, int_c<4>{}, int_c<2>{});
    else if (H <= 1024 * V) f(int_c<V>{}, al, int_c<4>{}, int_c<4>{});
    else if (H <= 2048 * V) f(int_c<V>{}, al, int_c<8>{}, int_c<4>{});
    else if constexpr (V == 4) f(int_c<V>{}, al, int_c<16>{}, int_c<4>{});  // (bf16 rows end at 16,384)
  };
  if (aligned) sized(std::true_type{});
  else sized(std::false_type{});
}
// Work-groups of the backward pass, each with a partial of the gain's gradient (8,192 x 4,096 bf16, both passes, 256 / 512 /
// 1,024 of them: 115 / 100 / 107 us; not measured at fewer rows, where 777 x 2,881 has two rows a group at most)
constexpr int kNormGroups = 512;
int norm_parts(int rows) { return std::min(std::max(rows, 0), kNormGroups) * 4; }

int norm_check(int rows, int H, int dtype, int kind) {
  if (rows < 0 || H < 1 || !size_of(dtype) || (kind != DFLARE_NORM_RMS && kind != DFLARE_NORM_LAYER))
    return DFLARE_ERR_INVALID_ARG;
  return H > kNormMaxH ? DFLARE_ERR_UNSUPPORTED : DFLARE_OK;
}
bool misplaced(const void* p, int size) { return ((uintptr_t)p & (size - 1)) != 0; }

int grad_check(const dflare_grad_tensor* t, int n) {
  if (n < 0 || (n > 0 && !t)) return DFLARE_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const int size = size_of(t[i].dtype);
    if (!size || t[i].n < 0 || (t[i].n > 0 && !t[i].data)) return DFLARE_ERR_INVALID_ARG;
    if (misplaced(t[i].data, size) || misplaced(t[i].out, size)) return DFLARE_ERR_INVALID_ARG;
    if (t[i].n > (1ll << 36)) return DFLARE_ERR_UNSUPPORTED;  // (a table's tensors then have less than 2^31 chunks)
  }
  return DFLARE_OK;
}

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
// what a call writes meets nothing else that it writes or reads, a tensor turned in place aside
bool rope_apart(const dflare_rope_tensor* t, int n, const int32_t* positions, int n_positions, int rows, int hd, int size) {
  auto x = [&](int k) { return Runs(t[k].x, t[k].x_row, t[k].x_head, rows, t[k].n_heads, hd, size); };
  auto y = [&](int k) { return Runs(t[k].y, t[k].y_row, t[k].y_head, rows, t[k].n_heads, hd, size); };
  for (int k = 0; k < n; ++k) {
    if (!y(k).empty() && !y(k).distinct()) return false;
    if (positions && !runs_apart(y(k), Runs(positions, 0, 0, 1, 1, n_positions, 4))) return false;
    if (t[k].x != t[k].y && !runs_apart(x(k), y(k))) return false;
  }
  return n == 1 || (runs_apart(y(0), y(1)) && runs_apart(y(0), x(1)) && runs_apart(y(1), x(0)));
}

long grad_chunks(const dflare_grad_tensor& t) {
  const int size = size_of(t.dtype);
  const long head = std::min<long>(((0u - (unsigned)(uintptr_t)t.data) & 15u) / size, t.n);
  const long np = (t.n - head) / (16 / size);
  return std::max<long>((np + kChunk - 1) / kChunk, t.n > 0 ? 1 : 0);
}

// f(table, work-groups) for every launch over the tensors (empty ones take no part)
template <bool OUT, typename F>
void grad_launches(const dflare_grad_tensor* t, int n, F&& f) {
  GradTab<OUT> tab;
  tab.count = 0;
  tab.first[0] = 0;
  auto flush = [&] {
    if (tab.count) f(tab, std::min(tab.first[tab.count], kGradGroups));
    tab.count = 0;
  };
  for (int i = 0; i < n; ++i) {
    const long c = grad_chunks(t[i]);
    if (!c) continue;
    if (tab.count == tab.N) flush();
    const int k = tab.count++;
    tab.p[k] = t[i].data;
    if (OUT) tab.out[k] = t[i].out ? t[i].out : t[i].data;
    tab.n[k] = (uint32_t)t[i].n;
    tab.tag[k] = (uint8_t)((t[i].dtype == DFLARE_F32) | (t[i].n >> 32) << 1);
    tab.first[k + 1] = tab.first[k] + (int)c;
  }
  flush();
}

// INVALID_ARG where a tensor written by a clip overlaps another one that it reads or writes, or sumsq
int grad_apart(const dflare_grad_tensor* t, int n, const double* sumsq) try {
  struct Span {
    uintptr_t a, b;
    bool out;
  };
  std::vector<Span> s;
  s.reserve(2 * (size_t)n + 1);
  s.push_back({(uintptr_t)sumsq, (uintptr_t)sumsq + sizeof(double), false});
  for (int i = 0; i < n; ++i) {
    if (!t[i].n) continue;
    const size_t bytes = (size_t)t[i].n * size_of(t[i].dtype);
    const uintptr_t d = (uintptr_t)t[i].data, o = t[i].out ? (uintptr_t)t[i].out : d;
    s.push_back({o, o + bytes, true});
    if (o != d) s.push_back({d, d + bytes, false});
  }
  std::sort(s.begin(), s.end(), [](const Span& x, const Span& y) { return x.a < y.a; });
  uintptr_t end_out = 0, end_any = 0;
  for (const Span& x : s) {
    if (x.a < end_out || (x.out && x.a < end_any)) return DFLARE_ERR_INVALID_ARG;
    end_any = std::max(end_any, x.b);
    if (x.out) end_out = std::max(end_out, x.b);
  }
  return DFLARE_OK;
} catch (const std::bad_alloc&) {
  return DFLARE_ERR_OUT_OF_MEMORY;
}

}  // namespace

}  // namespace dflare

using namespace dflare;

extern "C" {

int dflare_rope_frequencies(int32_t rotary_dim, double base, int32_t method, double factor, double original_len,
                            double* inv_freq, float* scale) {
  if (rotary_dim < 2 || rotary_dim % 2 || !(base > 0.0) || !isfinite(base) || !inv_freq) return DFLARE_ERR_INVALID_ARG;
  if (method < DFLARE_ROPE_PLAIN || method > DFLARE_ROPE_YARN) return DFLARE_ERR_INVALID_ARG;
  if (method != DFLARE_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return DFLARE_ERR_INVALID_ARG;
  if (method == DFLARE_ROPE_YARN && (!(original_len > 0.0) || !isfinite(original_len))) return DFLARE_ERR_INVALID_ARG;
  const int d = rotary_dim;
  if (method == DFLARE_ROPE_NTK && d > 2) base *= pow(factor, (double)d / (d - 2));
  for (int m = 0; m < d / 2; ++m) {
    double f = pow(base, -2.0 * m / d);
    if (method == DFLARE_ROPE_LINEAR) f /= factor;
    if (method == DFLARE_ROPE_YARN) {
      const double turns = original_len * f / 6.283185307179586;
      const double keep = std::min(std::max((turns - 1.0) / 31.0, 0.0), 1.0);
      f = f * keep + f / factor * (1.0 - keep);
    }
    inv_freq[m] = f;
  }
  if (scale) *scale = method == DFLARE_ROPE_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.f;
  return DFLARE_OK;
}

int dflare_rope(const dflare_rope_tensor* tensors, int32_t n_tensors, const int32_t* positions, const double* inv_freq,
                int32_t rows, int32_t B, int32_t head_dim, int32_t rotary_dim, int32_t dtype, int32_t layout,
                float scale, int32_t inverse, void* stream) {
  const int size = size_of(dtype);
  if (!tensors || n_tensors < 1 || n_tensors > 2 || !inv_freq || rows < 0 || B < 1 || !size) return DFLARE_ERR_INVALID_ARG;
  if (head_dim < 2 || rotary_dim < 2 || rotary_dim % 2 || rotary_dim > head_dim) return DFLARE_ERR_INVALID_ARG;
  if (layout != DFLARE_ROPE_HALF && layout != DFLARE_ROPE_INTERLEAVED) return DFLARE_ERR_INVALID_ARG;
  if (!isfinite(scale) || misplaced(positions, 4) || misplaced(inv_freq, 8)) return DFLARE_ERR_INVALID_ARG;
  if (head_dim > 1024) return DFLARE_ERR_UNSUPPORTED;
  RopeArgs a{};
  bool wide = true;
  long work = 0;
  const int ve = 16 / size;
  for (int k = 0; k < n_tensors; ++k) {
    const dflare_rope_tensor& t = tensors[k];
    if (t.n_heads < 0) return DFLARE_ERR_INVALID_ARG;
    if ((long)t.n_heads * head_dim > (1l << 20)) return DFLARE_ERR_UNSUPPORTED;
    if (rows > 0 && t.n_heads > 0 && (!t.x || !t.y)) return DFLARE_ERR_INVALID_ARG;
    if (misplaced(t.x, size) || misplaced(t.y, size)) return DFLARE_ERR_INVALID_ARG;
    if (t.x == t.y && (t.x_row != t.y_row || t.x_head != t.y_head)) return DFLARE_ERR_INVALID_ARG;
    a.t[k] = {t.x, t.y, t.x_row, t.x_head, t.y_row, t.y_head, t.n_heads};
    wide = wide && aligned16(t.x) && aligned16(t.y) && ((t.x_row | t.x_head | t.y_row | t.y_head) & (ve - 1)) == 0;
    work += t.n_heads;
  }
  if (rows == 0 || work == 0) return DFLARE_OK;
  const int n_positions = (int)((rows + B - 1l) / B);
  if (!rope_apart(tensors, n_tensors, positions, n_positions, rows, head_dim, size)) return DFLARE_ERR_INVALID_ARG;
  const int rc = stream_ok(stream);
  if (rc != DFLARE_OK) return rc;
  const int half = rotary_dim / 2;
  wide = wide && head_dim % ve == 0 && rotary_dim % ve == 0 && (layout != DFLARE_ROPE_HALF || half % ve == 0);
  a.positions = positions;
  a.freq = inv_freq;
  a.rows = rows;
  a.B = B;
  a.hd = head_dim;
  a.rot = rotary_dim;
  a.scale = scale;
  a.sign = inverse ? -1.f : 1.f;
  a.RW = std::max(1, std::min(kT / half, rows / 1024));
  const int groups = (int)((rows + a.RW - 1l) / a.RW);
  const size_t lds = (size_t)a.RW * half * 8;
  by_type(dtype, [&](auto z) {
    using T = decltype(z);
    auto go = [&](auto ve_c) {
      constexpr int VE = decltype(ve_c)::value;
      for (long g = 0; g < groups; g += kGroupsOfLaunch) {
        const dim3 grid((unsigned)std::min<long>(groups - g, kGroupsOfLaunch));
        a.group0 = (int)g;
        if (layout == DFLARE_ROPE_HALF)
          hipLaunchKernelGGL((k_rope<T, VE, true>), grid, dim3(kT), lds, (hipStream_t)stream, a);
        else
          hipLaunchKernelGGL((k_rope<T, VE, false>), grid, dim3(kT), lds, (hipStream_t)stream, a);
      }
    };
    if (wide) go(int_c<kVec<T>>{});
    else go(int_c<1>{});
  });
  return launched();
}

int dflare_norm_fwd(const void* x, const void* residual, const void* gain, const void* bias, int32_t rows, int32_t H,
                    int32_t dtype, int32_t kind, float eps, void* sum, void* y, float* mean, float* rstd, void* stream) {
  int rc = norm_check(rows, H, dtype, kind);
  if (rc != DFLARE_OK) return rc;
  const bool layer = kind == DFLARE_NORM_LAYER;
  const int size = size_of(dtype);
  if (!(eps >= 0.f) || !isfinite(eps) || (!layer && bias)) return DFLARE_ERR_INVALID_ARG;
  if (rows > 0 && (!x || !y || !rstd || (layer && !mean) || (residual && !sum))) return DFLARE_ERR_INVALID_ARG;
  for (const void* p : {x, residual, gain, bias, (const void*)sum, (const void*)y})
    if (misplaced(p, size)) return DFLARE_ERR_INVALID_ARG;
  if (misplaced(rstd, 4) || (layer && misplaced(mean, 4))) return DFLARE_ERR_INVALID_ARG;
  const size_t bytes = (size_t)rows * H * size;
  for (const void* p : {x, residual})
    if (!same_or_apart(y, p, bytes) || (residual && !same_or_apart(sum, p, bytes))) return DFLARE_ERR_INVALID_ARG;
  for (const void* p : {gain, bias})
    if (overlap(y, bytes, p, (size_t)H * size) || (residual && overlap(sum, bytes, p, (size_t)H * size))) return DFLARE_ERR_INVALID_ARG;
  if (residual && overlap(sum, bytes, y, bytes)) return DFLARE_ERR_INVALID_ARG;
  if (rows == 0) return DFLARE_OK;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  bool wide = (long)H * size % 16 == 0;
  // a row's statistics are written while other rows are read
  const size_t rb = (size_t)rows * 4, hb = (size_t)H * size;
  if (!apart({{rstd, rb}, {layer ? mean : nullptr, rb}},
             {{x, bytes}, {residual, bytes}, {gain, hb}, {bias, hb}, {residual ? sum : nullptr, bytes}, {y, bytes}}))
    return DFLARE_ERR_INVALID_ARG;
  for (const void* p : {x, residual, gain, bias, (const void*)sum, (const void*)y}) wide = wide && aligned16(p);
  NormArgs a{};
  a.x = x;
  a.res = residual;
  a.gain = gain;
  a.bias = bias;
  a.sum = sum;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  a.rows = rows;
  a.H = H;
  a.eps = eps;
  by_type(dtype, [&](auto z) {
    using T = decltype(z);
    norm_shape<T>(H, wide, [&](auto ve, auto al, auto wpr, auto s) {
      constexpr int VE = decltype(ve)::value, WPR = decltype(wpr)::value, S = decltype(s)::value, RG = WPR == 1 ? 4 : 1;
      constexpr bool AL = decltype(al)::value;
      for (long r = 0; r < rows; r += (long)kGroupsOfLaunch * RG) {
        const dim3 grid((unsigned)std::min<long>((rows - r + RG - 1) / RG, kGroupsOfLaunch));
        a.row0 = (int)r;
        if (layer) hipLaunchKernelGGL((k_norm_fwd<T, VE, AL, WPR, S, true>), grid, dim3(norm_threads<WPR>), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((k_norm_fwd<T, VE, AL, WPR, S, false>), grid, dim3(norm_threads<WPR>), 0, (hipStream_t)stream, a);
      }
    });
  });
  return launched();
}

size_t dflare_norm_bwd_workspace(int32_t rows, int32_t H, int32_t kind) {
  if (rows < 0 || H < 1 || H > kNormMaxH) return 0;
  return std::max<size_t>(16, (size_t)norm_parts(rows) * H * 4 * (kind == DFLARE_NORM_LAYER ? 2 : 1));
}

int dflare_norm_bwd(const void* dy, const void* h, const void* gain, const float* mean, const float* rstd,
                    const void* dsum, int32_t rows, int32_t H, int32_t dtype, int32_t kind, void* dx, float* dgain,
                    float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = norm_check(rows, H, dtype, kind);
  if (rc != DFLARE_OK) return rc;
  const bool layer = kind == DFLARE_NORM_LAYER;
  const int size = size_of(dtype);
  if (!dgain || !workspace || (!layer && dbias)) return DFLARE_ERR_INVALID_ARG;
  if (rows > 0 && (!dy || !h || !rstd || !dx || (layer && !mean))) return DFLARE_ERR_INVALID_ARG;
  if (workspace_bytes < dflare_norm_bwd_workspace(rows, H, kind) || misplaced(workspace, 16)) return DFLARE_ERR_INVALID_ARG;
  for (const void* p : {dy, h, gain, dsum, (const void*)dx})
    if (misplaced(p, size)) return DFLARE_ERR_INVALID_ARG;
  for (const float* p : {rstd, (const float*)dgain, (const float*)dbias, layer ? mean : nullptr})
    if (misplaced(p, 4)) return DFLARE_ERR_INVALID_ARG;
  for (const void* p : {dy, h, dsum})
    if (!same_or_apart(dx, p, (size_t)rows * H * size)) return DFLARE_ERR_INVALID_ARG;
  // the inputs are read until the last row; dgain and dbias are written after that
  const size_t bytes = (size_t)rows * H * size, rb = (size_t)rows * 4, hb = (size_t)H * 4, gb = (size_t)H * size;
  const size_t wb = dflare_norm_bwd_workspace(rows, H, kind);
  const float* mu = layer ? mean : nullptr;
  if (!apart({{dx, bytes}}, {{gain, gb}, {mu, rb}, {rstd, rb}}) ||
      !apart({{workspace, wb}}, {{dy, bytes}, {h, bytes}, {dsum, bytes}, {gain, gb}, {mu, rb}, {rstd, rb}}) ||
      !apart({{dx, bytes}, {dgain, hb}, {dbias, hb}, {workspace, wb}}, {}))
    return DFLARE_ERR_INVALID_ARG;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  bool wide = (long)H * size % 16 == 0;
  for (const void* p : {dy, h, gain, dsum, (const void*)dx}) wide = wide && aligned16(p);
  NormArgs a{};
  a.x = h;
  a.dy = dy;
  a.gain = gain;
  a.dsum = dsum;
  a.dx = dx;
  a.mean_in = mean;
  a.rstd_in = rstd;
  a.part = (float*)workspace;
  a.rows = rows;
  a.H = H;
  int parts = 0;
  if (rows > 0)
    by_type(dtype, [&](auto z) {
      using T = decltype(z);
      norm_shape<T>(H, wide, [&](auto ve, auto al, auto wpr, auto s) {
        constexpr int VE = decltype(ve)::value, WPR = decltype(wpr)::value, S = decltype(s)::value, RG = WPR == 1 ? 4 : 1;
        constexpr bool AL = decltype(al)::value;
        const int grid = (int)std::min<long>((rows + RG - 1l) / RG, kNormGroups);
        parts = grid * RG;
        if (layer) hipLaunchKernelGGL((k_norm_bwd<T, VE, AL, WPR, S, true>), dim3(grid), dim3(norm_threads<WPR>), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((k_norm_bwd<T, VE, AL, WPR, S, false>), dim3(grid), dim3(norm_threads<WPR>), 0, (hipStream_t)stream, a);
      });
    });
  const int n = layer ? 2 * H : H;
  hipLaunchKernelGGL(k_norm_cols, dim3((n + 15) / 16), dim3(kT), 0, (hipStream_t)stream, a.part, parts, n, H, dgain, dbias);
  return launched();
}

size_t dflare_grad_norm_workspace(int32_t n) {
  return n < 0 ? 0 : ((size_t)(n / GradTab<false>::N + 1) * kGradGroups + 8) * 8;
}

int dflare_grad_norm(const dflare_grad_tensor* tensors, int32_t n, double* sumsq, float* norm, void* workspace,
                     size_t workspace_bytes, void* stream) {
  int rc = grad_check(tensors, n);
  if (rc != DFLARE_OK) return rc;
  if (!sumsq || !workspace || misplaced(sumsq, 8) || misplaced(norm, 4) || misplaced(workspace, 8) ||
      workspace_bytes < dflare_grad_norm_workspace(n))
    return DFLARE_ERR_INVALID_ARG;
  // the partial sums are written while the gradients are read, the results while the partial sums are
  const Bytes work{workspace, dflare_grad_norm_workspace(n)};
  if (!apart({work, {sumsq, 8}, {norm, 4}}, {})) return DFLARE_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i)
    if (!apart({work, {sumsq, 8}, {norm, 4}}, {{tensors[i].data, (size_t)tensors[i].n * size_of(tensors[i].dtype)}})) return DFLARE_ERR_INVALID_ARG;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  double* part = (double*)workspace;
  int used = 0;
  grad_launches<false>(tensors, n, [&](const GradTab<false>& tab, int groups) {
    hipLaunchKernelGGL(k_grad_sumsq, dim3(groups), dim3(kT), 0, (hipStream_t)stream, tab, part + used);
    used += groups;
  });
  hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(kT), 0, (hipStream_t)stream, part, used, sumsq, norm);
  return launched();
}

int dflare_clip_grads(const dflare_grad_tensor* tensors, int32_t n, const double* sumsq, float max_norm, void* stream) {
  int rc = grad_check(tensors, n);
  if (rc != DFLARE_OK) return rc;
  if (!sumsq || misplaced(sumsq, 8) || !(max_norm >= 0.f)) return DFLARE_ERR_INVALID_ARG;
  if ((rc = grad_apart(tensors, n, sumsq)) != DFLARE_OK) return rc;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  bool out = false;
  for (int i = 0; i < n; ++i) out |= tensors[i].out && tensors[i].out != tensors[i].data;
  auto go = [&](const auto& tab, int groups) {
    using TAB = std::decay_t<decltype(tab)>;
    hipLaunchKernelGGL((k_grad_clip<TAB::N == GradTab<true>::N>), dim3(groups), dim3(kT), 0, (hipStream_t)stream, tab, sumsq, max_norm);
  };
  if (out) grad_launches<true>(tensors, n, go);
  else grad_launches<false>(tensors, n, go);
  return launched();
}

}  // extern "C"
