// The norm of each query and key head with its rotary position, in one pass over them, forward and backward, and their C-ABI
// entry points.  A head x at position p, with the gain g of its kind and the turn R(p):
//   n = x / sqrt(mean of x^2 + eps),  y = scale R(p) (n g)
//   d = scale R(-p) dy, e = d g,  dx = (e - n mean(e n)) / sqrt(mean of x^2 + eps),  dg = sum of d n over rows and heads
// Bound by memory: a head is read and written once (twice read, x and dy, going back); everything between stays in registers.
// 8,192 rows x 40 heads x 128 bf16: forward 35 to 37 us (168 MB, 4.6 TB/s), backward 52 (252 MB, 4.9 TB/s), a copy's rate on this card.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dflare.h"
#include "elements.h"

namespace dflare {

namespace {

struct Side {
  const void *x, *dy, *gain;
  void* y;  // y, or dx
  float* dgain;
  long x_row, x_head, dy_row, dy_head, y_row, y_head;
  int heads, groups;  // groups: work-groups, each of a contiguous part of the tensor's heads, row by row
};
struct Args {
  Side t[2];
  const int32_t* positions;
  const double* freq;
  float* part;  // [work-groups][hd] sums of the gains' gradients
  int rows, B, hd, rot, table_rows;  // table_rows: rows whose cosines and sines LDS holds
  float scale, inv, eps;        // inv: 1 / hd
};

// VE elements of type T at any element, in one access
template <typename T, int VE>
struct Access {
  struct __attribute__((packed, aligned(sizeof(T)))) Some {
    T v[VE];
  };
  Some v;
  __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const Some*>(p); }
  __device__ __forceinline__ void ones() {
#pragma unroll
    for (int e = 0; e < VE; ++e) v.v[e] = from_f<T>(1.f);
  }
  __device__ __forceinline__ void get(float* x) const {
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = to_f(v.v[e]);
  }
};
template <typename T>
struct Access<T, kVec<T>> {
  u32x4 v;
  __device__ __forceinline__ void load(const T* p) { v = reinterpret_cast<const Piece<sizeof(T)>*>(p)->v; }
  __device__ __forceinline__ void ones() {
    constexpr uint32_t one = sizeof(T) == 4 ? 0x3F800000u : 0x3F803F80u;
    v = u32x4{one, one, one, one};
  }
  __device__ __forceinline__ void get(float* x) const {
    float u[kVec<T>];
    unpack(v, u);
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) x[e] = u[e];
  }
};
template <typename T, int VE>
__device__ __forceinline__ void put(T* p, const float* x) {
  if constexpr (VE == kVec<T>) {
    float u[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) u[e] = x[e];
    reinterpret_cast<Piece<sizeof(T)>*>(p)->v = pack(u);
  } else {
    typename Access<T, VE>::Some s;
#pragma unroll
    for (int e = 0; e < VE; ++e) s.v[e] = from_f<T>(x[e]);
    *reinterpret_cast<typename Access<T, VE>::Some*>(p) = s;
  }
}

// An item of a head: pairs of elements, in VE floats and VE more rot / 2 elements on (half layout) or in max(VE, 2) side by side; or,
// past the rotated part, VE elements.  E floats; those that an item lacks are 0.
template <typename T, int VE, bool HALF>
struct Item {
  static constexpr int PV = HALF || VE == 1 ? VE : VE / 2, W = HALF ? VE : VE == 1 ? 2 : VE, E = HALF ? 2 * VE : W;
  struct Bits {
    Access<T, W> a;
    Access<T, HALF ? VE : 1> b;
  };
  int m, at;  // first pair, or -1 past the rotated part; first element
  bool any;
  __device__ __forceinline__ Item(int it, int items, int half, int rot) {
    const int turn = half / PV;
    any = it < items;
    m = any && it < turn ? it * PV : -1;
    at = it < turn ? (HALF ? it * PV : 2 * it * PV) : rot + (it - turn) * VE;
  }
  __device__ __forceinline__ void load(const T* p, int half, Bits& r) const {
    if (!any) return;
    if constexpr (W != VE) {
      if (m < 0) {  // (one element)
        r.a.v.v[0] = p[at];
        return;
      }
    }
    r.a.load(p + at);
    if constexpr (HALF) {
      if (m >= 0) r.b.load(p + at + half);
    }
  }
  __device__ __forceinline__ void get(const Bits& r, float (&x)[E]) const {
    r.a.get(x);
    if constexpr (HALF) r.b.get(x + VE);
    if (m >= 0) return;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e >= VE || !any) x[e] = 0.f;
  }
  __device__ __forceinline__ void store(T* p, int half, const float (&x)[E]) const {
    if (!any) return;
    if constexpr (W != VE) {
      if (m < 0) {
        p[at] = from_f<T>(x[0]);
        return;
      }
    }
    put<T, W>(p + at, x);
    if constexpr (HALF) {
      if (m >= 0) put<T, VE>(p + at + half, x + VE);
    }
  }
  // element of the head that float e is (e < VE past the rotated part)
  __device__ __forceinline__ int element(int e, int half) const { return HALF && e >= VE ? at + half + e - VE : at + e; }
  // by the angles of the row whose cosines and sines (sign times) lie at c and s
  __device__ __forceinline__ void turn(const float* c, const float* s, float sign, float (&x)[E]) const {
    if (m < 0) return;
#pragma unroll
    for (int e = 0; e < PV; ++e) {
      const int i = HALF ? e : 2 * e, j = HALF ? VE + e : 2 * e + 1;
      const float a = x[i], b = x[j], cs = c[m + e], sn = sign * s[m + e];
      x[i] = a * cs - b * sn;
      x[j] = b * cs + a * sn;
    }
  }
};

// cosines and sines of nr rows from row0 on (angles formed and reduced in 64 bits: p f in 32 would be off by 0.06 at position 1,000,000)
__device__ __forceinline__ void angles(const Args& a, int row0, int nr, float* tc, float* ts) {
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < nr * half; i += kT) {
    const int r = i / half, m = i - r * half, row = row0 + r;
    const double p = a.positions ? (double)a.positions[row / a.B] + row % a.B : (double)row;
    double t = p * a.freq[m] * 0.15915494309189535;  // turns: / 2 pi
    t -= rint(t);
    float s, c;
    sincospif((float)(2.0 * t), &s, &c);
    tc[i] = c * a.scale;
    ts[i] = s * a.scale;
  }
}

// sum over the L lanes of a head, the same in each of them
template <int L>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int off = L / 2; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// 1 / sqrt(sum / hd + eps), to a unit in the last place (fp32 heads come out 2e-7 off in the 2-norm, with a correctly rounded root
// 1e-7).  The card's root takes numbers below 2^-126 for zero.  BARE: eps is below 2^-90 and does not keep from them, so
// a sum below 2^-90 is multiplied by 2^64 first and the result by 2^32.  (Kernels of their own: with selects for every head 8,192 rows x
// 40 heads x 128 both ways take 2 to 3% longer, with a branch that is one way for the whole launch 3.6% backward.)
template <bool BARE>
__device__ __forceinline__ float rstd_of(const Args& a, float sum) {
  if constexpr (!BARE) return __builtin_amdgcn_rsqf(fmaf(sum, a.inv, a.eps));
  const bool small = sum < 0x1p-90f;
  const float up = small ? 0x1p64f : 1.f;
  return __builtin_amdgcn_rsqf(fmaf(sum * up, a.inv, a.eps * up)) * (small ? 0x1p32f : 1.f);
}

// A head is held by L lanes, S items each; the next one's is on its way while it is worked on.  BACK: dx and the work-group's
// sums of the gain's gradient; otherwise y.
template <typename T, int VE, bool HALF, int L, int S, bool BACK, bool BARE>
__global__ __launch_bounds__(kT, 1) void k_qk(Args a) {
  using I = Item<T, VE, HALF>;
  extern __shared__ float tab[];
  const int half = a.rot / 2, items = half / I::PV + (a.hd - a.rot) / VE, lane = threadIdx.x % L;
  const int k = (int)blockIdx.x >= a.t[0].groups ? 1 : 0, j = blockIdx.x - (k ? a.t[0].groups : 0);
  const Side& t = a.t[k];
  const int heads = t.heads;
  const long n = (long)a.rows * heads;
  const long first = n * j / t.groups, last = n * (j + 1) / t.groups;
  float *tc = tab, *ts = tab + a.table_rows * half;
  typename I::Bits rx[S], rd[BACK ? S : 1];
  long s = first + threadIdx.x / L;
  long fr = s / heads;  // row and head that are fetched next
  int fh = (int)(s - fr * heads);
  const int step_r = kT / L / heads, step_h = kT / L - step_r * heads;
  auto fetch = [&](long s) {
    if (s >= last) return;
    const T* x = (const T*)t.x + fr * t.x_row + fh * t.x_head;
    const T* dy = (const T*)t.dy + fr * t.dy_row + fh * t.dy_head;
    fr += step_r;
    fh += step_h;
    if (fh >= heads) {
      fh -= heads;
      ++fr;
    }
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const I it(lane + i * L, items, half, a.rot);
      it.load(x, half, rx[i]);
      if constexpr (BACK) it.load(dy, half, rd[i]);
    }
  };
  long r = fr;
  int h = fh;
  fetch(s);
  typename I::Bits rg[S];  // (the gain as it lies in memory: half the registers)
  float dg[BACK ? S : 1][I::E];
#pragma unroll
  for (int i = 0; i < S; ++i) {
    rg[i].a.ones();
    rg[i].b.ones();
    if (t.gain) I(lane + i * L, items, half, a.rot).load((const T*)t.gain, half, rg[i]);
    if constexpr (BACK) {
#pragma unroll
      for (int e = 0; e < I::E; ++e) dg[i][e] = 0.f;
    }
  }
  const int row_end = (int)((last + heads - 1) / heads);
  for (int row0 = (int)(first / heads); row0 < row_end; row0 += a.table_rows) {
    const int nr = min(a.table_rows, row_end - row0);
    __syncthreads();  // the rows before are done with
    angles(a, row0, nr, tc, ts);
    __syncthreads();
    const long end = min(last, (long)(row0 + nr) * heads);
    for (; s < end; s += kT / L) {
      const float *c = tc + (r - row0) * half, *sn = ts + (r - row0) * half;
      float v[S][I::E], d[BACK ? S : 1][I::E], q = 0.f, p = 0.f;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const I it(lane + i * L, items, half, a.rot);
        it.get(rx[i], v[i]);
        if constexpr (BACK) it.get(rd[i], d[i]);
      }
      T* y = (T*)t.y + r * t.y_row + h * t.y_head;
      r = fr;
      h = fh;
      fetch(s + kT / L);
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const I it(lane + i * L, items, half, a.rot);
        float g[I::E];
        if constexpr (BACK) {
          it.turn(c, sn, -1.f, d[i]);
          it.get(rg[i], g);
        }
#pragma unroll
        for (int e = 0; e < I::E; ++e) {
          q = fmaf(v[i][e], v[i][e], q);
          if constexpr (BACK) p = fmaf(d[i][e] * g[e], v[i][e], p);
        }
      }
      const float rstd = rstd_of<BARE>(a, head_sum<L>(q));
      float mean = 0.f;
      if constexpr (BACK) mean = head_sum<L>(p) * rstd * a.inv;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const I it(lane + i * L, items, half, a.rot);
        float g[I::E];
        it.get(rg[i], g);
#pragma unroll
        for (int e = 0; e < I::E; ++e) {
          const float nv = v[i][e] * rstd;
          if constexpr (BACK) {
            dg[i][e] = fmaf(d[i][e], nv, dg[i][e]);
            v[i][e] = rstd * (d[i][e] * g[e] - nv * mean);
          } else {
            v[i][e] = nv * g[e];
          }
        }
        if constexpr (!BACK) it.turn(c, sn, 1.f, v[i]);
        it.store(y, half, v[i]);
      }
    }
  }
  if constexpr (BACK) {  // over a wave's heads, then over the four waves, in order
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const I it(lane + i * L, items, half, a.rot);
#pragma unroll
      for (int e = 0; e < I::E; ++e) {
#pragma unroll
        for (int off = L; off < 64; off <<= 1) dg[i][e] += __shfl_xor(dg[i][e], off);
        if ((threadIdx.x & 63) < L && it.any && (it.m >= 0 || e < VE)) tab[(threadIdx.x >> 6) * a.hd + it.element(e, half)] = dg[i][e];
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.hd; e += kT)
      a.part[(long)blockIdx.x * a.hd + e] = (tab[e] + tab[a.hd + e]) + (tab[2 * a.hd + e] + tab[3 * a.hd + e]);
  }
}

// the gains' gradients from the work-groups' sums (64 groups of these, then the groups' in order); work-groups of 1,024 threads take 16
// elements of a gain
__global__ __launch_bounds__(1024) void k_qk_cols(const float* part, int groups0, int groups1, int hd, float* dgain0, float* dgain1) {
  __shared__ float s[64][17];
  const int cols = (hd + 15) / 16, k = (int)blockIdx.x >= cols ? 1 : 0;
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, c = (blockIdx.x - k * cols) * 16 + l;
  const int first = k ? groups0 : 0, n = k ? groups1 : groups0;
  float v = 0.f;
  if (c < hd) {
#pragma unroll 8
    for (int p = g; p < n; p += 64) v += part[(long)(first + p) * hd + c];
  }
  s[g][l] = v;
  __syncthreads();
  float* to = k ? dgain1 : dgain0;
  if (g == 0 && c < hd && to) {
    for (int i = 1; i < 64; ++i) v += s[i][l];
    to[c] = v;
  }
}

// ---- host side ----
constexpr int kMostHead = 512;    // elements of a head: 64 lanes of at most 8 items
constexpr int kFwdGroups = 4096;  // work-groups of a launch, at most about (8,192 rows x 40 heads x 128 bf16, 1,024 / 2,048 / 4,096: 43 / 37 / 35 us)
constexpr int kBwdGroups = 1280;  // (1,024 / 1,280 / 2,048: 55 / 52 / 54 us; 1,280 are what the CUs hold)
constexpr int kTable = 2048;      // pairs of the rows in LDS

int check(int n, const int32_t* positions, const double* freq, int rows, int B, int hd, int rot, int dtype, int layout, float scale, float eps) {
  if (n < 1 || n > 2 || !freq || rows < 0 || B < 1 || !size_of(dtype)) return DFLARE_ERR_INVALID_ARG;
  if (hd < 2 || rot < 2 || rot % 2 || rot > hd) return DFLARE_ERR_INVALID_ARG;
  if (layout != DFLARE_ROPE_HALF && layout != DFLARE_ROPE_INTERLEAVED) return DFLARE_ERR_INVALID_ARG;
  if (!isfinite(scale) || !(eps >= 0.f) || !isfinite(eps) || misplaced(positions, 4) || misplaced(freq, 8)) return DFLARE_ERR_INVALID_ARG;
  return hd > kMostHead ? DFLARE_ERR_UNSUPPORTED : DFLARE_OK;
}
int check_heads(int heads, int hd) {
  if (heads < 0) return DFLARE_ERR_INVALID_ARG;
  return (long)heads * hd > (1l << 20) ? DFLARE_ERR_UNSUPPORTED : DFLARE_OK;
}
Runs flat(const void* p, long n, int size) { return Runs(p, 0, 0, p ? 1 : 0, 1, (int)n, size); }

// f(VE, L, S): the widest accesses that the sizes divide into, up to 4 elements (with 8 in bf16 a lane of the backward pass needs 132
// registers instead of 96, and three waves to a SIMD take 61 us where five take 52)
template <typename T, typename F>
void shaped(bool half_layout, int hd, int rot, F&& f) {
  constexpr int V = 4;
  auto fits = [&](int ve) { return hd % ve == 0 && rot % ve == 0 && (!half_layout || rot / 2 % ve == 0); };
  auto items = [&](int ve) { return rot / 2 / (half_layout || ve == 1 ? ve : ve / 2) + (hd - rot) / ve; };
  if (fits(V)) {
    const int n = items(V);
    if (n <= 4) f(int_c<V>{}, int_c<4>{}, int_c<1>{});
    else if (n <= 8) f(int_c<V>{}, int_c<8>{}, int_c<1>{});
    else if (n <= 16) f(int_c<V>{}, int_c<16>{}, int_c<1>{});
    else if (n <= 32) f(int_c<V>{}, int_c<32>{}, int_c<1>{});
    else if (n <= 64) f(int_c<V>{}, int_c<64>{}, int_c<1>{});
    else f(int_c<V>{}, int_c<64>{}, int_c<2>{});
  } else if (fits(2)) {
    const int n = items(2);
    if (n <= 32) f(int_c<2>{}, int_c<32>{}, int_c<1>{});
    else if (n <= 64) f(int_c<2>{}, int_c<64>{}, int_c<1>{});
    else f(int_c<2>{}, int_c<64>{}, int_c<4>{});
  } else if (items(1) <= 64) {
    f(int_c<1>{}, int_c<64>{}, int_c<1>{});
  } else {
    f(int_c<1>{}, int_c<64>{}, int_c<8>{});
  }
}
// rows that a work-group of tensor k has a part of, at most
long over_groups(const Args& a, int k) {
  const Side& t = a.t[k];
  if (!t.groups) return 0;
  const long n = ((long)a.rows * t.heads + t.groups - 1) / t.groups;  // heads
  return (n + t.heads - 2) / t.heads + 1;
}
// both passes: the tensors' heads over their work-groups, as many to each as it has heads of theirs, and the launch
template <bool BACK>
void launch(Args& a, int n_tensors, int dtype, int layout, hipStream_t st) {
  const int half = a.rot / 2, most = BACK ? kBwdGroups : kFwdGroups;
  a.table_rows = std::max(1, kTable / half);
  by_type(dtype, [&](auto z) {
    using T = decltype(z);
    shaped<T>(layout == DFLARE_ROPE_HALF, a.hd, a.rot, [&](auto ve_c, auto l, auto s) {
      constexpr int VE = decltype(ve_c)::value, L = decltype(l)::value, S = decltype(s)::value;
      const long all = (long)a.rows * (a.t[0].heads + (n_tensors == 2 ? a.t[1].heads : 0));
      for (int k = 0; k < n_tensors; ++k) {
        const long n = (long)a.rows * a.t[k].heads, turns = (n + kT / L - 1) / (kT / L);
        // forward: whole turns, up to six where that leaves 1,024 work-groups, so that some do not take one and others two, and the
        // angles of a work-group's rows are formed for more than a few heads (2,048 rows x 40 heads x 128 14.1 -> 11.6 us, 1,024 rows 9.3
        // -> 7.9; up to 4 or 8 turns 0 to +6%; backward no change)
        if (!BACK) {
          const long total = (all + kT / L - 1) / (kT / L), each = std::max(std::clamp(total / 1024, 1l, 6l), (total + most - 1) / most);
          a.t[k].groups = (int)((turns + each - 1) / each);
          continue;
        }
        a.t[k].groups = (int)std::min(turns, n ? std::max(1l, most * n / all) : 0l);
      }
      const int groups = a.t[0].groups + (n_tensors == 2 ? a.t[1].groups : 0);
      if (!groups) return;
      // (no work-group has more rows than these)
      const long rows = std::max(over_groups(a, 0), n_tensors == 2 ? over_groups(a, 1) : 0l);
      a.table_rows = (int)std::min<long>(a.table_rows, rows);
      const size_t lds = std::max((size_t)a.table_rows * half * 8, BACK ? (size_t)a.hd * 16 : 0);
      auto go = [&](auto half_c, auto bare) {
        hipLaunchKernelGGL((k_qk<T, VE, decltype(half_c)::value, L, S, BACK, decltype(bare)::value>), dim3(groups), dim3(kT), lds, st, a);
      };
      const bool bare = a.eps < 0x1p-90f;
      if (layout == DFLARE_ROPE_HALF) bare ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
      else bare ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
    });
  });
}

}  // namespace

}  // namespace dflare

using namespace dflare;

extern "C" {

int dflare_qk_norm_rope_fwd(const dflare_qk_tensor* tensors, int32_t n_tensors, const int32_t* positions, const double* inv_freq, int32_t rows,
                            int32_t B, int32_t head_dim, int32_t rotary_dim, int32_t dtype, int32_t layout, float scale, float eps, void* stream) {
  if (!tensors) return DFLARE_ERR_INVALID_ARG;
  int rc = check(n_tensors, positions, inv_freq, rows, B, head_dim, rotary_dim, dtype, layout, scale, eps);
  if (rc != DFLARE_OK) return rc;
  const int size = size_of(dtype);
  Args a{};
  long work = 0;
  for (int k = 0; k < n_tensors; ++k) {
    const dflare_qk_tensor& t = tensors[k];
    if ((rc = check_heads(t.n_heads, head_dim)) != DFLARE_OK) return rc;
    if (rows > 0 && t.n_heads > 0 && (!t.x || !t.y)) return DFLARE_ERR_INVALID_ARG;
    if (misplaced(t.x, size) || misplaced(t.y, size) || misplaced(t.gain, size)) return DFLARE_ERR_INVALID_ARG;
    if (t.x == t.y && (t.x_row != t.y_row || t.x_head != t.y_head)) return DFLARE_ERR_INVALID_ARG;
    a.t[k] = Side{t.x, nullptr, t.gain, t.y, nullptr, t.x_row, t.x_head, 0, 0, t.y_row, t.y_head, t.n_heads, 0};
    work += t.n_heads;
  }
  if (rows == 0 || work == 0) return DFLARE_OK;
  // what is written meets nothing else that is written or read, a tensor turned in place aside
  const long n_positions = (rows + B - 1l) / B;
  auto x = [&](int k) { return Runs(tensors[k].x, tensors[k].x_row, tensors[k].x_head, rows, tensors[k].n_heads, head_dim, size); };
  auto y = [&](int k) { return Runs(tensors[k].y, tensors[k].y_row, tensors[k].y_head, rows, tensors[k].n_heads, head_dim, size); };
  for (int k = 0; k < n_tensors; ++k) {
    const Runs w = y(k);
    if (w.empty()) continue;
    if (!w.distinct() || !runs_apart(w, flat(positions, n_positions, 4)) || !runs_apart(w, flat(inv_freq, rotary_dim / 2, 8))) return DFLARE_ERR_INVALID_ARG;
    for (int j = 0; j < n_tensors; ++j) {
      if (!runs_apart(w, flat(tensors[j].gain, head_dim, size))) return DFLARE_ERR_INVALID_ARG;
      if (j != k && !runs_apart(w, y(j))) return DFLARE_ERR_INVALID_ARG;
      if (!(j == k && tensors[k].x == tensors[k].y) && !runs_apart(w, x(j))) return DFLARE_ERR_INVALID_ARG;
    }
  }
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  a.positions = positions;
  a.freq = inv_freq;
  a.rows = rows;
  a.B = B;
  a.hd = head_dim;
  a.rot = rotary_dim;
  a.scale = scale;
  a.inv = 1.f / (float)head_dim;
  a.eps = eps;
  launch<false>(a, n_tensors, dtype, layout, (hipStream_t)stream);
  return launched();
}

size_t dflare_qk_norm_rope_bwd_workspace(int32_t rows, int32_t head_dim, int32_t n_tensors) {
  if (rows < 0 || head_dim < 2 || head_dim > kMostHead || n_tensors < 1 || n_tensors > 2) return 0;
  return rows ? (size_t)(kBwdGroups + 1) * head_dim * 4 : 16;
}

int dflare_qk_norm_rope_bwd(const dflare_qk_grad* tensors, int32_t n_tensors, const int32_t* positions, const double* inv_freq, int32_t rows,
                            int32_t B, int32_t head_dim, int32_t rotary_dim, int32_t dtype, int32_t layout, float scale, float eps,
                            void* workspace, size_t workspace_bytes, void* stream) {
  if (!tensors || !workspace || misplaced(workspace, 16)) return DFLARE_ERR_INVALID_ARG;
  int rc = check(n_tensors, positions, inv_freq, rows, B, head_dim, rotary_dim, dtype, layout, scale, eps);
  if (rc != DFLARE_OK) return rc;
  const size_t ws = dflare_qk_norm_rope_bwd_workspace(rows, head_dim, n_tensors);
  if (workspace_bytes < ws) return DFLARE_ERR_INVALID_ARG;
  const int size = size_of(dtype);
  Args a{};
  for (int k = 0; k < n_tensors; ++k) {
    const dflare_qk_grad& t = tensors[k];
    if ((rc = check_heads(t.n_heads, head_dim)) != DFLARE_OK) return rc;
    if (rows > 0 && t.n_heads > 0 && (!t.x || !t.dy || !t.dx)) return DFLARE_ERR_INVALID_ARG;
    if (misplaced(t.x, size) || misplaced(t.dy, size) || misplaced(t.dx, size) || misplaced(t.gain, size) || misplaced(t.dgain, 4))
      return DFLARE_ERR_INVALID_ARG;
    if (t.x == t.dx && (t.x_row != t.dx_row || t.x_head != t.dx_head)) return DFLARE_ERR_INVALID_ARG;
    if (t.dy == t.dx && (t.dy_row != t.dx_row || t.dy_head != t.dx_head)) return DFLARE_ERR_INVALID_ARG;
    a.t[k] = Side{t.x, t.dy, t.gain, t.dx, t.dgain, t.x_row, t.x_head, t.dy_row, t.dy_head, t.dx_row, t.dx_head, t.n_heads, 0};
  }
  const long n_positions = (rows + B - 1l) / B;
  auto x = [&](int k) { return Runs(tensors[k].x, tensors[k].x_row, tensors[k].x_head, rows, tensors[k].n_heads, head_dim, size); };
  auto dy = [&](int k) { return Runs(tensors[k].dy, tensors[k].dy_row, tensors[k].dy_head, rows, tensors[k].n_heads, head_dim, size); };
  auto dx = [&](int k) { return Runs(tensors[k].dx, tensors[k].dx_row, tensors[k].dx_head, rows, tensors[k].n_heads, head_dim, size); };
  // what is written: dx of each tensor (which may be its x or dy), the gains' gradients, the workspace
  auto meets = [&](const Runs& w, int own) {  // own: the tensor whose dx this is, or -1
    if (!runs_apart(w, flat(positions, n_positions, 4)) || !runs_apart(w, flat(inv_freq, rotary_dim / 2, 8))) return true;
    for (int j = 0; j < n_tensors; ++j) {
      const dflare_qk_grad& t = tensors[j];
      if (!runs_apart(w, flat(t.gain, head_dim, size))) return true;
      if (j != own && !runs_apart(w, dx(j))) return true;
      if (!(j == own && t.x == t.dx) && !runs_apart(w, x(j))) return true;
      if (!(j == own && t.dy == t.dx) && !runs_apart(w, dy(j))) return true;
    }
    return false;
  };
  for (int k = 0; k < n_tensors; ++k) {
    if (!dx(k).empty() && (!dx(k).distinct() || meets(dx(k), k))) return DFLARE_ERR_INVALID_ARG;
    const Runs g = flat(tensors[k].dgain, head_dim, 4);
    if (!g.empty() && (meets(g, -1) || overlap(tensors[k].dgain, (size_t)head_dim * 4, workspace, ws))) return DFLARE_ERR_INVALID_ARG;
  }
  if (n_tensors == 2 && overlap(tensors[0].dgain, (size_t)head_dim * 4, tensors[1].dgain, (size_t)head_dim * 4)) return DFLARE_ERR_INVALID_ARG;
  if (meets(flat(workspace, (long)(ws / 4), 4), -1)) return DFLARE_ERR_INVALID_ARG;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  a.positions = positions;
  a.freq = inv_freq;
  a.rows = rows;
  a.B = B;
  a.hd = head_dim;
  a.rot = rotary_dim;
  a.scale = scale;
  a.inv = 1.f / (float)head_dim;
  a.eps = eps;
  a.part = (float*)workspace;
  if (rows > 0) launch<true>(a, n_tensors, dtype, layout, (hipStream_t)stream);
  hipLaunchKernelGGL(k_qk_cols, dim3((head_dim + 15) / 16 * n_tensors), dim3(1024), 0, (hipStream_t)stream, a.part, a.t[0].groups, a.t[1].groups,
                     head_dim, tensors[0].dgain, n_tensors == 2 ? tensors[1].dgain : nullptr);
  return launched();
}

}  // extern "C"
