// The norm of each query and key head with its rotary position, in one pass over them, forward and backward, and their C-ABI
// entry points.  A head x at position p, with the gain g of its kind and the turn R(p):
//   n = x / sqrt(mean of x^2 + eps),  y = scale R(p) (n g)
//   d = scale R(-p) dy, e = d g,  dx = (e - n mean(e n)) / sqrt(mean of x^2 + eps),  dg = sum of d n over rows and heads
// Bound by memory: a head is read and written once (twice read, x and dy, going back); everything between stays in registers.
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
  int heads;
};
struct Args {
  Side t[2];
  const int32_t* positions;
  const double* freq;
  float* part;  // [work-groups][2][hd] sums of the gains' gradients
  int rows, B, hd, rot, RW, groups, group0, n;  // RW: rows of a group; group0: first group of the launch
  float scale, eps;
};

// An item of a head: the elements of one 16-byte access (half layout: of two, rot / 2 apart), or VE elements past
// the rotated part; E floats, of which a pair's two are PV apart (half) or side by side.
template <typename T, int VE, bool HALF>
struct Item {
  static constexpr int PV = HALF || VE == 1 ? VE : VE / 2, E = HALF ? 2 * VE : VE == 1 ? 2 : VE;
  int m, at;   // first pair, or -1 past the rotated part; first element
  bool any;
  __device__ __forceinline__ Item(int it, int items, int half, int rot) {
    const int turn = half / PV;
    any = it < items;
    m = it < turn ? it * PV : -1;
    at = it < turn ? (HALF ? m : 2 * m) : rot + (it - turn) * VE;
  }
  __device__ __forceinline__ void load(const T* p, int half, float (&x)[E]) const {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.f;
    if (!any) return;
    if (!HALF && m >= 0) {
      load_n<T, E>(p + at, x);
      return;
    }
    float u[VE];
    load_n<T, VE>(p + at, u);
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = u[e];
    if (HALF && m >= 0) {
      load_n<T, VE>(p + at + half, u);
#pragma unroll
      for (int e = 0; e < VE; ++e) x[VE + e] = u[e];
    }
  }
  __device__ __forceinline__ void store(T* p, int half, const float (&x)[E]) const {
    if (!any) return;
    if (!HALF && m >= 0) return store_n<T, E>(p + at, x);
    float u[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) u[e] = x[e];
    store_n<T, VE>(p + at, u);
    if (HALF && m >= 0) {
#pragma unroll
      for (int e = 0; e < VE; ++e) u[e] = x[VE + e];
      store_n<T, VE>(p + at + half, u);
    }
  }
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

// cosines and sines of the rows from row0 on, for all heads (angles formed and reduced in 64 bits: p f in 32 would be off by 0.06
// at position 1,000,000)
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

// A head is held by L lanes, S items each.
template <typename T, int VE, bool HALF, int L, int S>
__global__ __launch_bounds__(kT) void k_qk_fwd(Args a) {
  using I = Item<T, VE, HALF>;
  extern __shared__ float tab[];
  const int half = a.rot / 2, items = half / I::PV + (a.hd - a.rot) / VE, lane = threadIdx.x % L;
  const int row0 = (a.group0 + (int)blockIdx.x) * a.RW, nr = min(a.RW, a.rows - row0);
  float *tc = tab, *ts = tab + a.RW * half;
  angles(a, row0, nr, tc, ts);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const Side& t = a.t[k];
    const int n = nr * t.heads;
    if (n == 0) continue;
    float g[S][I::E];
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
      for (int e = 0; e < I::E; ++e) g[i][e] = 1.f;
      if (t.gain) I(lane + i * L, items, half, a.rot).load((const T*)t.gain, half, g[i]);
    }
    for (int s = threadIdx.x / L; s < n; s += kT / L) {
      const int r = s / t.heads, h = s - r * t.heads;
      const T* x = (const T*)t.x + (row0 + r) * t.x_row + h * t.x_head;
      T* y = (T*)t.y + (row0 + r) * t.y_row + h * t.y_head;
      float v[S][I::E], q = 0.f;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        I(lane + i * L, items, half, a.rot).load(x, half, v[i]);
#pragma unroll
        for (int e = 0; e < I::E; ++e) q = fmaf(v[i][e], v[i][e], q);
      }
      const float rstd = 1.f / sqrtf(head_sum<L>(q) / (float)a.hd + a.eps);
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const I it(lane + i * L, items, half, a.rot);
#pragma unroll
        for (int e = 0; e < I::E; ++e) v[i][e] = v[i][e] * rstd * g[i][e];
        it.turn(tc + r * half, ts + r * half, 1.f, v[i]);
        it.store(y, half, v[i]);
      }
    }
  }
}

template <typename T, int VE, bool HALF, int L, int S>
__global__ __launch_bounds__(kT) void k_qk_bwd(Args a) {
  using I = Item<T, VE, HALF>;
  extern __shared__ float tab[];
  const int half = a.rot / 2, items = half / I::PV + (a.hd - a.rot) / VE, lane = threadIdx.x % L;
  float *tc = tab, *ts = tab + a.RW * half;
  float dg[2][S][I::E];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int e = 0; e < I::E; ++e) dg[k][i][e] = 0.f;
  for (int group = blockIdx.x; group < a.groups; group += gridDim.x) {
    const int row0 = group * a.RW, nr = min(a.RW, a.rows - row0);
    __syncthreads();  // the rows before are done with
    angles(a, row0, nr, tc, ts);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const Side& t = a.t[k];
      const int n = nr * t.heads;
      if (n == 0) continue;
      for (int s = threadIdx.x / L; s < n; s += kT / L) {
        const int r = s / t.heads, h = s - r * t.heads;
        const T* x = (const T*)t.x + (row0 + r) * t.x_row + h * t.x_head;
        const T* dy = (const T*)t.dy + (row0 + r) * t.dy_row + h * t.dy_head;
        T* dx = (T*)t.y + (row0 + r) * t.y_row + h * t.y_head;
        float v[S][I::E], d[S][I::E], q = 0.f, p = 0.f;
#pragma unroll
        for (int i = 0; i < S; ++i) {
          const I it(lane + i * L, items, half, a.rot);
          it.load(x, half, v[i]);
          it.load(dy, half, d[i]);
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
          const I it(lane + i * L, items, half, a.rot);
          float g[I::E];
#pragma unroll
          for (int e = 0; e < I::E; ++e) g[e] = 1.f;
          if (t.gain) it.load((const T*)t.gain, half, g);
          it.turn(tc + r * half, ts + r * half, -1.f, d[i]);
#pragma unroll
          for (int e = 0; e < I::E; ++e) {
            q = fmaf(v[i][e], v[i][e], q);
            p = fmaf(d[i][e] * g[e], v[i][e], p);
          }
        }
        const float rstd = 1.f / sqrtf(head_sum<L>(q) / (float)a.hd + a.eps);
        const float mean = head_sum<L>(p) * rstd / (float)a.hd;
#pragma unroll
        for (int i = 0; i < S; ++i) {
          const I it(lane + i * L, items, half, a.rot);
          float g[I::E];
#pragma unroll
          for (int e = 0; e < I::E; ++e) g[e] = 1.f;
          if (t.gain) it.load((const T*)t.gain, half, g);
#pragma unroll
          for (int e = 0; e < I::E; ++e) {
            const float nv = v[i][e] * rstd;
            dg[k][i][e] = fmaf(d[i][e], nv, dg[k][i][e]);
            v[i][e] = rstd * (d[i][e] * g[e] - nv * mean);
          }
          it.store(dx, half, v[i]);
        }
      }
    }
  }
  // each wave's sums over its heads
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int e = 0; e < I::E; ++e)
#pragma unroll
        for (int off = L; off < 64; off <<= 1) dg[k][i][e] += __shfl_xor(dg[k][i][e], off);
  if ((threadIdx.x & 63) < L) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k >= a.n) break;
      float* to = a.part + (((long)blockIdx.x * 4 + (threadIdx.x >> 6)) * a.n + k) * a.hd;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const I it(lane + i * L, items, half, a.rot);
        if (!it.any) continue;
#pragma unroll
        for (int e = 0; e < I::E; ++e) {
          if (it.m < 0) {
            if (e < VE) to[it.at + e] = dg[k][i][e];
          } else {
            to[HALF && e >= VE ? it.at + half + e - VE : it.at + e] = dg[k][i][e];
          }
        }
      }
    }
  }
}

// the gains' gradients from the waves' sums (16 groups of these, then the groups' in order)
__global__ __launch_bounds__(kT) void k_qk_cols(const float* part, int parts, int n, int hd, float* dgain0, float* dgain1) {
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
    float* to = c < hd ? dgain0 : dgain1;
    if (to) to[c < hd ? c : c - hd] = v;
  }
}

// ---- host side ----
constexpr int kMostHead = 512;   // elements of a head: 64 lanes of at most 8 items
constexpr int kBwdGroups = 512;  // work-groups of the backward pass

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

// f(VE, L, S): items of one access where alignment and sizes allow it
template <typename T, typename F>
void shaped(bool wide, bool half_layout, int hd, int rot, F&& f) {
  constexpr int V = kVec<T>;
  auto lanes = [&](auto ve) {
    constexpr int VE = decltype(ve)::value;
    const int pv = half_layout || VE == 1 ? VE : VE / 2, items = rot / 2 / pv + (hd - rot) / VE;
    if (items <= 4) f(ve, int_c<4>{}, int_c<1>{});
    else if (items <= 8) f(ve, int_c<8>{}, int_c<1>{});
    else if (items <= 16) f(ve, int_c<16>{}, int_c<1>{});
    else if (items <= 64) f(ve, int_c<64>{}, int_c<1>{});
    else if (VE == 1) f(ve, int_c<64>{}, int_c<8>{});
    else f(ve, int_c<64>{}, int_c<2>{});
  };
  if (wide) lanes(int_c<V>{});
  else lanes(int_c<1>{});
}
bool whole_accesses(int hd, int rot, int layout, int ve) {
  return hd % ve == 0 && rot % ve == 0 && (layout != DFLARE_ROPE_HALF || rot / 2 % ve == 0);
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
  const int size = size_of(dtype), ve = 16 / size;
  Args a{};
  bool wide = whole_accesses(head_dim, rotary_dim, layout, ve);
  long work = 0;
  for (int k = 0; k < n_tensors; ++k) {
    const dflare_qk_tensor& t = tensors[k];
    if ((rc = check_heads(t.n_heads, head_dim)) != DFLARE_OK) return rc;
    if (rows > 0 && t.n_heads > 0 && (!t.x || !t.y)) return DFLARE_ERR_INVALID_ARG;
    if (misplaced(t.x, size) || misplaced(t.y, size) || misplaced(t.gain, size)) return DFLARE_ERR_INVALID_ARG;
    if (t.x == t.y && (t.x_row != t.y_row || t.x_head != t.y_head)) return DFLARE_ERR_INVALID_ARG;
    a.t[k] = Side{t.x, nullptr, t.gain, t.y, nullptr, t.x_row, t.x_head, 0, 0, t.y_row, t.y_head, t.n_heads};
    wide = wide && aligned16(t.x) && aligned16(t.y) && aligned16(t.gain) && ((t.x_row | t.x_head | t.y_row | t.y_head) & (ve - 1)) == 0;
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
  const int half = rotary_dim / 2;
  a.positions = positions;
  a.freq = inv_freq;
  a.rows = rows;
  a.B = B;
  a.hd = head_dim;
  a.rot = rotary_dim;
  a.scale = scale;
  a.eps = eps;
  a.n = n_tensors;
  a.RW = std::max(1, std::min(kT / half, rows / 1024));
  a.groups = (int)((rows + a.RW - 1l) / a.RW);
  const size_t lds = (size_t)a.RW * half * 8;
  by_type(dtype, [&](auto z) {
    using T = decltype(z);
    shaped<T>(wide, layout == DFLARE_ROPE_HALF, head_dim, rotary_dim, [&](auto ve_c, auto l, auto s) {
      constexpr int VE = decltype(ve_c)::value, L = decltype(l)::value, S = decltype(s)::value;
      for (long g = 0; g < a.groups; g += kGroupsOfLaunch) {
        const dim3 grid((unsigned)std::min<long>(a.groups - g, kGroupsOfLaunch));
        a.group0 = (int)g;
        if (layout == DFLARE_ROPE_HALF) hipLaunchKernelGGL((k_qk_fwd<T, VE, true, L, S>), grid, dim3(kT), lds, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((k_qk_fwd<T, VE, false, L, S>), grid, dim3(kT), lds, (hipStream_t)stream, a);
      }
    });
  });
  return launched();
}

size_t dflare_qk_norm_rope_bwd_workspace(int32_t rows, int32_t head_dim, int32_t n_tensors) {
  if (rows < 0 || head_dim < 2 || head_dim > kMostHead || n_tensors < 1 || n_tensors > 2) return 0;
  return std::max<size_t>(16, (size_t)std::min(rows, kBwdGroups) * 4 * n_tensors * head_dim * 4);
}

int dflare_qk_norm_rope_bwd(const dflare_qk_grad* tensors, int32_t n_tensors, const int32_t* positions, const double* inv_freq, int32_t rows,
                            int32_t B, int32_t head_dim, int32_t rotary_dim, int32_t dtype, int32_t layout, float scale, float eps,
                            void* workspace, size_t workspace_bytes, void* stream) {
  if (!tensors || !workspace || misplaced(workspace, 16)) return DFLARE_ERR_INVALID_ARG;
  int rc = check(n_tensors, positions, inv_freq, rows, B, head_dim, rotary_dim, dtype, layout, scale, eps);
  if (rc != DFLARE_OK) return rc;
  const size_t ws = dflare_qk_norm_rope_bwd_workspace(rows, head_dim, n_tensors);
  if (workspace_bytes < ws) return DFLARE_ERR_INVALID_ARG;
  const int size = size_of(dtype), ve = 16 / size;
  Args a{};
  bool wide = whole_accesses(head_dim, rotary_dim, layout, ve);
  for (int k = 0; k < n_tensors; ++k) {
    const dflare_qk_grad& t = tensors[k];
    if ((rc = check_heads(t.n_heads, head_dim)) != DFLARE_OK) return rc;
    if (rows > 0 && t.n_heads > 0 && (!t.x || !t.dy || !t.dx)) return DFLARE_ERR_INVALID_ARG;
    if (misplaced(t.x, size) || misplaced(t.dy, size) || misplaced(t.dx, size) || misplaced(t.gain, size) || misplaced(t.dgain, 4))
      return DFLARE_ERR_INVALID_ARG;
    if (t.x == t.dx && (t.x_row != t.dx_row || t.x_head != t.dx_head)) return DFLARE_ERR_INVALID_ARG;
    if (t.dy == t.dx && (t.dy_row != t.dx_row || t.dy_head != t.dx_head)) return DFLARE_ERR_INVALID_ARG;
    a.t[k] = Side{t.x, t.dy, t.gain, t.dx, t.dgain, t.x_row, t.x_head, t.dy_row, t.dy_head, t.dx_row, t.dx_head, t.n_heads};
    wide = wide && aligned16(t.x) && aligned16(t.dy) && aligned16(t.dx) && aligned16(t.gain) &&
           ((t.x_row | t.x_head | t.dy_row | t.dy_head | t.dx_row | t.dx_head) & (ve - 1)) == 0;
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
  const int half = rotary_dim / 2;
  a.positions = positions;
  a.freq = inv_freq;
  a.rows = rows;
  a.B = B;
  a.hd = head_dim;
  a.rot = rotary_dim;
  a.scale = scale;
  a.eps = eps;
  a.part = (float*)workspace;
  a.n = n_tensors;
  a.RW = std::max(1, std::min(kT / half, rows / 1024));
  a.groups = (int)((rows + a.RW - 1l) / a.RW);
  const int grid = std::min(a.groups, kBwdGroups);
  const size_t lds = (size_t)a.RW * half * 8;
  if (rows > 0)
    by_type(dtype, [&](auto z) {
      using T = decltype(z);
      shaped<T>(wide, layout == DFLARE_ROPE_HALF, head_dim, rotary_dim, [&](auto ve_c, auto l, auto s) {
        constexpr int VE = decltype(ve_c)::value, L = decltype(l)::value, S = decltype(s)::value;
        if (layout == DFLARE_ROPE_HALF) hipLaunchKernelGGL((k_qk_bwd<T, VE, true, L, S>), dim3(grid), dim3(kT), lds, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((k_qk_bwd<T, VE, false, L, S>), dim3(grid), dim3(kT), lds, (hipStream_t)stream, a);
      });
    });
  const int n = n_tensors * head_dim;
  hipLaunchKernelGGL(k_qk_cols, dim3((n + 15) / 16), dim3(kT), 0, (hipStream_t)stream, a.part, grid * 4, n, head_dim, tensors[0].dgain,
                     n_tensors == 2 ? tensors[1].dgain : nullptr);
  return launched();
}

}  // extern "C"
