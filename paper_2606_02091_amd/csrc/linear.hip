// Projections and the gated feed-forward block of a draft layer's training step, forward and backward, and their
// C-ABI entry points.  Over rows of x, with weights W [N, K] as nn.Linear keeps them:
//   projection   z = x W^T + b, y = act(z) + residual;  dz = dy act'(z), dx = dz W, dW = dz^T x, db = sum dz
//   gated block  g = x Wg^T, u = x Wu^T, h = act(g) u;  dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu,
//                dWg = dg^T x, dWu = du^T x
// Both are the same three products (of one matrix or of two); the gated block's forward product takes its tiles' rows of W
// from both matrices in turn, so that a lane holds g and u of the same element and h is formed in registers.
// Bound by the matrix cores (and there by the card's power: 66 to 73% busy at 1.4 to 1.8 GHz), up to some 100 rows by reading W.
// 8,192 rows x 4,096 x 12,288 gated: forward with g and u 1.35 to 1.43 ms (1,150 to 1,220 TFLOP/s), gradients 0.19 + 2.6 ms (1,250); 16 rows
// forward 37 us (5.4 TB/s).
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "dflare.h"
#include "product.h"

namespace dflare {

namespace {

// ---- activations: value and derivative in fp32.  Arguments are clamped where both have reached their limits (0, z, 1), so that
// infinities give these and no 0 x infinity; NaN stays. ----
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float rcp_(float x) { return __builtin_amdgcn_rcpf(x); }
constexpr float kLog2E = 1.4426950408889634f;
__device__ __forceinline__ float from_below(float z, float least) { return z < least ? least : z; }
__device__ __forceinline__ float within(float z, float most) { return z < -most ? -most : z > most ? most : z; }

// Phi(z), and exp(-z^2 / 2).  Phi(-a) = exp(-a^2 / 2) t P(t), t = 1 / (1 + 0.31 a), for a >= 0: P is a least-maximum fit of degree 7
// to t^-1 erfcx(a / sqrt 2) / 2 on [0, 20], off by 4e-7 of it in fp32 (and by less than 1e-6 past it)
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float a = fabsf(z), t = rcp_(fmaf(0.31f, a, 1.f));
  float p = 0.03591751679778099f;
  p = fmaf(p, t, -0.14193730056285858f);
  p = fmaf(p, t, 0.15567456185817719f);
  p = fmaf(p, t, -0.0154969971626997f);
  p = fmaf(p, t, 0.11044538021087646f);
  p = fmaf(p, t, 0.10766226798295975f);
  p = fmaf(p, t, 0.12407905608415604f);
  p = fmaf(p, t, 0.12365560233592987f);
  e = exp2_(-0.5f * kLog2E * a * a);
  const float q = e * t * p;
  return z < 0.f ? q : 1.f - q;
}

template <int ACT>
struct Activation {
  static __device__ __forceinline__ float value(float z) {
    float d;
    if constexpr (ACT == DFLARE_ACT_RELU) return z <= 0.f ? 0.f : z;
    if constexpr (ACT == DFLARE_ACT_SILU) {
      z = from_below(z, -128.f);
      return z * rcp_(1.f + exp2_(-kLog2E * z));
    }
    if constexpr (ACT == DFLARE_ACT_GELU) {
      z = from_below(z, -64.f);
      return z * normal_cdf(z, d);
    }
    if constexpr (ACT == DFLARE_ACT_GELU_TANH) {
      z = from_below(z, -64.f);
      return z * rcp_(1.f + exp2_(-kLog2E * inner(z)));
    }
    return z;
  }
  // 2 sqrt(2 / pi) (z + 0.044715 z^3): 0.5 z (1 + tanh of half of it) = z / (1 + exp(-it))
  static __device__ __forceinline__ float inner(float z) { return 1.5957691216057308f * z * fmaf(0.044715f * z, z, 1.f); }
  // the value, and its derivative in d
  static __device__ __forceinline__ float both(float z, float& d) {
    if constexpr (ACT == DFLARE_ACT_RELU) {
      d = z <= 0.f ? 0.f : z > 0.f ? 1.f : z;
      return value(z);
    }
    if constexpr (ACT == DFLARE_ACT_SILU) {
      const float c = within(z, 128.f), s = rcp_(1.f + exp2_(-kLog2E * c));
      d = fmaf(c * s, 1.f - s, s);
      return from_below(z, -128.f) * s;
    }
    if constexpr (ACT == DFLARE_ACT_GELU) {
      float e;
      const float c = within(z, 64.f), p = normal_cdf(c, e);
      d = fmaf(0.3989422804014327f * c, e, p);
      return from_below(z, -64.f) * p;
    }
    if constexpr (ACT == DFLARE_ACT_GELU_TANH) {
      const float c = within(z, 64.f), s = rcp_(1.f + exp2_(-kLog2E * inner(c)));
      d = fmaf(c * s * (1.f - s), 1.5957691216057308f * fmaf(0.134145f * c, c, 1.f), s);
      return from_below(z, -64.f) * s;
    }
    d = 1.f;
    return z;
  }
};
template <typename F>
__host__ __device__ __forceinline__ void with_act(int act, F&& f) {
  switch (act) {
    case DFLARE_ACT_RELU: return f(int_c<DFLARE_ACT_RELU>{});
    case DFLARE_ACT_SILU: return f(int_c<DFLARE_ACT_SILU>{});
    case DFLARE_ACT_GELU: return f(int_c<DFLARE_ACT_GELU>{});
    case DFLARE_ACT_GELU_TANH: return f(int_c<DFLARE_ACT_GELU_TANH>{});
    default: return f(int_c<DFLARE_ACT_NONE>{});
  }
}

// The products of a call.  n2: matrices (2: the gated block)
struct Call {
  const uint16_t *x, *w[2], *bias, *res;  // [rows, K], [N, K], [N], [rows, N]
  const uint16_t* d[2];                   // [rows, N] gradients of z, or of g and u
  uint16_t *y, *z[2];                     // [rows, N] outputs: y or h; z, or g and u, or null
  uint16_t *dx, *dw[2];                   // [rows, K], [N, K]
  float* part;                            // sums of a product's parts: y's, or dx's
  float* part_w;                          // and dW's
  int rows, N, K, n2, act, parts, parts_w;
  int groups_x, split;                    // work-groups of dx in the launch of both gradients; of the rows before `split`
};

// a part's stages of k: [first, past the last) of `stages`
__device__ __forceinline__ void part_of(int stages, int parts, int ks, int& s0, int& s1) {
  s0 = (int)((long)stages * ks / parts);
  s1 = (int)((long)stages * (ks + 1) / parts);
}

// the stage of k that a work-group begins with: another one on each XCD, whose requests then meet fewer others for the same lines (from k = 0
// on all of them, by turns over 12 products of 2,048 and 8,192 rows: 1.4% faster to 1.9% slower)
__device__ __forceinline__ int first_stage(int kn) { return (int)(blockIdx.x % 8) * (kn / kBK) / 8; }

// 4 values as bf16 into LDS rows of TMO values; piece p of row n at p ^ (n mod the pieces)
template <int TMO>
__device__ __forceinline__ void put4(char* lds, int n, int p, int h, f32x4 v) {
  *reinterpret_cast<uint2*>(lds + n * (TMO * 2) + ((p ^ (n & (TMO / 8 - 1))) << 4) + h * 8) =
      make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
}
// and from there, 16 bytes at a time, to to(row, piece) where that is not null.  The large tile's are streamed: there are many of
// them, and the operands keep their places in L2 (8,192 rows gated with three outputs, the two by turns:
// x 4,096 x 12,288 1,332 -> 1,305 us, x 4,096 x 4,096 447 -> 431).
template <typename S, int TMO, typename F>
__device__ __forceinline__ void take(const char* lds, F&& to) {
  constexpr int P = TMO / 8, RW = S::TN / S::W;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll 4
  for (int it = 0; it < RW * P / 64; ++it) {
    const int n = w * RW + it * (64 / P) + lane / P, p = lane % P;
    if (uint16_t* at = to(n, p)) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(lds + n * (TMO * 2) + ((p ^ (n & (P - 1))) << 4));
      if constexpr (std::is_same_v<S, Large>) __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(at));
      else *reinterpret_cast<u32x4*>(at) = v;
    }
  }
}
__device__ __forceinline__ f32x4 four(const f32x16& v, int q) { return f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]}; }
__device__ __forceinline__ f32x4 bf4(const uint16_t* p) {
  const u32x2 v = *reinterpret_cast<const u32x2*>(p);
  return unpack4(v[0], v[1]);
}

// y = act(sums) + residual of a tile (y may lie on the residual).  The sums go through LDS in fp32, a 32-row tile of every wave at a
// time, so that they wait there for their activation (with all of a wave's 128 in its lanes' registers these spill), and the
// residual is read as wide as y is written.
template <typename S>
__device__ __forceinline__ void finish_tile(char* lds, const Acc<S>& acc, int act, const uint16_t* res, uint16_t* y, int ld, int nv, int mv) {
  constexpr int TMO = S::TM, P = TMO / 8, ROWS = S::TN / S::NT, N = ROWS * P / S::T;  // rows of a turn, a thread's pieces of 8 columns
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int wm = w % S::WM, wn = w / S::WM, p = threadIdx.x % P, m = min(p * 8, mv - 8);
  static_assert(ROWS * TMO * 4 <= 2 * S::kStageBytes && ROWS * P % S::T == 0 && S::T % P == 0);
#pragma unroll
  for (int j = 0; j < S::NT; ++j) {
    auto row_of = [&](int i) { return (int)threadIdx.x / P + i * (S::T / P); };  // of the turn
    auto n_of = [&](int row) { return row / 32 * (S::NT * 32) + j * 32 + row % 32; };
    u32x4 r[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      r[i] = res ? *reinterpret_cast<const u32x4*>(res + (uint32_t)(min(n_of(row_of(i)), nv - 1) * ld + m)) : u32x4{0u, 0u, 0u, 0u};
    const int row = wn * 32 + (lane & 31);
#pragma unroll
    for (int t = 0; t < S::MT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(lds + row * (TMO * 4) + ((((wm * S::MT + t) * 8 + 2 * q + h) ^ (row & 31)) << 4)) = four(acc[t][j], q);
    __syncthreads();
    with_act(act, [&](auto a) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = row_of(i), n = n_of(row);
        const char* from = lds + row * (TMO * 4);
        f32x4 u = *reinterpret_cast<const f32x4*>(from + (((2 * p) ^ (row & 31)) << 4));
        f32x4 v = *reinterpret_cast<const f32x4*>(from + (((2 * p + 1) ^ (row & 31)) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          u[e] = Activation<a.value>::value(u[e]);
          v[e] = Activation<a.value>::value(v[e]);
        }
        if (res) {
          u += unpack4(r[i][0], r[i][1]);
          v += unpack4(r[i][2], r[i][3]);
        }
        if (n < nv && p * 8 < mv)
          *reinterpret_cast<u32x4*>(y + (uint32_t)(n * ld + p * 8)) = u32x4{pack2(u[0], u[1]), pack2(u[2], u[3]), pack2(v[0], v[1]), pack2(v[2], v[3])};
      }
    });
    __syncthreads();
  }
}

// z = x W^T, tile `id` of those over `rows` rows of x from row0 on x TM rows of W, and its epilogue; or a part's sums.  (A gated block's
// call by reference: a copy's two matrices would be chosen from in registers.  The other's by value: by reference the large tile needs 43
// registers more than there are.)
template <typename S, bool GATED>
__device__ __forceinline__ void tile_of_y(const std::conditional_t<GATED, const Call&, Call> a, int id, char* lds, int row0, int rows) {
  constexpr int MT = S::MT, NT = S::NT, HT = GATED ? MT / 2 : MT;  // HT: a wave's 32-row tiles of one matrix
  constexpr int PART = GATED ? HT * 32 : 0, TMO = GATED ? S::TM / 2 : S::TM;
  const int nb = (rows + S::TN - 1) / S::TN, na = (a.N + TMO - 1) / TMO;
  int unit, tb;
  if (!tile_of(id, na * a.parts, nb, unit, tb)) return;
  const int ks = unit / na, m0 = unit % na * TMO, r0 = row0 + tb * S::TN;
  int s0, s1;
  part_of((a.K + kBK - 1) / kBK, a.parts, ks, s0, s1);
  const int k0 = s0 * kBK, kn = min(s1 * kBK, a.K) - k0, nv = min(row0 + rows - r0, S::TN), mv = min(a.N - m0, TMO);
  const long wo = (long)m0 * a.K + k0;
  Operand ow{a.w[0] + wo, a.K, mv, kn}, ox{a.x + (long)r0 * a.K + k0, a.K, nv, kn};
  if constexpr (GATED) ow.other = a.w[1] + wo;
  ow.s0 = ox.s0 = first_stage(kn);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int wm = w % S::WM, n_wave = w / S::WM * (NT * 32) + (lane & 31);
  Acc<S> acc;
  clear<S>(acc);
  product<S, false, false, true, PART>(ow, ox, kn, lds, acc, [&](Acc<S>& z) {  // (the bias is the sums' first term)
    if (GATED || a.parts > 1 || !a.bias) return;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 b = bf4(a.bias + m0 + min((wm * MT + t) * 32 + 8 * q + 4 * h, mv - 4));
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[t][j][4 * q + e] = b[e];
      }
  });
  // f(32-row tile t of one matrix, j, q, row of the tile, first of four columns of the tile)
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) f(t, j, q, n_wave + j * 32, (wm * HT + t) * 32 + 8 * q + 4 * h);
  };
  if (a.parts > 1) {
    const long ld = (GATED ? 2l : 1l) * a.N;
    float* out = a.part + ((long)ks * a.rows + r0) * ld + m0;
    each([&](int t, int j, int q, int n, int m) {
      if (n >= nv || m >= mv) return;
      *reinterpret_cast<f32x4*>(out + n * ld + m) = four(acc[t][j], q);
      if constexpr (GATED) *reinterpret_cast<f32x4*>(out + n * ld + a.N + m) = four(acc[HT + t][j], q);
    });
    return;
  }
  const long at0 = (long)r0 * a.N + m0;
  auto out_at = [&](uint16_t* to) {
    return [=](int n, int p) { return n < nv && p * 8 < mv ? to + at0 + (long)n * a.N + p * 8 : nullptr; };
  };
  if constexpr (GATED) {
    if (a.z[0]) {
      each([&](int t, int j, int q, int n, int m) {
        const int p = (wm * MT + t) * 4 + q;  // rows of the tile as they lie in LDS: HT tiles of g, then of u
        put4<S::TM>(lds, n, p, h, four(acc[t][j], q));
        put4<S::TM>(lds, n, p + HT * 4, h, four(acc[HT + t][j], q));
      });
      __syncthreads();
      take<S, S::TM>(lds, [&](int n, int p) -> uint16_t* {
        const int c = p * 8, m = c / (2 * PART) * PART + c % PART;
        return n < nv && m < mv ? a.z[c / PART & 1] + at0 + (long)n * a.N + m : nullptr;
      });
      __syncthreads();
    }
    with_act(a.act, [&](auto act) {
      each([&](int t, int j, int q, int n, int m) {
        f32x4 v = four(acc[t][j], q);
        const f32x4 u = four(acc[HT + t][j], q);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = Activation<act.value>::value(v[e]) * u[e];
        put4<TMO>(lds, n, m / 8, h, v);
      });
    });
  } else {
    if (a.z[0]) {
      each([&](int t, int j, int q, int n, int m) { put4<TMO>(lds, n, m / 8, h, four(acc[t][j], q)); });
      __syncthreads();
      take<S, TMO>(lds, out_at(a.z[0]));
      __syncthreads();
    }
    if (a.res || a.act != DFLARE_ACT_NONE) return finish_tile<S>(lds, acc, a.act, a.res ? a.res + at0 : nullptr, a.y + at0, a.N, nv, mv);
    each([&](int t, int j, int q, int n, int m) { put4<TMO>(lds, n, m / 8, h, four(acc[t][j], q)); });
  }
  __syncthreads();
  take<S, TMO>(lds, out_at(a.y));
}

// ---- forward products on one tile ----
template <typename S, bool GATED>
__global__ __launch_bounds__(S::T, 2) void k_forward(Call a) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * S::kStageBytes];
  tile_of_y<S, GATED>(a, blockIdx.x, lds, 0, a.rows);
}
// on small tiles, and on halves of them from row `split` on: where there are more small tiles than CUs but not twice as many, some CUs
// would take two and others one
template <bool GATED>
__global__ __launch_bounds__(Small::T, 2) void k_forward_halves(Call a) {
  static_assert(Small::T == Few::T && Small::TM == Few::TM && Small::kStageBytes >= Few::kStageBytes);
  __shared__ __attribute__((aligned(1024))) char lds[2 * Small::kStageBytes];
  if ((int)blockIdx.x < a.groups_x) tile_of_y<Small, GATED>(a, blockIdx.x, lds, 0, a.split);
  else tile_of_y<Few, GATED>(a, blockIdx.x - a.groups_x, lds, a.split, a.rows - a.split);
}

// ---- the same for up to 32 rows, bound by the way of W from memory (16 rows x 4,096 x 12,288 gated: 37 us, on tiles of 128 x 64 with parts
// of k and their sums 41; 4,096 x 4,096: 9.0 and 13.4; for more than 32 rows LDS does
// not hold two stages of such rings, but of one matrix for up to 48).  A work-group per CU walks tiles of 16 T rows of each matrix.
// Its eight waves take a part of k each, all of it through rings of NS stages of 64 k in LDS that are a wave's own, so that none
// waits for another while a tile lasts and the stages of the next tile are on their way at the end of one.  There the waves' sums
// meet in LDS, in order. ----
template <bool GATED, int RT, int T>
struct FewRows {
  static constexpr int W = 8, TW = GATED ? 2 * T : T;       // waves, tiles of W
  static constexpr int kStage = (TW + RT) * 2048;           // bytes of a wave's stage: 16 rows of 128 bytes a tile
  static constexpr int kSums = W * TW * RT * 1024;
  static constexpr int NS = (kLdsBytes - kSums) / (W * kStage) > 4 ? 4 : (kLdsBytes - kSums) / (W * kStage);
  static constexpr int kLds = W * NS * kStage + kSums;
  static_assert(NS >= 2);
};
template <bool GATED, int RT, int T>
__global__ __launch_bounds__(512, 2) void k_few(Call a) {
  using F = FewRows<GATED, RT, T>;
  constexpr int W = F::W, TW = F::TW, NS = F::NS, L = (TW + RT) * 2;  // L: loads of a stage
  __shared__ __attribute__((aligned(1024))) char lds[F::kLds];
  char* sums = lds + W * NS * F::kStage;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* ring = lds + w * NS * F::kStage;
  const uint32_t ring0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LDSP char*)ring);
  const int groups = (a.N + 16 * T - 1) / (16 * T), stages = (a.K + kBK - 1) / kBK, tail = a.K % kBK;
  int s0, s1;
  part_of(stages, W, w, s0, s1);
  // a lane's pieces: rows lane / 8 and 8 more of a tile, piece c of them at c ^ (row / 2 mod 8); where a stage ends
  // within the row, the pieces past it are its first again
  uint32_t piece[2], cut[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = i * 8 + (lane >> 3), c = (lane & 7) ^ ((row >> 1) & 7);
    piece[i] = c * 16;
    cut[i] = tail && c * 8 >= tail ? c * 16 : 0;
  }
  uint32_t xo[RT][2], wo[T][2];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < 2; ++i) xo[r][i] = (uint32_t)(min(r * 16 + i * 8 + (lane >> 3), a.rows - 1) * a.K * 2) + piece[i];
  int ig = blockIdx.x, is = s0;  // tile group and stage to load
  auto at_group = [&] {
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        wo[t][i] = (uint32_t)(min(t * 16 + i * 8 + (lane >> 3), a.N - 1 - ig * 16 * T) * a.K * 2) + piece[i];
  };
  at_group();
  int ahead = 0;  // stages on their way or in the ring
  auto issue = [&](uint32_t slot) {
    if (ig >= groups || s0 == s1) return;
    const bool last = tail && is == stages - 1;
    const uint32_t dst = ring0 + slot * F::kStage;
#pragma unroll
    for (int t = 0; t < TW; ++t) {
      const char* p = reinterpret_cast<const char*>(a.w[t / T] + (long)ig * 16 * T * a.K) + (long)is * 128;
#pragma unroll
      for (int i = 0; i < 2; ++i) load_lds(p, wo[t % T][i] - (last ? cut[i] : 0), dst + (2 * t + i) * 1024);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        load_lds(reinterpret_cast<const char*>(a.x) + (long)is * 128, xo[r][i] - (last ? cut[i] : 0), dst + (2 * (TW + r) + i) * 1024);
    ++ahead;
    if (++is == s1) {
      is = s0;
      ig += gridDim.x;
      at_group();
    }
  };
#pragma unroll
  for (int k = 0; k < NS; ++k) issue(k);
  uint32_t slot = 0;
  for (int grp = blockIdx.x; grp < groups; grp += gridDim.x) {
    const int m0 = grp * 16 * T;
    f32x4 acc[TW][RT];
#pragma unroll
    for (int t = 0; t < TW; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) acc[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = s0; s < s1; ++s) {
      if (ahead == NS) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 1) * L) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const char* from = ring + slot * F::kStage;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const int row = lane & 15, c = ks * 4 + (lane >> 4);
        const uint32_t at = row * 128 + ((c ^ ((row >> 1) & 7)) << 4);
        u32x4 fw[TW], fx[RT];
#pragma unroll
        for (int t = 0; t < TW; ++t) fw[t] = *reinterpret_cast<const u32x4*>(from + t * 2048 + at);
#pragma unroll
        for (int r = 0; r < RT; ++r) fx[r] = *reinterpret_cast<const u32x4*>(from + (TW + r) * 2048 + at);
        if (tail && s == stages - 1 && c * 8 >= tail) {  // past the end of k
#pragma unroll
          for (int t = 0; t < TW; ++t) fw[t] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
          for (int r = 0; r < RT; ++r) fx[r] = u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int t = 0; t < TW; ++t)
#pragma unroll
          for (int r = 0; r < RT; ++r) acc[t][r] = mfma(fw[t], fx[r], acc[t][r]);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage is read: its place takes another
      --ahead;
      issue(slot);
      slot = slot + 1 == NS ? 0 : slot + 1;
    }
    auto meet = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };  // (not for what is on its way)
    meet();  // the sums of the tile before are read
#pragma unroll
    for (int t = 0; t < TW; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) *reinterpret_cast<f32x4*>(sums + (((w * TW + t) * RT + r) * 64 + lane) * 16) = acc[t][r];
    meet();
    const int l = threadIdx.x & 63, r = (threadIdx.x >> 6) % RT, t = (threadIdx.x >> 6) / RT, row = r * 16 + (l & 15);
    const int m = m0 + t * 16 + (l >> 4) * 4;
    if (t < T && row < a.rows && m < a.N) {  // four columns of a row
      auto sum = [&](int tile) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < W; ++k) v += *reinterpret_cast<const f32x4*>(sums + (((k * TW + tile) * RT + r) * 64 + l) * 16);
        return v;
      };
      f32x4 v = sum(t), u = v;
      if constexpr (GATED) u = sum(T + t);
      const long at = (long)row * a.N + m;
      auto put = [&](uint16_t* to, f32x4 x) { *reinterpret_cast<uint2*>(to + at) = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3])); };
      if (!GATED && a.bias) v += bf4(a.bias + m);
      if (a.z[0]) {
        put(a.z[0], v);
        if constexpr (GATED) put(a.z[1], u);
      }
      with_act(a.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = Activation<act.value>::value(v[e]);
      });
      if constexpr (GATED) v = v * u;
      else if (a.res) v += bf4(a.res + at);
      put(a.y, v);
    }
  }
}

// a forward product's parts, added in order, and its epilogue; a thread takes 8 columns of a row
template <bool GATED>
__global__ __launch_bounds__(kT) void k_finish(Call a) {
  const int P = a.N / 8;
  const long i = blockIdx.x * (long)kT + threadIdx.x;
  if (i >= (long)a.rows * P) return;
  const long row = i / P, m = (i - row * P) * 8, at = row * a.N + m, ld = (GATED ? 2l : 1l) * a.N;
  float v[8], u[8];
  auto sum = [&](float(&s)[8], const float* from) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.f;
#pragma unroll 4
    for (int k = 0; k < a.parts; ++k) {
      const f32x4* p = reinterpret_cast<const f32x4*>(from + k * a.rows * ld);
      const f32x4 x = p[0], y = p[1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] += x[e];
        s[4 + e] += y[e];
      }
    }
  };
  const float* from = a.part + row * ld + m;
  auto put = [&](uint16_t* to, const float(&s)[8]) { *reinterpret_cast<u32x4*>(to + at) = pack(s); };
  sum(v, from);
  if constexpr (GATED) {
    sum(u, from + a.N);
    if (a.z[0]) {
      put(a.z[0], v);
      put(a.z[1], u);
    }
  } else {
    if (a.bias) {
      unpack(*reinterpret_cast<const u32x4*>(a.bias + m), u);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    if (a.z[0]) put(a.z[0], v);
  }
  with_act(a.act, [&](auto act) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = Activation<act.value>::value(v[e]);
  });
  if constexpr (GATED) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= u[e];
  } else if (a.res) {
    unpack(*reinterpret_cast<const u32x4*>(a.res + at), u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += u[e];
  }
  put(a.y, v);
}

// the tile's sums, as a part or as they are stored
template <typename S>
__device__ __forceinline__ void put_sums(char* lds, const Acc<S>& acc, float* part, uint16_t* out, long ld, int nv, int mv) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int wm = w % S::WM, n_wave = w / S::WM * (S::NT * 32) + (lane & 31);
#pragma unroll
  for (int j = 0; j < S::NT; ++j)
#pragma unroll
    for (int t = 0; t < S::MT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n_wave + j * 32, m = (wm * S::MT + t) * 32 + 8 * q + 4 * h;
        if (!part) put4<S::TM>(lds, n, m / 8, h, four(acc[t][j], q));
        else if (n < nv && m < mv) *reinterpret_cast<f32x4*>(part + n * ld + m) = four(acc[t][j], q);
      }
  if (part) return;
  __syncthreads();
  take<S, S::TM>(lds, [&](int n, int p) { return n < nv && p * 8 < mv ? out + n * ld + p * 8 : nullptr; });
}

// dx = d W over the rows of W (of both matrices, one after the other)
template <typename S>
__device__ __forceinline__ void tile_of_dx(const Call& a, int id, char* lds) {
  const int nb = (a.rows + S::TN - 1) / S::TN, na = (a.K + S::TM - 1) / S::TM;
  int unit, tb;
  if (!tile_of(id, na * a.parts, nb, unit, tb)) return;
  const int ks = unit / na, m0 = unit % na * S::TM, r0 = tb * S::TN, one = (a.N + kBK - 1) / kBK;
  int s0, s1;
  part_of(a.n2 * one, a.parts, ks, s0, s1);
  const int nv = min(a.rows - r0, S::TN), mv = min(a.K - m0, S::TM);
  Acc<S> acc;
  clear<S>(acc);
#pragma unroll 1
  for (int p = 0; p < a.n2; ++p) {
    const int k0 = max(s0 - p * one, 0) * kBK, kn = min((s1 - p * one) * kBK, a.N) - k0;
    if (kn <= 0) continue;
    Operand ow{a.w[p] + (long)k0 * a.K + m0, a.K, mv, kn}, od{a.d[p] + (long)r0 * a.N + k0, a.N, nv, kn};
    ow.s0 = od.s0 = first_stage(kn);
    product<S, true, false, true>(ow, od, kn, lds, acc, [](Acc<S>&) {});
  }
  const long at = (long)r0 * a.K + m0;
  put_sums<S>(lds, acc, a.parts > 1 ? a.part + (long)ks * a.rows * a.K + at : nullptr, a.dx + at, a.K, nv, mv);
}

// dW = d^T x over the rows, for each matrix
template <typename S>
__device__ __forceinline__ void tile_of_dw(const Call& a, int id, char* lds) {
  const int one = (a.N + S::TN - 1) / S::TN, nb = a.n2 * one, na = (a.K + S::TM - 1) / S::TM;
  int unit, tb;
  if (!tile_of(id, na * a.parts_w, nb, unit, tb)) return;
  const int ks = unit / na, m0 = unit % na * S::TM, p = tb / one, n0 = tb % one * S::TN;
  int s0, s1;
  part_of((a.rows + kBK - 1) / kBK, a.parts_w, ks, s0, s1);
  const int k0 = s0 * kBK, kn = min(s1 * kBK, a.rows) - k0;
  const int nv = min(a.N - n0, S::TN), mv = min(a.K - m0, S::TM);
  Acc<S> acc;
  clear<S>(acc);
  Operand ox{a.x + (long)k0 * a.K + m0, a.K, mv, kn}, od{a.d[p] + (long)k0 * a.N + n0, a.N, nv, kn};
  ox.s0 = od.s0 = first_stage(kn);
  product<S, true, true, true>(ox, od, kn, lds, acc, [](Acc<S>&) {});
  const long at = (long)n0 * a.K + m0;
  put_sums<S>(lds, acc, a.parts_w > 1 ? a.part_w + ((long)ks * a.n2 + p) * a.N * a.K + at : nullptr, a.dw[p] + at, a.K, nv, mv);
}

// ---- both gradients in one launch, dx's tiles first: their sums are the longer ones where rows are few, and the tiles of dW fill
// the CUs that they leave (1,003 rows x 2,880 x 2,880 gated: 79 us, in two launches with parts of dx 104; 8,192 x 4,096 x 12,288 2.64 ms,
// 2.74) ----
template <typename SX, typename SW>
__global__ __launch_bounds__(SX::T, 2) void k_gradients(Call a) {
  static_assert(SX::T == SW::T);
  constexpr int LDS = 2 * (SX::kStageBytes > SW::kStageBytes ? SX::kStageBytes : SW::kStageBytes);
  __shared__ __attribute__((aligned(1024))) char lds[LDS];
  if ((int)blockIdx.x < a.groups_x) tile_of_dx<SX>(a, blockIdx.x, lds);
  else tile_of_dw<SW>(a, blockIdx.x - a.groups_x, lds);
}

// What is left of the gradients' launch: sums of parts, added in order and rounded, of dx (first `values` of `parts`) and of dW (n0
// values of each matrix); and the bias' gradient from the chunks' sums.  The work-groups of each come one after another.
struct Rest {
  const float *part, *part_w, *sums;
  uint16_t *dx, *dw[2], *dbias;
  long values, values_w, n0;
  int parts, parts_w, chunks, N, groups, groups_w;
};
__device__ __forceinline__ u32x4 add_parts(const float* part, int parts, long values, long i) {
  float s[8] = {};
#pragma unroll 4
  for (int k = 0; k < parts; ++k) {
    const f32x4* p = reinterpret_cast<const f32x4*>(part + k * values + i);
    const f32x4 x = p[0], y = p[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[e] += x[e];
      s[4 + e] += y[e];
    }
  }
  return pack(s);
}
__global__ __launch_bounds__(kT) void k_rest(Rest a) {
  int id = blockIdx.x;
  if (id < a.groups) {
    const long i = (id * (long)kT + threadIdx.x) * 8;
    if (i < a.values) *reinterpret_cast<u32x4*>(a.dx + i) = add_parts(a.part, a.parts, a.values, i);
    return;
  }
  if ((id -= a.groups) < a.groups_w) {
    const long i = (id * (long)kT + threadIdx.x) * 8;
    if (i < a.values_w) *reinterpret_cast<u32x4*>(i < a.n0 ? a.dw[0] + i : a.dw[1] + (i - a.n0)) = add_parts(a.part_w, a.parts_w, a.values_w, i);
    return;
  }
  id -= a.groups_w;
  __shared__ float s[16][17];  // 16 groups of chunks, then these in order
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, c = id * 16 + l;
  float v = 0.f;
  if (c < a.N) {
#pragma unroll 8
    for (int k = g; k < a.chunks; k += 16) v += a.sums[(long)k * a.N + c];
  }
  s[g][l] = v;
  __syncthreads();
  if (g == 0 && c < a.N) {
    for (int k = 1; k < 16; ++k) v += s[k][l];
    a.dbias[c] = (uint16_t)pack2(v, 0.f);
  }
}

// ---- gradients of the pre-activations.  A thread takes 8 columns of the rows of a chunk; with a bias it adds them up.  Bound by memory:
// 8,192 x 12,288 gated 195 us, 5.2 TB/s. ----
struct Pre {
  const uint16_t *dy, *z[2];  // [rows, N]; z, or g and u, or null (no activation: d is dy, and only the sums are wanted)
  uint16_t* d[2];
  float* sums;                // [chunks][N], or null
  int rows, N, act, chunks;
};
template <bool GATED>
__global__ __launch_bounds__(kT) void k_pre(Pre a) {
  const int P = a.N / 8, groups = (P + kT - 1) / kT;
  const int c = blockIdx.x / groups, p = (blockIdx.x - c * groups) * kT + threadIdx.x;
  if (p >= P) return;
  const int first = (int)((long)a.rows * c / a.chunks), last = (int)((long)a.rows * (c + 1) / a.chunks);
  float s[8] = {};
  with_act(a.act, [&](auto act) {
#pragma unroll 2
    for (int r = first; r < last; ++r) {
      const long at = (long)r * a.N + p * 8;
      float dy[8], z[8], u[8], d[8];
      unpack(*reinterpret_cast<const u32x4*>(a.dy + at), dy);
      if (GATED || act.value != DFLARE_ACT_NONE) {
        unpack(*reinterpret_cast<const u32x4*>(a.z[0] + at), z);
        if constexpr (GATED) unpack(*reinterpret_cast<const u32x4*>(a.z[1] + at), u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = Activation<act.value>::both(z[e], d[e]);
          if constexpr (GATED) {
            z[e] = dy[e] * v;
            dy[e] *= u[e];
          }
          dy[e] *= d[e];
        }
        *reinterpret_cast<u32x4*>(a.d[0] + at) = pack(dy);
        if constexpr (GATED) *reinterpret_cast<u32x4*>(a.d[1] + at) = pack(z);
      }
      if constexpr (!GATED) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += dy[e];
      }
    }
  });
  if (GATED || !a.sums) return;
  f32x4* to = reinterpret_cast<f32x4*>(a.sums + (long)c * a.N + p * 8);
  to[0] = f32x4{s[0], s[1], s[2], s[3]};
  to[1] = f32x4{s[4], s[5], s[6], s[7]};
}

// ---- host side ----
constexpr int kMostParts = 128;         // of a product
constexpr long kPartValues = 1l << 25;  // and most sums of these together
constexpr int kPreGroups = 2048;        // work-groups of k_pre, about

size_t up(size_t n) { return (n + 255) / 256 * 256; }
constexpr int kPartStages = 4;          // of a part, at least
constexpr int kPartGroups = 2048;       // work-groups of a product in parts, at most
// bytes of the parts of any product of up to `values` sums over up to `stages` of k: grows with all three.  Up to 64 rows the work-groups are
// of tiles of 128 columns, and so there are 2^18 sums of a row at most.
size_t part_bytes(int rows, long values, long stages) {
  const long parts = std::min<long>(kMostParts, stages / kPartStages), sums = std::min(kPartValues, parts * values);
  return parts < 2 ? 0 : up((size_t)(rows <= Few::TN ? std::min(sums, (long)rows * kPartGroups * Few::TM) : sums) * 4);
}
// and of those that a product is cut into
size_t own_bytes(int parts, long values) { return parts < 2 ? 0 : up((size_t)values * parts * 4); }

long over(long a, long b) { return (a + b - 1) / b; }
// A product of `tiles` over `stages` of k, cut into parts of k, and its costs in us, fitted to 34 products and pairs of them under some 25
// plans each (1 to 8,192 rows, K and N from 256 to 12,288; the plan that is least by them takes 2.4% longer than the best one,
// at the mean).  A stage takes 1.40 on the large tile (256 work-groups at once); on the smaller ones 0.50 where a work-group has its
// CU for itself, 0.94 where two share it; a work-group begins and ends in 5 (3); parts are written and read at 6.1 TB/s and
// added by a launch more (1.9).  Up to 64 rows the first product's stages wait for memory, 1.3 each (16 rows x 4,096 x 12,288 gated,
// gradients: 110 us by 0.94, 96 by this).
struct Work {
  long tiles, values;
  int stages;
  bool can(int k) const { return k == 1 || (stages >= kPartStages * k && values * k <= kPartValues); }
  double sums(int k) const { return k > 1 ? (double)values * k * 8 / 6.1e6 + 1.9 : 0.0; }
};
// When all work-groups have ended: nx that take ux each, then nw that take uw, each where a slot is free first
double end_of(long nx, double ux, long nw, double uw, long slots, double pole) {
  if (!nw) return (double)over(nx, slots) * ux;
  if (!nx) return (double)over(nw, slots) * uw;
  const long r = nx / slots, late = nx % slots;  // `late` slots have r + 1 of the first, the others r
  const double t0 = (double)r * ux, t1 = t0 + ux;
  auto done = [&](double t) {
    return (slots - late) * (long)std::max(0.0, (t - t0) / uw + 1e-9) + late * (long)std::max(0.0, (t - t1) / uw + 1e-9);
  };
  double end = 1e300;
  for (const double from : {t0, t1}) {
    double t = from + (double)std::max(0l, (long)(((double)nw + (double)late * (t1 - from) / uw - (double)(slots - late) * (from - t0) / uw) / (double)slots) - 2) * uw;
    while (done(t) < nw) t += uw;
    end = std::min(end, t);
  }
  return std::max(end, pole * (late ? t1 : t0));
}
// The last of a product's turns of work-groups over the CUs, us a stage, of n: the large tile's alone on a CU, the small one's in pairs
// where there are more than CUs
double last_stage(int tile, double n) {
  const double f = n / 256.0;
  return n == 0 ? 0.0 : tile == 0 ? 1.07 + 0.36 * f * f : f <= 1.0 ? 0.58 + 0.09 * f : 0.80 + 0.17 * (f - 1.0);
}
double cost_of(int tile, bool few, const Work& x, int kx, const Work& w, int kw) {
  const long slots = tile == 0 ? 256 : 512, nx = x.tiles * kx, nw = w.tiles * kw;
  if (!nw && !few) {
    const double s = (double)over(x.stages, kx);
    return (double)(nx / slots) * (tile == 0 ? 1.40 * s + 2.0 : 0.97 * s + 1.0) + last_stage(tile, (double)(nx % slots)) * s + (tile == 0 ? 5.0 : 3.0) + x.sums(kx);
  }
  const double stage = tile == 0 ? 1.40 : 0.50 + 0.44 * (double)std::min(std::max(nx + nw - 256, 0l), 256l) / 256.0, ends = tile == 0 ? 5.0 : 3.0;
  // (the last of dx's work-groups have a small tile's CU for themselves at the end)
  return end_of(nx, (double)over(x.stages, kx) * (few ? 1.3 : stage) + ends, nw, (double)over(w.stages, kw) * stage + ends, slots, tile == 0 ? 1.0 : 0.75) +
         x.sums(kx) + w.sums(kw);
}
// A forward product's rows that go to small tiles, where there are more of these than CUs and at most two to a CU: some CUs would take
// two (0.9 us a stage) and others one (0.6), so the fewest of the rows behind them go to halves of the tile that leave at most one to
// each CU, and two work-groups as before (1,003 gated rows of 2,880 x 2,880 45.6 -> 41.0 us, 777 x 5,120 x 2,880 40.6 -> 33.9).
// All rows: no halves.
int rows_before_halves(long columns, int rows) {
  const long halves = over(rows, Few::TN);
  if (columns * over(rows, Small::TN) > 512) return rows;
  for (long b = 0; b <= halves; ++b) {
    const long big = columns * ((halves - b) / 2);
    if ((halves - b) % 2 || big > 256) continue;
    return b && big + columns * b <= 512 ? (int)(halves - b) * Few::TN : rows;
  }
  return rows;
}

struct Plan {
  int tile, kx, kw;  // 0: the large tile, 1: the small one; parts
};
// f(tile) gives the two products' work on a tile (the second may be empty); few: on the small ones alone.  The parts of one are chosen beside those of the other, in
// turn, from numbers that come near to any.
template <typename F>
Plan plan_of(bool few, F&& f) {
  static constexpr int numbers[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 64, 96, kMostParts};
  Plan best{few, 1, 1};
  double least = 1e300;
  for (int t = few; t < 2; ++t) {
    const std::pair<Work, Work> p = f(t);
    int kx = 1, kw = 1;
    double low = cost_of(t, few, p.first, 1, p.second, 1);
    auto search = [&](const Work& own, int& k) {
      for (int n : numbers) {
        if (!own.can(n) || (n > 1 && own.tiles * n > kPartGroups)) break;
        const int was = k;
        k = n;
        const double c = cost_of(t, few, p.first, kx, p.second, kw);
        if (c < low) low = c;
        else k = was;
      }
    };
    search(p.first, kx);
    if (p.second.tiles) {
      search(p.second, kw);
      search(p.first, kx);
    }
    if (low < least) {
      least = low;
      best = Plan{t, kx, kw};
    }
  }
  return best;
}

int check(int rows, int N, int K, int act) {
  if (rows < 0 || N < 1 || K < 1 || act < DFLARE_ACT_NONE || act > DFLARE_ACT_GELU_TANH) return DFLARE_ERR_INVALID_ARG;
  if (N % 8 || K % 8 || N > (1 << 18) || K > (1 << 18) || rows > (1 << 22)) return DFLARE_ERR_UNSUPPORTED;
  // a launch has less than 2^32 threads: of 256 over tiles of 128 x 64, and over 8 values each
  const long tiles = std::max({(rows + 63l) / 64 * ((std::max(N, K) + 63l) / 64), (N + 63l) / 64 * 2 * ((K + 127l) / 128)});
  return tiles >= (1l << 23) ? DFLARE_ERR_UNSUPPORTED : DFLARE_OK;
}

unsigned whole_turns(long groups) { return (unsigned)((groups + 7) / 8 * 8); }  // of the XCDs
int stages_of(long k) { return (int)((k + kBK - 1) / kBK); }

// What a call's products run on, and their parts.  split: rows before the halves
struct Chosen {
  int tiles, parts, parts_w, split;
};
constexpr int kFewRows = 32;
Chosen forward_plan(int rows, int N, int K, int n2) {
  if (rows <= kFewRows) return {DFLARE_TILES_NONE, 1, 1, rows};
  auto work = [&](auto s) {
    return std::make_pair(Work{over(N, s.TM / n2) * over(rows, s.TN), (long)rows * N * n2, stages_of(K)}, Work{0, 0, 0});
  };
  // up to 64 rows the small tile's other half would be empty
  const bool few = rows <= Few::TN;
  const Plan p = plan_of(few, [&](int t) { return few ? work(Few{}) : t == 0 ? work(Large{}) : work(Small{}); });
  if (few || p.tile == 0) return {few ? DFLARE_TILES_64 : DFLARE_TILES_256, p.kx, 1, rows};
  const int split = p.kx == 1 ? rows_before_halves(over(N, Small::TM / n2), rows) : rows;
  return {split < rows ? DFLARE_TILES_128_64 : DFLARE_TILES_128, p.kx, 1, split};
}
long tiles_of_dx(long rows, long K, int tn, int tm) { return over(K, tm) * over(rows, tn); }
long tiles_of_dw(long N, long K, int n2, int tn, int tm) { return over(K, tm) * over(N, tn) * n2; }
// dx and dW, each where it is wanted
Chosen gradients_plan(int rows, int N, int K, int n2, bool dx, bool dw) {
  const bool few = rows <= Few::TN;
  Chosen c{few ? DFLARE_TILES_64 : DFLARE_TILES_128, 1, 1, rows};
  if (!rows || !(dx || dw)) return c;
  auto work = [&](auto sx, auto sw) {
    return std::make_pair(Work{dx ? tiles_of_dx(rows, K, sx.TN, sx.TM) : 0l, (long)rows * K, n2 * stages_of(N)},
                          Work{dw ? tiles_of_dw(N, K, n2, sw.TN, sw.TM) : 0l, (long)n2 * N * K, stages_of(rows)});
  };
  const Plan p = plan_of(few, [&](int t) { return few ? work(Few{}, Small{}) : t == 0 ? work(Large{}, Large{}) : work(Small{}, Small{}); });
  if (p.tile == 0) c.tiles = DFLARE_TILES_256;
  if (dx) c.parts = p.kx;
  if (dw) c.parts_w = p.kw;
  return c;
}

// the parts' sums of a forward product, as y
template <bool GATED>
void finish(const Call& a, hipStream_t st) {
  if (a.parts == 1) return;
  const long threads = (long)a.rows * (a.N / 8);
  hipLaunchKernelGGL((k_finish<GATED>), dim3((unsigned)((threads + kT - 1) / kT)), dim3(kT), 0, st, a);
}
template <bool GATED>
void forward_few(const Call& a, hipStream_t st) {
  auto go = [&](auto rt, auto t) {
    constexpr int RT = decltype(rt)::value, T = decltype(t)::value;
    hipLaunchKernelGGL((k_few<GATED, RT, T>), dim3(std::min((a.N + 16 * T - 1) / (16 * T), 256)), dim3(512), 0, st, a);
  };
  const bool wide = !GATED && a.N > 16 * 256;
  if (a.rows <= 16) wide ? go(int_c<1>{}, int_c<GATED ? 1 : 2>{}) : go(int_c<1>{}, int_c<1>{});
  else wide ? go(int_c<2>{}, int_c<GATED ? 1 : 2>{}) : go(int_c<2>{}, int_c<1>{});
}
template <bool GATED>
void forward(Call a, const Chosen& c, hipStream_t st) {
  a.parts = c.parts;
  a.split = c.split;
  auto go = [&](auto s) {
    using S = decltype(s);
    const long tiles = over(a.N, S::TM / a.n2) * over(a.rows, S::TN);
    hipLaunchKernelGGL((k_forward<S, GATED>), dim3(whole_turns(tiles * a.parts)), dim3(S::T), 0, st, a);
    finish<GATED>(a, st);
  };
  const long columns = over(a.N, Small::TM / a.n2);
  switch (c.tiles) {
    case DFLARE_TILES_NONE: return forward_few<GATED>(a, st);
    case DFLARE_TILES_64: return go(Few{});
    case DFLARE_TILES_128: return go(Small{});
    case DFLARE_TILES_256: return go(Large{});
  }
  a.groups_x = (int)whole_turns(columns * (a.split / Small::TN));
  hipLaunchKernelGGL((k_forward_halves<GATED>), dim3(a.groups_x + whole_turns(columns * over(a.rows - a.split, Few::TN))), dim3(Small::T), 0, st, a);
}
// dx and dW, and the bias' gradient from `chunks` sums
void gradients(Call a, const Chosen& c, const float* sums, int chunks, uint16_t* dbias, hipStream_t st) {
  const long one = (long)a.N * a.K;
  a.parts = c.parts;
  a.parts_w = c.parts_w;
  if (a.dx || a.dw[0]) {
    auto go = [&](auto sx, auto sw) {
      using SX = decltype(sx);
      using SW = decltype(sw);
      a.groups_x = a.dx ? (int)whole_turns(tiles_of_dx(a.rows, a.K, SX::TN, SX::TM) * a.parts) : 0;
      const long tiles = a.dw[0] ? tiles_of_dw(a.N, a.K, a.n2, SW::TN, SW::TM) : 0;
      hipLaunchKernelGGL((k_gradients<SX, SW>), dim3(a.groups_x + whole_turns(tiles * a.parts_w)), dim3(SX::T), 0, st, a);
    };
    if (c.tiles == DFLARE_TILES_64) go(Few{}, Small{});
    else if (c.tiles == DFLARE_TILES_256) go(Large{}, Large{});
    else go(Small{}, Small{});
  }
  Rest r{};
  r.part = a.part;
  r.part_w = a.part_w;
  r.sums = sums;
  r.dx = a.dx;
  r.dw[0] = a.dw[0];
  r.dw[1] = a.dw[1];
  r.dbias = dbias;
  r.values = (long)a.rows * a.K;
  r.values_w = a.n2 * one;
  r.n0 = one;
  r.parts = a.parts;
  r.parts_w = a.parts_w;
  r.chunks = chunks;
  r.N = a.N;
  r.groups = a.parts > 1 ? (int)over(r.values / 8, kT) : 0;
  r.groups_w = a.parts_w > 1 ? (int)over(r.values_w / 8, kT) : 0;
  const long groups = r.groups + (long)r.groups_w + (dbias ? over(a.N, 16) : 0);
  if (groups) hipLaunchKernelGGL(k_rest, dim3((unsigned)groups), dim3(kT), 0, st, r);
}
// work-groups over 2,048 columns each, and chunks of rows
int pre_chunks(int rows, int N, bool sums) {
  return (int)std::max(1l, std::min<long>(sums ? over(rows, 4) : rows, kPreGroups / over(N / 8, kT)));
}
template <bool GATED>
void pre_gradients(const Pre& a, hipStream_t st) {
  const long groups = (long)(a.N / 8 + kT - 1) / kT * a.chunks;
  hipLaunchKernelGGL((k_pre<GATED>), dim3((unsigned)groups), dim3(kT), 0, st, a);
}

bool off16(std::initializer_list<const void*> ps) {
  for (const void* p : ps)
    if (misplaced(p, 16)) return true;
  return false;
}

// A call's workspace.  d: n_d gradients of [rows, N]; sums of a bias' gradient; the products' parts
struct Layout {
  size_t d, sums, part, part_w, total;
  Layout(size_t d_bytes, size_t sum_bytes, size_t x_bytes, size_t w_bytes)
      : d(0), sums(d_bytes), part(sums + sum_bytes), part_w(part + x_bytes), total(std::max<size_t>(part_w + w_bytes, 256)) {}
};
Layout forward_layout(const Chosen& c, int rows, int N, int n2) { return Layout(0, 0, own_bytes(c.parts, (long)rows * N * n2), 0); }
Layout backward_layout(const Chosen& c, int rows, int N, int K, int n2, int n_d, bool sums) {
  return Layout(n_d * up((size_t)rows * N * 2), sums ? up((size_t)pre_chunks(rows, N, true) * N * 4) : 0, own_bytes(c.parts, (long)rows * K),
                own_bytes(c.parts_w, (long)n2 * N * K));
}
// what any call of up to these sizes takes: grows with each of them
size_t forward_most(int rows, int N, int K, int n2) {
  return Layout(0, 0, rows <= kFewRows ? 0 : part_bytes(rows, (long)rows * N * n2, stages_of(K)), 0).total;
}
size_t backward_most(int rows, int N, int K, int n2, int n_d, bool sums, bool dx, bool dw) {
  // (sums: pre_chunks' at most, but growing with N)
  return Layout(n_d * up((size_t)rows * N * 2),
                sums ? up((size_t)std::min(std::max(over(rows, 4), 1l) * N, kPreGroups * 8l * kT) * 4) : 0,
                dx ? part_bytes(rows, (long)rows * K, (long)n2 * stages_of(N)) : 0,
                dw ? part_bytes(INT_MAX, (long)n2 * N * K, stages_of(rows)) : 0)
      .total;
}
void describe(const Chosen& c, const Layout& L, dflare_product_plan* to) {
  *to = dflare_product_plan{c.tiles, c.parts, c.parts_w, c.split, L.total};
}
// zeros by a kernel (a memset node of a captured graph is not relied upon)
__global__ __launch_bounds__(kT) void k_zero(u32x4* p, long n) {
  const long i = blockIdx.x * (long)kT + threadIdx.x;
  if (i < n) p[i] = u32x4{0u, 0u, 0u, 0u};
}
void zero(void* p, size_t bytes, hipStream_t st) {
  if (p) hipLaunchKernelGGL(k_zero, dim3((unsigned)((bytes / 16 + kT - 1) / kT)), dim3(kT), 0, st, (u32x4*)p, (long)(bytes / 16));
}

}  // namespace

}  // namespace dflare

using namespace dflare;

extern "C" {

size_t dflare_linear_fwd_workspace(int32_t rows, int32_t N, int32_t K) {
  return check(rows, N, K, 0) == DFLARE_OK ? forward_most(rows, N, K, 1) : 0;
}

int dflare_linear_fwd(const void* x, const void* w, const void* bias, const void* residual, int32_t rows, int32_t N, int32_t K, int32_t act,
                      void* y, void* z, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(rows, N, K, act);
  if (rc != DFLARE_OK) return rc;
  if (!w || !workspace || (rows > 0 && (!x || !y))) return DFLARE_ERR_INVALID_ARG;
  const Chosen c = forward_plan(rows, N, K, 1);
  const size_t xb = (size_t)rows * K * 2, wb = (size_t)N * K * 2, yb = (size_t)rows * N * 2, ws = forward_layout(c, rows, N, 1).total;
  if (off16({x, w, bias, residual, y, z, workspace}) || workspace_bytes < ws) return DFLARE_ERR_INVALID_ARG;
  if (!apart({{y, yb}, {z, yb}, {workspace, ws}}, {{x, xb}, {w, wb}, {bias, (size_t)N * 2}}) ||
      !apart({{z, yb}, {workspace, ws}}, {{residual, yb}}) || !same_or_apart(y, residual, yb))
    return DFLARE_ERR_INVALID_ARG;
  if (rows == 0) return DFLARE_OK;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  Call a{};
  a.x = (const uint16_t*)x;
  a.w[0] = (const uint16_t*)w;
  a.bias = (const uint16_t*)bias;
  a.res = (const uint16_t*)residual;
  a.y = (uint16_t*)y;
  a.z[0] = (uint16_t*)z;
  a.part = (float*)workspace;
  a.rows = rows;
  a.N = N;
  a.K = K;
  a.n2 = 1;
  a.act = act;
  forward<false>(a, c, (hipStream_t)stream);
  return launched();
}

size_t dflare_linear_bwd_workspace(int32_t rows, int32_t N, int32_t K, int32_t act, int32_t dx, int32_t dw, int32_t dbias) {
  if (check(rows, N, K, act) != DFLARE_OK) return 0;
  return backward_most(rows, N, K, 1, act != DFLARE_ACT_NONE, dbias != 0, dx != 0, dw != 0);
}

int dflare_linear_bwd(const void* dy, const void* x, const void* w, const void* z, int32_t rows, int32_t N, int32_t K, int32_t act, void* dx,
                      void* dw, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(rows, N, K, act);
  if (rc != DFLARE_OK) return rc;
  const bool named = act != DFLARE_ACT_NONE;
  if (!workspace || (rows > 0 && (!dy || (named && !z) || (dx && !w) || (dw && !x)))) return DFLARE_ERR_INVALID_ARG;
  if (off16({dy, x, w, z, dx, dw, dbias, workspace})) return DFLARE_ERR_INVALID_ARG;
  const Chosen c = gradients_plan(rows, N, K, 1, dx != nullptr, dw != nullptr);
  const Layout L = backward_layout(c, rows, N, K, 1, named, dbias != nullptr);
  if (workspace_bytes < L.total) return DFLARE_ERR_INVALID_ARG;
  const size_t xb = (size_t)rows * K * 2, wb = (size_t)N * K * 2, yb = (size_t)rows * N * 2;
  if (!apart({{dx, xb}, {dw, wb}, {dbias, (size_t)N * 2}, {workspace, L.total}},
             {{dy, yb}, {dw ? x : nullptr, xb}, {dx ? w : nullptr, wb}, {named ? z : nullptr, yb}}))
    return DFLARE_ERR_INVALID_ARG;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (rows == 0) {
    zero(dw, wb, st);
    zero(dbias, (size_t)N * 2, st);
    return launched();
  }
  char* ws = (char*)workspace;
  Call a{};
  a.x = (const uint16_t*)x;
  a.w[0] = (const uint16_t*)w;
  a.dx = (uint16_t*)dx;
  a.dw[0] = (uint16_t*)dw;
  a.part = (float*)(ws + L.part);
  a.part_w = (float*)(ws + L.part_w);
  a.rows = rows;
  a.N = N;
  a.K = K;
  a.n2 = 1;
  a.d[0] = named ? (const uint16_t*)(ws + L.d) : (const uint16_t*)dy;
  const int chunks = pre_chunks(rows, N, dbias != nullptr);
  if (dbias || (named && (dx || dw))) {
    Pre p{};
    p.dy = (const uint16_t*)dy;
    p.z[0] = (const uint16_t*)z;
    p.d[0] = (uint16_t*)(ws + L.d);
    p.sums = dbias ? (float*)(ws + L.sums) : nullptr;
    p.rows = rows;
    p.N = N;
    p.act = act;
    p.chunks = chunks;
    pre_gradients<false>(p, st);
  }
  gradients(a, c, (const float*)(ws + L.sums), chunks, (uint16_t*)dbias, st);
  return launched();
}

int dflare_linear_plan(int32_t rows, int32_t N, int32_t K, int32_t act, int32_t dx, int32_t dw, int32_t dbias, dflare_product_plan* fwd,
                       dflare_product_plan* bwd) {
  const int rc = check(rows, N, K, act);
  if (rc != DFLARE_OK) return rc;
  if (fwd) {
    const Chosen c = forward_plan(rows, N, K, 1);
    describe(c, forward_layout(c, rows, N, 1), fwd);
  }
  if (bwd) {
    const Chosen c = gradients_plan(rows, N, K, 1, dx != 0, dw != 0);
    describe(c, backward_layout(c, rows, N, K, 1, act != DFLARE_ACT_NONE, dbias != 0), bwd);
  }
  return DFLARE_OK;
}

int dflare_gated_plan(int32_t rows, int32_t H, int32_t F, int32_t dx, int32_t dw, dflare_product_plan* fwd, dflare_product_plan* bwd) {
  const int rc = check(rows, F, H, 0);
  if (rc != DFLARE_OK) return rc;
  if (fwd) {
    const Chosen c = forward_plan(rows, F, H, 2);
    describe(c, forward_layout(c, rows, F, 2), fwd);
  }
  if (bwd) {
    const Chosen c = gradients_plan(rows, F, H, 2, dx != 0, dw != 0);
    describe(c, backward_layout(c, rows, F, H, 2, 2, false), bwd);
  }
  return DFLARE_OK;
}

size_t dflare_gated_fwd_workspace(int32_t rows, int32_t H, int32_t F) {
  return check(rows, F, H, 0) == DFLARE_OK ? forward_most(rows, F, H, 2) : 0;
}

int dflare_gated_fwd(const void* x, const void* w_gate, const void* w_up, int32_t rows, int32_t H, int32_t F, int32_t act, void* h, void* gate,
                     void* up, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check(rows, F, H, act);
  if (rc != DFLARE_OK) return rc;
  if (!w_gate || !w_up || !workspace || (rows > 0 && (!x || !h)) || !gate != !up) return DFLARE_ERR_INVALID_ARG;
  const Chosen c = forward_plan(rows, F, H, 2);
  const size_t ws = forward_layout(c, rows, F, 2).total;
  if (off16({x, w_gate, w_up, h, gate, up, workspace}) || workspace_bytes < ws) return DFLARE_ERR_INVALID_ARG;
  const size_t xb = (size_t)rows * H * 2, wb = (size_t)F * H * 2, yb = (size_t)rows * F * 2;
  if (!apart({{h, yb}, {gate, yb}, {up, yb}, {workspace, ws}}, {{x, xb}, {w_gate, wb}, {w_up, wb}}))
    return DFLARE_ERR_INVALID_ARG;
  if (rows == 0) return DFLARE_OK;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  Call a{};
  a.x = (const uint16_t*)x;
  a.w[0] = (const uint16_t*)w_gate;
  a.w[1] = (const uint16_t*)w_up;
  a.y = (uint16_t*)h;
  a.z[0] = (uint16_t*)gate;
  a.z[1] = (uint16_t*)up;
  a.part = (float*)workspace;
  a.rows = rows;
  a.N = F;
  a.K = H;
  a.n2 = 2;
  a.act = act;
  forward<true>(a, c, (hipStream_t)stream);
  return launched();
}

size_t dflare_gated_bwd_workspace(int32_t rows, int32_t H, int32_t F, int32_t dx, int32_t dw) {
  return check(rows, F, H, 0) == DFLARE_OK ? backward_most(rows, F, H, 2, 2, false, dx != 0, dw != 0) : 0;
}

int dflare_gated_bwd(const void* dh, const void* x, const void* gate, const void* up_, const void* w_gate, const void* w_up, int32_t rows,
                     int32_t H, int32_t F, int32_t act, void* dx, void* dw_gate, void* dw_up, void* workspace, size_t workspace_bytes,
                     void* stream) {
  int rc = check(rows, F, H, act);
  if (rc != DFLARE_OK) return rc;
  if (!workspace || !dw_gate != !dw_up) return DFLARE_ERR_INVALID_ARG;
  if (rows > 0 && (!dh || !gate || !up_ || (dx && (!w_gate || !w_up)) || (dw_gate && !x))) return DFLARE_ERR_INVALID_ARG;
  if (off16({dh, x, gate, up_, w_gate, w_up, dx, dw_gate, dw_up, workspace})) return DFLARE_ERR_INVALID_ARG;
  const Chosen c = gradients_plan(rows, F, H, 2, dx != nullptr, dw_gate != nullptr);
  const Layout L = backward_layout(c, rows, F, H, 2, 2, false);
  if (workspace_bytes < L.total) return DFLARE_ERR_INVALID_ARG;
  const size_t xb = (size_t)rows * H * 2, wb = (size_t)F * H * 2, yb = (size_t)rows * F * 2;
  if (!apart({{dx, xb}, {dw_gate, wb}, {dw_up, wb}, {workspace, L.total}},
             {{dh, yb}, {gate, yb}, {up_, yb}, {dw_gate ? x : nullptr, xb}, {dx ? w_gate : nullptr, wb}, {dx ? w_up : nullptr, wb}}))
    return DFLARE_ERR_INVALID_ARG;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (rows == 0) {
    zero(dw_gate, wb, st);
    zero(dw_up, wb, st);
    return launched();
  }
  char* ws = (char*)workspace;
  Call a{};
  a.x = (const uint16_t*)x;
  a.w[0] = (const uint16_t*)w_gate;
  a.w[1] = (const uint16_t*)w_up;
  a.dx = (uint16_t*)dx;
  a.dw[0] = (uint16_t*)dw_gate;
  a.dw[1] = (uint16_t*)dw_up;
  a.part = (float*)(ws + L.part);
  a.part_w = (float*)(ws + L.part_w);
  a.rows = rows;
  a.N = F;
  a.K = H;
  a.n2 = 2;
  Pre p{};
  p.dy = (const uint16_t*)dh;
  p.z[0] = (const uint16_t*)gate;
  p.z[1] = (const uint16_t*)up_;
  p.d[0] = (uint16_t*)(ws + L.d);
  p.d[1] = (uint16_t*)(ws + L.d + up((size_t)rows * F * 2));
  p.rows = rows;
  p.N = F;
  p.act = act;
  p.chunks = pre_chunks(rows, F, false);
  a.d[0] = p.d[0];
  a.d[1] = p.d[1];
  if (dx || dw_gate) pre_gradients<true>(p, st);
  gradients(a, c, nullptr, 0, nullptr, st);
  return launched();
}

}  // extern "C"
