// The LM head with the position-weighted cross-entropy (Sec. 3.3, Sec. 4.3, Eq. 5) and its gradients,
// without logits in memory.  With z = h W^T over the rows that carry a loss, c_r = w_r / sum w,
//   ce_r = lse(z_r) - z_r[y_r],  loss = sum c ce,  dz = c (softmax(z) - onehot(y)),
//   dh = dz W,  dW = dz^T h.
// The rows with a loss are gathered first (the others take no part in any product).
// The loss alone is one product, whose epilogue leaves every row's maximum and sum per wave's words.
// With dh alone the vocabulary is walked once, in pieces, as one pass of a softmax: a piece's product leaves
// 2^(z log2 e - R) in bf16 and the sums of these, R being a reference of the row, at first its label's logit to the
// next whole number; a second product adds (these) W to dh, which is divided by the whole sum at the end.  bf16 has
// the range of fp32, so that R need not be the maximum: only values more than 2^40 times it (which a wave's words
// then take as their own reference, raise a flag and have the row rescaled) move it.  References are whole numbers,
// so that what is rescaled is not rounded again.
// dW needs dz of all words of a row at its final scale.  Where the vocabulary is one piece, the rows of h take the
// scale instead (rounded to bf16; the labels' terms, most of dW, are not taken from them); otherwise the maxima
// and sums come first, and each piece's logits are formed again: 2 rows V H operations more.
// The label's word is left out of dz: its -c (1 - p), the largest value of its row, goes into dh and dW in fp32
// (rounded to bf16 with the others it would be 0.7 of the gradients' whole error).
// Bound by the matrix cores (up to some 128 rows by reading the head): 2 rows V H operations for the loss, 4 with dh,
// 6 with both from one piece, 8 from more.
#include <hip/hip_runtime.h>
#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dflare.h"
#include "product.h"

namespace dflare {

namespace {

constexpr int kBlock = 256; // words of a block of dz; rows and words are padded to it
constexpr float kL2E = 1.4426950408889634f;
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }

struct Lce {
  const uint16_t *hidden, *head;
  const int32_t* labels;
  float *loss, *row_ce;
  uint16_t *dhidden, *dhead;
  int rows, V, H, B;
  float gamma;
  // workspace; i counts the rows with a loss, Mp = rows rounded up to whole tiles
  int* count;     // [2] rows with a loss, parts of dh
  int* src;       // [Mp] i -> row
  int* pos;       // [rows] row -> i, -1 without a loss
  int* word;      // [Mp] i -> label, -1 past the last
  float* c;       // [Mp] w / sum w, 0 past the last
  uint16_t* hc;   // [Mp][ldh] gathered rows, zeros past H and past the last row of the last tile
  uint16_t* hs;   // [Mp][ldh] hc times fac, for dW from one piece: a place of its own, or hc's; else null
  float2* part;   // [words of a piece / a wave's][Mp] a reference R (log2 domain) and the sum of 2^(z log2 e - R), without the
                  // label's word
  float* zlab;    // [Mp] z at the label
  float* lab;     // [Mp] c (1 - p of the label)
  float *ref, *sum;  // [Mp] a row's reference and its sum over the pieces so far
  float* fac;     // [Mp] c over the whole sum (the label's word in it)
  bool one_pass;  // dz is 2^(z log2 e - R); otherwise at its final scale
  int* flag;      // of the pieces in one pass: a word took a reference of its own
  uint16_t* dz;   // [words of a piece / 256][Mp][256] dz of a piece of the vocabulary
  float* dacc;    // [parts][rows of whole tiles][H] dh of the pieces so far; then [dw_parts][V][H] dW
  int Mp, ldh;
  int stages;     // stages of k of the first (longest) piece
  int dw_parts;   // dW's rows are split into
  int dh_tile;    // dh on the large tile (0), the small one, or that for few rows
};

// dh's tiles for n rows with a loss.  The words of a piece are split into `parts` where there are few tiles for the
// work-groups that 256 CUs hold: the number with the least time, a round of work-groups costing its stages of k
// and about 8 more for its start and its sums in memory, the sum of the parts n H / 1.45 M each (in stages: 1.45 us
// measured on the large tile).  More than one part makes at most two rounds, which is what dacc is sized by (more was not
// measured; 290 tiles, as of 7,296 rows x 2,560, stay whole and fill 57% of two rounds).  The number depends on the rows
// with a loss, so that it is chosen on the device (k_lce_rows).
constexpr int kMostParts = 128;
__host__ __device__ constexpr int dh_slots(int tile) { return 256 * (tile + 1); }  // work-groups that the CUs hold
struct DhPlan {
  int tn, nb, na, parts;
  __device__ __forceinline__ DhPlan(const Lce& a, int n) {
    static_assert(Few::TM == Small::TM);
    tn = a.dh_tile == 2 ? Few::TN : a.dh_tile ? Small::TN : Large::TN;
    nb = (n + tn - 1) / tn;
    na = a.dh_tile ? (a.H + Small::TM - 1) / Small::TM : (a.H + Large::TM - 1) / Large::TM;
    parts = a.count[1];
  }
  __device__ __forceinline__ long part_rows() const { return (long)nb * tn; }
  // by one wave
  __device__ __forceinline__ int choose(const Lce& a, int n) const {
    const int slots = dh_slots(a.dh_tile);
    unsigned best = ~0u;  // cost and parts
    for (int k = 1 + (threadIdx.x & 63); k <= kMostParts; k += 64) {
      if (k > 1 && (nb * (long)na * k > 2 * slots || a.stages < 4 * k)) continue;
      const long cost = (nb * (long)na * k + slots - 1) / slots * ((a.stages + k - 1) / k + 8) +
                        (long)n * a.H * k / 1450000;
      best = min(best, (unsigned)min(cost, (1l << 24) - 2) << 8 | k);
    }
    for (int off = 32; off > 0; off >>= 1) best = min(best, (unsigned)__shfl_xor((int)best, off));
    return best & 255;
  }
};

// ---- rows with a loss, in order; their weights; work-group of 1,024 threads ----
__global__ __launch_bounds__(1024) void k_lce_rows(Lce a, int pieces) {
  __shared__ int wc[16];
  __shared__ double ws[16];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  int n = 0;
  double sum = 0.0;
  for (int base = 0; base < a.rows; base += 1024) {
    const int r = base + tid;
    const int b = r % a.B, y = r < a.rows ? a.labels[r] : -1;
    const bool on = b > 0 && y >= 0 && y < a.V;
    const uint64_t m = __builtin_amdgcn_ballot_w64(on);
    if (lane == 0) wc[wv] = __builtin_popcountll(m);
    __syncthreads();
    int i = n + __builtin_popcountll(m & ((1ull << lane) - 1));
    for (int k = 0; k < 16; ++k) {
      if (k < wv) i += wc[k];
      n += wc[k];
    }
    __syncthreads();
    if (on) {
      const float w = expf(-(float)(b - 1) / a.gamma);
      sum += w;
      a.src[i] = r;
      a.word[i] = y;
      a.c[i] = w;
    }
    if (r < a.rows) {
      a.pos[r] = on ? i : -1;
      if (!on) a.row_ce[r] = 0.f;
    }
  }
  auto total = [&](double v) {  // over the work-group
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    __syncthreads();
    if (lane == 0) ws[wv] = v;
    __syncthreads();
    v = 0.0;
    for (int k = 0; k < 16; ++k) v += ws[k];
    return v;
  };
  sum = total(sum);
  if (n > 0 && sum < 1e-30) {  // the first rows with a loss lie so late in their blocks that the weights leave fp32: from there
    int lo = INT_MAX;
    for (int i = tid; i < n; i += 1024) lo = min(lo, a.src[i] % a.B);
    for (int off = 32; off > 0; off >>= 1) lo = min(lo, __shfl_xor(lo, off));
    if (lane == 0) wc[wv] = lo;
    __syncthreads();
    for (int k = 0; k < 16; ++k) lo = min(lo, wc[k]);
    sum = 0.0;
    for (int i = tid; i < n; i += 1024) {
      const float w = expf(-(float)(a.src[i] % a.B - lo) / a.gamma);
      sum += w;
      a.c[i] = w;
    }
    sum = total(sum);
  }
  const double inv = sum > 0.0 ? 1.0 / sum : 0.0;
  const int np = min((n + kBlock - 1) / kBlock * kBlock, a.Mp);
  for (int i = tid; i < np; i += 1024) {
    a.c[i] = i < n ? (float)(a.c[i] * inv) : 0.f;
    if (i >= n) a.word[i] = -1;
  }
  if (a.flag)
    for (int i = tid; i < pieces; i += 1024) a.flag[i] = 0;
  if (wv == 0) {
    const int parts = DhPlan(a, n).choose(a, n);
    if (tid == 0) {
      a.count[0] = n;
      a.count[1] = parts;
    }
  }
}

// a row of hc; one pass: also the label's logit and the first reference
__global__ __launch_bounds__(256) void k_lce_gather(Lce a) {
  __shared__ float red[4];
  const int n = a.count[0], i = blockIdx.x;
  if (i >= (n + kBlock - 1) / kBlock * kBlock) return;
  const u32x4 z = {0u, 0u, 0u, 0u};
  const int row = i < n ? a.src[i] : 0;
  const u32x4* from = reinterpret_cast<const u32x4*>(a.hidden + (long)row * a.H);
  u32x4* to = reinterpret_cast<u32x4*>(a.hc + (long)i * a.ldh);
  const bool dot = a.one_pass && i < n;
  const u32x4* word = reinterpret_cast<const u32x4*>(a.head + (dot ? (long)a.word[i] * a.H : 0));
  float s = 0.f;
  for (int p = threadIdx.x; p < a.ldh / 8; p += 256) {
    const bool in = i < n && p < a.H / 8;
    const u32x4 v = in ? from[p] : z;
    to[p] = v;
    if (dot && in) {
      const u32x4 x = word[p];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s = fmaf(__uint_as_float(v[e] << 16), __uint_as_float(x[e] << 16), s);
        s = fmaf(__uint_as_float(v[e] & 0xFFFF0000u), __uint_as_float(x[e] & 0xFFFF0000u), s);
      }
    }
  }
  if (!a.one_pass) return;
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = (red[0] + red[1]) + (red[2] + red[3]);
    a.zlab[i] = s;
    a.ref[i] = rintf(s * kL2E);
  }
}

enum { kStats, kDz, kExp, kDh, kDw };
// how far above its reference (log2) a row's values may lie: their sums and these' inverses stay far inside fp32
constexpr float kRise = 40.f;

// One tile of a product and its epilogue:
//   kStats  z tile (words x rows) -> part, zlab
//   kDz     z tile of the piece from word v0 on -> dz
//   kExp    the same -> 2^(z log2 e - R) in the place of dz, part
//   kDh     dacc (+)= dz W over the piece's words, in parts
//   kDw     dhead rows of the piece = dz^T h
template <typename S, int MODE>
__global__ __launch_bounds__(S::T, 2) void k_lce_product(Lce a, int v0, int nv, int piece) {
  __shared__ __attribute__((aligned(1024))) char lds[2 * S::kStageBytes];
  constexpr int TM = S::TM, TN = S::TN, MT = S::MT, NT = S::NT, WM = MT * 32, WN = NT * 32;  // (a wave's m and n)
  const int n = a.count[0], nb = (n + TN - 1) / TN;  // rows with a loss, tiles of them
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = lane >> 5, wm = w % S::WM, wn = w / S::WM;
  Acc<S> acc;
  int ta, tb;
  if constexpr (MODE <= kExp) {
    if (!tile_of(blockIdx.x, (nv + TM - 1) / TM, nb, ta, tb)) return;
    const int vt = v0 + ta * TM, r0 = tb * TN;
    product<S, false, false>(Operand{a.head + (long)vt * a.H, a.H, min(a.V - vt, TM), a.H},
                          Operand{a.hc + (long)r0 * a.ldh, a.ldh, TN, INT_MAX}, a.H, lds, acc, [](Acc<S>&) {});
    const int vw = vt + wm * WM;  // the wave's first word
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int rl = wn * WN + j * 32 + (lane & 31), i = r0 + rl;
      // the label's place among the wave's words, if it is there
      const int rel = i < n ? a.word[i] - vw : -1;
      const bool here = rel >= 0 && rel < WM && ((rel >> 2) & 1) == h;
      const int le = here ? (rel >> 5) * 16 + ((rel & 31) >> 3) * 4 + (rel & 3) : -1;  // its (tile, element) of this lane
      auto each = [&](auto f) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float z = acc[t][j][e];
            f(t, e, z);
            acc[t][j][e] = z;
          }
      };
      if (vw + WM > a.V)  // words past the last do not take part
        each([&](int t, int e, float& z) {
          if (vw + t * 32 + 8 * (e >> 2) + 4 * h + (e & 3) >= a.V) z = -INFINITY;
        });
      if constexpr (MODE == kStats) {
        if (__builtin_amdgcn_ballot_w64(here)) {  // (left out of the sum: 1 - p would be lost in it where p is nearly 1)
          float zl = 0.f;
          each([&](int t, int e, float& z) {
            const bool l = t * 16 + e == le;
            zl = l ? z : zl;
            z = l ? -INFINITY : z;
          });
          if (here) a.zlab[i] = zl;
        }
        float m = -FLT_MAX, s = 0.f;
        each([&](int, int, float& z) { m = fmaxf(m, z); });
        m = fmaxf(fmaxf(m, __shfl_xor(m, 32)) * kL2E, -FLT_MAX);  // (finite where the wave has no words: they add 0)
        each([&](int, int, float& z) { s += ex2(fmaf(z, kL2E, -m)); });
        s += __shfl_xor(s, 32);
        if (h == 0) a.part[(long)((vw - v0) / WM) * a.Mp + i] = make_float2(m, s);
      } else {
        if constexpr (MODE == kDz) {
          const float c = a.c[i], f = a.fac[i], r = a.ref[i];
          each([&](int t, int e, float& z) {
            z = f * ex2(fmaf(z, kL2E, -r));
            if (t * 16 + e == le || c == 0.f) z = 0.f;
          });
        } else {
          if (__builtin_amdgcn_ballot_w64(here)) each([&](int t, int e, float& z) { z = t * 16 + e == le ? -INFINITY : z; });
          float m = -FLT_MAX, s = 0.f, r = a.ref[i];
          each([&](int, int, float& z) { m = fmaxf(m, z); });
          m = fmaxf(m, __shfl_xor(m, 32)) * kL2E;
          const bool over = m > r + kRise;
          if (__builtin_amdgcn_ballot_w64(over) && lane == 0) a.flag[piece] = 1;
          r = over ? rintf(m) : r;
          each([&](int, int, float& z) {
            z = ex2(fmaf(z, kL2E, -r));
            s += z;
          });
          s += __shfl_xor(s, 32);
          if (h == 0) a.part[(long)((vw - v0) / WM) * a.Mp + i] = make_float2(r, s);
        }
        put_tile<S>(lds, acc, j, rl, wm * MT, h);
      }
    }
    if constexpr (MODE != kStats) {
      __syncthreads();
      store_tile<S>(lds, a.dz + ((long)(ta * TM / kBlock) * a.Mp + r0) * kBlock + ta * TM % kBlock, kBlock, TN, TM);
    }
  } else if constexpr (MODE == kDh) {
    const DhPlan plan(a, n);
    const int na = plan.na, parts = plan.parts, stages = (nv + kBK - 1) / kBK;
    int unit;
    if (!tile_of(blockIdx.x, na * parts, nb, unit, tb)) return;
    ta = unit % na;
    const int ks = unit / na, m0 = ta * TM, r0 = tb * TN;
    // this part's words: whole stages
    const int s0 = (int)((long)stages * ks / parts), s1 = (int)((long)stages * (ks + 1) / parts);
    const int words = min(s1 * kBK, nv) - s0 * kBK;
    product<S, true, false>(Operand{a.head + (long)(v0 + s0 * kBK) * a.H + m0, a.H, min(a.H - m0, TM), words},
                         Operand{a.dz + (long)r0 * kBlock, kBlock, TN, INT_MAX, (long)a.Mp * kBlock * 2, s0}, words, lds, acc, [](Acc<S>&) {});
    float* out = a.dacc + ks * plan.part_rows() * a.H;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float* row = out + (long)(r0 + wn * WN + j * 32 + (lane & 31)) * a.H;
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int m = m0 + wm * WM + t * 32 + q * 8 + 4 * h;
          if (m >= a.H) continue;
          f32x4* at = reinterpret_cast<f32x4*>(row + m);
          const f32x4 v = {acc[t][j][4 * q], acc[t][j][4 * q + 1], acc[t][j][4 * q + 2], acc[t][j][4 * q + 3]};
          *at = piece == 0 ? v : *at + v;
        }
    }
  } else {
    const int na = (a.H + TM - 1) / TM, stages = (n + kBK - 1) / kBK;
    int unit;
    if (!tile_of(blockIdx.x, na * a.dw_parts, (nv + TN - 1) / TN, unit, tb)) return;
    const int ks = unit / na, m0 = unit % na * TM, n0 = tb * TN;
    // this part's rows: whole stages
    const int i_first = (int)((long)stages * ks / a.dw_parts) * kBK, i_end = min((int)((long)stages * (ks + 1) / a.dw_parts) * kBK, n);
    product<S, true, true>(Operand{(a.hs ? a.hs : a.hc) + (long)i_first * a.ldh + m0, a.ldh, min(a.ldh - m0, TM), a.Mp - i_first},
                        Operand{a.dz + ((long)(n0 / kBlock) * a.Mp + i_first) * kBlock + n0 % kBlock, kBlock, TN, a.Mp - i_first},
                        max(i_end - i_first, 0), lds, acc, [&](Acc<S>& d) {
      // The label terms: the rows whose label is one of the wave's words, in order.  A lane keeps the next row of each of its
      // two words; when one would have a second, all that are kept are added at once.  (One row at a time, by the wave: 7,300
      // rows of 1,000 words x 4,096 582 us the call against 378.)  Rows of one label come one after another, a microsecond each: 7,300
      // rows of 32,003 words x 2,560 4.1 ms where no label stands out, 4.1 with one in 5% of them, 11 where all are the same.
      static_assert(NT == 2, "a lane's words");
      const int word0 = v0 + n0 + wn * WN;
      const bool scaled = a.hs == a.hc;  // hc holds hs: the rows themselves are read where they came from
      const long ld = scaled ? a.H : a.ldh;
      const uint16_t* col = (scaled ? a.hidden : a.hc) + m0 + wm * WM + 4 * h;
      const int most = (int)ld - 4 - (m0 + wm * WM + 4 * h);  // (columns past the last are not kept)
      int kept[2] = {-1, -1};
      uint64_t taken = 0;  // words that have a row
      auto add_kept = [&] {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (kept[j] >= 0) {
            const float f = -a.lab[kept[j]];
            const uint16_t* row = col + (scaled ? a.src[kept[j]] : kept[j]) * ld;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const u32x2 v = *reinterpret_cast<const u32x2*>(row + min(t * 32 + q * 8, most));
                const f32x4 x = unpack4(v[0], v[1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) d[t][j][4 * q + e] = fmaf(f, x[e], d[t][j][4 * q + e]);
              }
          }
          kept[j] = -1;
        }
        taken = 0;
      };
      for (int i0 = i_first; i0 < i_end; i0 += 256) {
        int y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + 64 * k + lane;
          y[k] = i < i_end ? a.word[i] - word0 : -1;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint64_t hit = __builtin_amdgcn_ballot_w64((unsigned)y[k] < (unsigned)WN);
          while (hit) {
            const int b = __builtin_ctzll(hit), wl = __builtin_amdgcn_readlane(y[k], b);
            hit &= hit - 1;
            if (taken >> wl & 1) add_kept();
            taken |= 1ull << wl;
            if ((lane & 31) == (wl & 31)) {
              if (wl < 32) kept[0] = i0 + 64 * k + b;
              else kept[1] = i0 + 64 * k + b;
            }
          }
        }
      }
      if (taken) add_kept();
    });
    if (a.dw_parts > 1) {
      float* out = a.dacc + ((long)ks * nv + n0) * a.H;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int wl = wn * WN + j * 32 + (lane & 31);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int m = m0 + wm * WM + t * 32 + q * 8 + 4 * h;
            if (n0 + wl < nv && m < a.H)
              *reinterpret_cast<f32x4*>(out + (long)wl * a.H + m) =
                  f32x4{acc[t][j][4 * q], acc[t][j][4 * q + 1], acc[t][j][4 * q + 2], acc[t][j][4 * q + 3]};
          }
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) put_tile<S>(lds, acc, j, wn * WN + j * 32 + (lane & 31), wm * MT, h);
    __syncthreads();
    store_tile<S>(lds, a.dhead + (long)(v0 + n0) * a.H + m0, a.H, min(nv - n0, TN), min(a.H - m0, TM));
  }
}

// A row's values from its parts: work-groups of 1,024 threads take R rows, each by 1,024 / R groups of parts

// The cross-entropy log(1 + s / 2^y) of row i, s and the label's 2^y (y = z log2 e - r) on the reference r, and what the
// gradients take
__device__ __forceinline__ float close_row(const Lce& a, int i, float s, float r) {
  const float y = fmaf(a.zlab[i], kL2E, -r), ey = ex2(y), c = a.c[i], inv = 1.f / (s + ey), f = c * inv;
  a.fac[i] = f;
  a.lab[i] = c * (s * inv);
  // far below the reference 2^y may be 0
  a.row_ce[a.src[i]] = y > -60.f ? log1pf(s / ey) : (log2f(s + ey) - y) * 0.6931471805599453f;
  return f;
}

// After a piece of the first pass over the maxima: a row's sum so far from its parts; after the last, its cross-entropy
template <int R>
__global__ __launch_bounds__(1024) void k_lce_lse(Lce a, int parts, bool first, bool last) {
  __shared__ float2 sh[16][R];
  const int n = a.count[0], l = threadIdx.x % R, g = threadIdx.x / R, i = blockIdx.x * R + l;
  if ((int)blockIdx.x * R >= n) return;
  float m = -FLT_MAX, s = 0.f;
  auto add = [&](float x, float y) {
    const float mn = fmaxf(m, x);
    s = s * ex2(m - mn) + y * ex2(x - mn);
    m = mn;
  };
#pragma unroll 8
  for (int p = g; p < parts; p += 1024 / R) {
    const float2 v = a.part[(long)p * a.Mp + i];
    add(v.x, v.y);
  }
  for (int off = 32; off >= R; off >>= 1) add(__shfl_xor(m, off), __shfl_xor(s, off));
  if ((threadIdx.x & 63) < R) sh[threadIdx.x >> 6][l] = make_float2(m, s);
  __syncthreads();
  if (g != 0 || i >= n) return;
  for (int k = 1; k < 16; ++k) add(sh[k][l].x, sh[k][l].y);
  if (!first) add(a.ref[i], a.sum[i]);
  if (!last) {
    a.ref[i] = m;
    a.sum[i] = s;
    return;
  }
  const float r = fmaxf(m, a.zlab[i] * kL2E);  // of all words: 2^y is 1 at most
  a.ref[i] = r;
  close_row(a, i, s * ex2(m - r), r);
}

// Row i of a piece in which some words took a reference of their own: the row's reference becomes the highest of them
// (returned), and what was written under others, dh of the pieces before it included, is scaled to it.  By a
// work-group; red: a float per wave.
__device__ __forceinline__ float rebase_row(const Lce& a, int i, int nv, int piece, int wave, float* red) {
  const int groups = (nv + wave - 1) / wave;  // groups of a wave's words
  const float2* p = a.part + i;
  const float old = a.ref[i];
  float r = old;
  for (int g = threadIdx.x; g < groups; g += blockDim.x) r = fmaxf(r, p[(long)g * a.Mp].x);
  for (int off = 32; off > 0; off >>= 1) r = fmaxf(r, __shfl_xor(r, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = r;
  __syncthreads();
  for (int k = 0; k < (int)blockDim.x / 64; ++k) r = fmaxf(r, red[k]);
  if (!(r > old)) return old;
  for (int e = threadIdx.x; e < groups * (wave / 8); e += blockDim.x) {  // 8 words each
    const int g = e / (wave / 8);
    const float f = ex2(p[(long)g * a.Mp].x - r);
    if (f == 1.f) continue;
    u32x4* at = reinterpret_cast<u32x4*>(a.dz + ((long)(e / (kBlock / 8)) * a.Mp + i) * kBlock) + e % (kBlock / 8);
    u32x4 v = *at;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = pack2(__uint_as_float(v[k] << 16) * f, __uint_as_float(v[k] & 0xFFFF0000u) * f);
    *at = v;
  }
  if (piece > 0) {
    const DhPlan plan(a, a.count[0]);
    for (int k = 0; k < plan.parts; ++k) {
      float* d = a.dacc + (k * plan.part_rows() + i) * a.H;
      for (int m = threadIdx.x; m < a.H; m += blockDim.x) d[m] *= ex2(old - r);
    }
  }
  if (threadIdx.x == 0) a.ref[i] = r;
  return r;
}

// One pass, after a piece's logits: its rows rescaled where it needs that, and the rows' sums so far from their parts; after the
// last piece their cross-entropy and the factors of dh, and with dhead hs.  (In launches of their own these
// made 207 rows x 32,003 x 264 6 us of 68 longer.)  7,296 rows x 30,464 words: 9.4 us.
template <int R>
__global__ __launch_bounds__(1024) void k_lce_close(Lce a, int nv, int piece, bool last, int wave) {
  __shared__ float sh[16][R], red[16], ref[R], fac[R];
  const int n = a.count[0], row0 = blockIdx.x * R, parts = (nv + wave - 1) / wave;
  if (row0 >= (a.hs ? (n + kBlock - 1) / kBlock * kBlock : n)) return;
  const int l = threadIdx.x % R, g = threadIdx.x / R, i = row0 + l;
  const float old = i < n ? a.ref[i] : 0.f;
  if (threadIdx.x < R) {
    ref[l] = old;
    fac[l] = 0.f;
  }
  if (a.flag[piece])
    for (int k = 0; k < R && row0 + k < n; ++k) {
      const float r = rebase_row(a, row0 + k, nv, piece, wave, red);
      if (threadIdx.x == 0) ref[k] = r;
    }
  __syncthreads();
  const float r = ref[l];
  float s = 0.f;
  if (i < n) {
#pragma unroll 8
    for (int p = g; p < parts; p += 1024 / R) {
      const float2 v = a.part[(long)p * a.Mp + i];
      s += v.y * ex2(v.x - r);
    }
  }
  for (int off = 32; off >= R; off >>= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) < R) sh[threadIdx.x >> 6][l] = s;
  __syncthreads();
  if (g == 0 && i < n) {
    for (int k = 1; k < 16; ++k) s += sh[k][l];  // all words but the label's
    if (piece > 0) s += a.sum[i] * ex2(old - r);
    if (last) fac[l] = close_row(a, i, s, r);
    else a.sum[i] = s;
  }
  if (!a.hs) return;
  __syncthreads();
  const int P = a.ldh / 8;
  for (int e = threadIdx.x; e < R * P; e += 1024) {
    const long at = (long)(row0 + e / P) * P + e % P;
    const float f = fac[e / P];
    u32x4 v = reinterpret_cast<const u32x4*>(a.hc)[at];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = pack2(__uint_as_float(v[k] << 16) * f, __uint_as_float(v[k] & 0xFFFF0000u) * f);
    reinterpret_cast<u32x4*>(a.hs)[at] = v;
  }
}

// loss = sum of c ce in 64 bits, in a fixed order, by one work-group of 256
__device__ __forceinline__ void sum_loss(const Lce& a) {
  __shared__ double ws[4];
  const int n = a.count[0];
  double s = 0.0;
#pragma unroll 8
  for (int i = threadIdx.x; i < n; i += 256) s += (double)a.c[i] * a.row_ce[a.src[i]];
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) ws[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.loss[0] = (float)((ws[0] + ws[1]) + (ws[2] + ws[3]));
}
__global__ __launch_bounds__(256) void k_lce_loss(Lce a) { sum_loss(a); }

// dhidden: the parts' sum, scaled, with the label's term; rounded once; zeros in rows without a loss.  G threads take
// 8 values of a row, each every G-th part.  The first work-group forms the loss.
template <int G>
__global__ __launch_bounds__(256) void k_lce_dhidden(Lce a) {
  if (blockIdx.x == 0) return sum_loss(a);
  const int P = a.H / 8, g = threadIdx.x % G;
  const long at = (blockIdx.x - 1) * (256l / G) + threadIdx.x / G;
  if (at >= (long)a.rows * P) return;
  const int row = (int)(at / P), p = (int)(at - (long)row * P), i = a.pos[row];
  u32x4 out = {0u, 0u, 0u, 0u};
  if (i >= 0) {
    const DhPlan plan(a, a.count[0]);
    const float f = a.one_pass ? a.fac[i] : 1.f, fl = a.lab[i];
    const u32x4 v = reinterpret_cast<const u32x4*>(a.head + (long)a.word[i] * a.H)[p];
    const f32x4* from = reinterpret_cast<const f32x4*>(a.dacc + (long)i * a.H) + 2 * p;
    const long step = plan.part_rows() * a.H / 4;
    f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll 4
    for (int k = g; k < plan.parts; k += G) {
      x += from[k * step];
      y += from[k * step + 1];
    }
#pragma unroll
    for (int off = 1; off < G; off <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] += __shfl_xor(x[e], off);
        y[e] += __shfl_xor(y[e], off);
      }
    x = x * f - fl * unpack4(v[0], v[1]);
    y = y * f - fl * unpack4(v[2], v[3]);
    out = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(y[0], y[1]), pack2(y[2], y[3])};
  }
  if (g == 0) reinterpret_cast<u32x4*>(a.dhidden)[at] = out;
}

// dhead from its parts; rounded once
__global__ __launch_bounds__(256) void k_lce_dhead(Lce a) {
  const long at = blockIdx.x * 256l + threadIdx.x, n = (long)a.V * a.H / 8;
  if (at >= n) return;
  const f32x4* from = reinterpret_cast<const f32x4*>(a.dacc) + 2 * at;
  f32x4 x = from[0], y = from[1];
#pragma unroll 4
  for (int k = 1; k < a.dw_parts; ++k) {
    x += from[k * 2 * n];
    y += from[k * 2 * n + 1];
  }
  reinterpret_cast<u32x4*>(a.dhead)[at] = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(y[0], y[1]), pack2(y[2], y[3])};
}

// ---- host side ----
template <int N>
using mode_c = std::integral_constant<int, N>;
constexpr size_t kDzBytes = 512u << 20;    // room for dz of a piece of the vocabulary
constexpr size_t kPartBytes = 128u << 20;  // and for the parts of one (8,192 rows x 201,088 words, the loss alone: one piece)
// hs has a place of its own up to this size: 8,192 rows x 1,024 are scaled in 9.7 us there and in 13.7 in hc's place (of 156
// the call with 1,000 words), x 4,096 in 24.0 and 24.5
constexpr size_t kScaledBytes = 32u << 20;

struct LceLayout {
  size_t part_bytes, count, src, pos, word, c, hc, hs, part, zlab, ref, sum, fac, lab, flag, dz, dacc, total;
  int Mp, ldh, Vp;
};

LceLayout lce_layout(int rows, int V, int H, bool dhidden, bool dhead) {
  LceLayout L{};
  auto al = [](size_t x) { return (x + 255) / 256 * 256; };
  L.Mp = (rows + kBlock - 1) / kBlock * kBlock;
  L.ldh = (H + 63) / 64 * 64;
  const int words = (int)((V + (long)kBlock - 1) / kBlock);  // tiles of the vocabulary
  // pieces of equal numbers of tiles
  const int most = (int)std::max<size_t>(1, std::min<size_t>(words, kDzBytes / ((size_t)L.Mp * kBlock * 2)));
  const int pieces = (words + most - 1) / most;
  L.Vp = (words + pieces - 1) / pieces * kBlock;
  size_t o = 0;
  auto take = [&](size_t& at, size_t bytes) {
    at = o;
    o = al(o + bytes);
  };
  take(L.count, 8);
  take(L.src, (size_t)L.Mp * 4);
  take(L.pos, (size_t)rows * 4);
  take(L.word, (size_t)L.Mp * 4);
  take(L.c, (size_t)L.Mp * 4);
  take(L.hc, (size_t)L.Mp * L.ldh * 2);
  if (dhead) take(L.hs, std::min((size_t)L.Mp * L.ldh * 2, kScaledBytes));
  // (a wave of the small tile has 64 words, so a piece with dz, of 2^28 logits or one block of words, has 32 MB or a block's)
  L.part_bytes = std::min((size_t)words * L.Mp * 32, std::max(kPartBytes, (size_t)L.Mp * 32));
  take(L.part, L.part_bytes);
  take(L.zlab, (size_t)L.Mp * 4);
  take(L.ref, (size_t)L.Mp * 4);
  take(L.sum, (size_t)L.Mp * 4);
  take(L.fac, (size_t)L.Mp * 4);
  take(L.lab, (size_t)L.Mp * 4);
  take(L.flag, (size_t)words * 4);
  // (bounds of what is used that grow with every size: a workspace for the largest call serves the smaller ones)
  const size_t tile = (size_t)L.Mp * kBlock * 2, values = (size_t)L.Mp * H;
  if (dhidden || dhead) take(L.dz, std::min(tile * words, std::max(kDzBytes, tile)));
  const size_t dh = std::max(values, std::min(kMostParts * values, (size_t)512 * 65536)),
               dw = std::min(kMostParts * (size_t)V * H, (size_t)512 * 65536);
  if (dhidden || dhead) take(L.dacc, std::max(dhidden ? dh : 0, dhead ? dw : 0) * 4);
  L.total = o;
  return L;
}

int lce_check(int rows, int V, int H, int B) {
  if (rows < 1 || V < 1 || H < 1 || B < 1 || rows % B) return DFLARE_ERR_INVALID_ARG;
  if (H % 8 || H > 16384 || rows > (1 << 22)) return DFLARE_ERR_UNSUPPORTED;
  // a launch has less than 2^32 threads
  const long tiles = (long)((rows + kBlock - 1) / kBlock) * ((V + (long)kBlock - 1) / kBlock);
  if (tiles >= (1l << 22) - 8 || (long)rows * H > (1l << 35) - 4096) return DFLARE_ERR_UNSUPPORTED;
  return DFLARE_OK;
}

}  // namespace

}  // namespace dflare

using namespace dflare;

extern "C" {

size_t dflare_linear_ce_workspace(int32_t rows, int32_t V, int32_t H, int32_t dhidden, int32_t dhead) {
  if (lce_check(rows, V, H, 1) != DFLARE_OK) return 0;
  return lce_layout(rows, V, H, dhidden != 0, dhead != 0).total;
}

int dflare_linear_ce(const void* hidden, const void* head, const int32_t* labels, int32_t rows, int32_t V, int32_t H,
                     int32_t B, float gamma, float* loss, float* row_ce, void* dhidden, void* dhead, void* workspace,
                     size_t workspace_bytes, void* stream) {
  const int rc = lce_check(rows, V, H, B);
  if (rc != DFLARE_OK) return rc;
  if (!hidden || !head || !labels || !loss || !row_ce || !workspace || !(gamma > 0.f) || !isfinite(gamma))
    return DFLARE_ERR_INVALID_ARG;
  for (const void* p : {hidden, head, (const void*)dhidden, (const void*)dhead, (const void*)workspace})
    if ((uintptr_t)p & 15) return DFLARE_ERR_INVALID_ARG;
  for (const void* p : {(const void*)labels, (const void*)loss, (const void*)row_ce})
    if ((uintptr_t)p & 3) return DFLARE_ERR_INVALID_ARG;
  const LceLayout L = lce_layout(rows, V, H, dhidden != nullptr, dhead != nullptr);
  if (workspace_bytes < L.total) return DFLARE_ERR_INVALID_ARG;
  // (the inputs are read until the last launch, row_ce is written by the first)
  const size_t hb = (size_t)rows * H * 2, wb = (size_t)V * H * 2, rb = (size_t)rows * 4;
  if (!apart({{loss, 4}, {row_ce, rb}, {dhidden, hb}, {dhead, wb}, {workspace, L.total}}, {{hidden, hb}, {head, wb}, {labels, rb}}))
    return DFLARE_ERR_INVALID_ARG;
  hipStream_t st = (hipStream_t)stream;
  if (st) {
    int dev = -1, sdev = -1;
    if (hipGetDevice(&dev) != hipSuccess || hipStreamGetDevice(st, &sdev) != hipSuccess) return DFLARE_ERR_HIP;
    if (dev != sdev) return DFLARE_ERR_INVALID_ARG;
  }
  char* w = static_cast<char*>(workspace);
  Lce a{};
  a.hidden = (const uint16_t*)hidden;
  a.head = (const uint16_t*)head;
  a.labels = labels;
  a.loss = loss;
  a.row_ce = row_ce;
  a.dhidden = (uint16_t*)dhidden;
  a.dhead = (uint16_t*)dhead;
  a.rows = rows;
  a.V = V;
  a.H = H;
  a.B = B;
  a.gamma = gamma;
  a.count = (int*)(w + L.count);
  a.src = (int*)(w + L.src);
  a.pos = (int*)(w + L.pos);
  a.word = (int*)(w + L.word);
  a.c = (float*)(w + L.c);
  a.lab = (float*)(w + L.lab);
  a.hc = (uint16_t*)(w + L.hc);
  a.part = (float2*)(w + L.part);
  a.zlab = (float*)(w + L.zlab);
  a.ref = (float*)(w + L.ref);
  a.sum = (float*)(w + L.sum);
  a.fac = (float*)(w + L.fac);
  a.dz = (uint16_t*)(w + L.dz);
  a.dacc = (float*)(w + L.dacc);
  a.Mp = L.Mp;
  a.ldh = L.ldh;
  a.stages = (std::min(V, L.Vp) + kBK - 1) / kBK;
  const int words = (int)((V + (long)kBlock - 1) / kBlock);
  const int pieces = (words + L.Vp / kBlock - 1) / (L.Vp / kBlock);
  const bool one_pass = dhead ? pieces == 1 : dhidden != nullptr;
  a.one_pass = one_pass;
  if (one_pass) {
    a.flag = (int*)(w + L.flag);
    if (dhead) a.hs = (size_t)L.Mp * L.ldh * 2 <= kScaledBytes ? (uint16_t*)(w + L.hs) : a.hc;
  }
  // The small tile wastes less where rows or tiles are few.  A round of its work-groups takes about 5/8 of a large
  // one's time (151,936 words x 4,096, logits, large / small: 125 rows 399 / 330 us, 180 403 / 435, 300 614 / 564, 500
  // 649 / 755; 32,003 x 2,880: 180 85 / 69, 300 85 / 101, 640 169 / 145, 900 185 / 218); for dh, whose words are
  // split into parts that fill the rounds, the rows' tiles alone count (4,096: 125 rows 327 / 258 us, 180 345 / 414,
  // 380 586 / 528, 640 901 / 817, 900 1,078 / 1,381).  dW is not faster on it (60 rows 363 / 373, 640 1,063 / 1,274).
  const int most = std::max(1, rows / B * (B - 1));  // rows with a loss, at most
  auto tiles = [](auto s, long m, long n) { return ((m + s.TM - 1) / s.TM) * ((n + s.TN - 1) / s.TN); };
  const long rounds_s = (tiles(Small{}, V, most) + 511) / 512, rounds_l = (tiles(Large{}, V, most) + 255) / 256;
  const bool z_small = 5 * rounds_s < 8 * rounds_l;
  const bool dh_small = 4 * tiles(Small{}, 1, most) < 7 * tiles(Large{}, 1, most) ||
               tiles(Large{}, H, most) * (a.stages / 4) < 256;  // (too few words for parts on all CUs)
  // Up to 64 rows the calls are bound by the head's way from memory, of which three work-groups to a CU keep more
  // under way (small tile / this: 13 rows of 151,936 x 2,880 with dh 423 / 357 us, 14 of 151,936 x 4,096 loss alone 287 / 232;
  // two of them for 120 rows lose: of 151,936 x 4,096 with dh 555 / 661).
  const bool few = most <= Few::TN;
  a.dh_tile = few ? 2 : dh_small;
  static_assert(Few::MT == Small::MT, "a wave's words");
  // dW of few tiles is split over its rows: the least time, in stages of 1.8 us, of rounds of work-groups, each with its
  // stages, 8 more for its start and its end, its labels' rows (added some 10 at a time), and of the parts' sum
  a.dw_parts = 1;
  if (dhead && one_pass) {
    const long t = tiles(Large{}, H, V), stages = (most + kBK - 1) / kBK, labels = (long)most * 64 / V;
    long best = LONG_MAX;
    for (long k = 1; k <= kMostParts && (k == 1 || (t * k <= 512 && stages >= 4 * k)); ++k) {
      const long cost = (t * k + 255) / 256 * ((stages + k - 1) / k + 8 + labels / (8 * k)) + (k > 1 ? 3 + (long)V * H * k / 1450000 : 0);
      if (cost < best) {
        best = cost;
        a.dw_parts = (int)k;
      }
    }
  }
  const int wave = z_small || few ? Small::MT * 32 : Large::MT * 32;
  auto grid = [](long tiles) { return (unsigned)((tiles + 7) / 8 * 8); };  // whole turns of the XCDs
  auto product = [&](bool small, auto mode, int v0, int nv, int piece) {
    constexpr int MODE = decltype(mode)::value;
    auto go = [&](auto s) {
      using S = decltype(s);
      long t = MODE <= kExp ? tiles(s, nv, most) : MODE == kDw ? tiles(s, H, nv) * a.dw_parts : tiles(s, H, most);
      if (MODE == kDh) t = std::max(t, std::min(kMostParts * t, 2l * dh_slots(a.dh_tile)));  // (the most that the plan makes)
      hipLaunchKernelGGL((k_lce_product<S, MODE>), dim3(grid(t)), dim3(S::T), 0, st, a, v0, nv, piece);
    };
    if constexpr (MODE != kDw) {
      if (few) return go(Few{});
      if (small) return go(Small{});
    }
    go(Large{});
  };
  // four rows a work-group keep more of them busy, 16 use whole lines of the parts (4 / 16: 207 rows of 32,003 x 264 62 / 64 us
  // the call, 701 of 201,088 the same, 7,296 of 151,936 57 / 25 the launch)
  auto by_rows = [&](auto go) {
    if (most <= 1024) go(mode_c<4>{});
    else go(mode_c<16>{});
  };
  hipLaunchKernelGGL(k_lce_rows, dim3(1), dim3(1024), 0, st, a, pieces);
  hipLaunchKernelGGL(k_lce_gather, dim3(L.Mp), dim3(256), 0, st, a);
  if (!one_pass) {  // in pieces whose parts have room
    const int most_words = (int)std::min<size_t>(words, L.part_bytes / ((size_t)L.Mp * 8) * wave / kBlock);
    const int turns = (words + most_words - 1) / most_words, step = (words + turns - 1) / turns * kBlock;
    for (int v0 = 0; v0 < V; v0 += step) {
      const int nv = std::min(V - v0, step);
      product(z_small, mode_c<kStats>{}, v0, nv, 0);
      by_rows([&](auto r) {
        hipLaunchKernelGGL((k_lce_lse<r.value>), dim3(L.Mp / r.value), dim3(1024), 0, st, a, (nv + wave - 1) / wave, v0 == 0, nv == V - v0);
      });
    }
  }
  if (dhidden || dhead)
    for (int piece = 0; piece < pieces; ++piece) {
      const int v0 = piece * L.Vp, nv = std::min(V - v0, L.Vp);
      if (one_pass) {
        product(z_small, mode_c<kExp>{}, v0, nv, piece);
        by_rows([&](auto r) {
          hipLaunchKernelGGL((k_lce_close<r.value>), dim3(L.Mp / r.value), dim3(1024), 0, st, a, nv, piece, piece == pieces - 1, wave);
        });
      } else {
        product(z_small, mode_c<kDz>{}, v0, nv, piece);
      }
      if (dhidden) product(dh_small, mode_c<kDh>{}, v0, nv, piece);
      if (dhead && !one_pass) product(false, mode_c<kDw>{}, v0, nv, piece);
    }
  if (dhidden) {
    // few values have many parts: 16 threads share their sum (207 rows x 264, 64 parts: 18 -> 7 us)
    const long values = (long)rows * (H / 8);
    auto go = [&](auto kernel, int g) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)((values * g + 255) / 256 + 1)), dim3(256), 0, st, a);
    };
    if (values <= 65536) go(k_lce_dhidden<16>, 16);
    else go(k_lce_dhidden<1>, 1);
  } else {
    hipLaunchKernelGGL(k_lce_loss, dim3(1), dim3(256), 0, st, a);
  }
  if (dhead && one_pass) {  // (in parts it takes the place of dh's sums)
    product(false, mode_c<kDw>{}, 0, V, 0);
    if (a.dw_parts > 1) hipLaunchKernelGGL(k_lce_dhead, dim3((unsigned)(((long)V * H / 8 + 255) / 256)), dim3(256), 0, st, a);
  }
  return hipGetLastError() == hipSuccess ? DFLARE_OK : DFLARE_ERR_HIP;
}

}  // extern "C"
