// The AdamW step over many tensors (Loshchilov and Hutter, "Decoupled weight decay regularization", 2019) and its C-ABI entry
// point.  With the clipped gradient g, decoupled decay w and step t:
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr w) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
// Clipping takes place here, by the gradients' sum of squares, so that no pass of its own reads and writes them.
// States in 8 bits: m and sqrt(v) as e4m3 numbers times a scale for each 256 values of a tensor, its largest over 448.  The
// root, because e4m3 then covers 2^36 of v instead of 2^18; what is above zero stays above zero, so that no step divides a
// remembered m by eps alone.
// Bound by memory: 28 bytes a value (bf16 with an fp32 master and fp32 states): 402 M values 2,290 us, 4.9 TB/s, a copy's rate on this
// card; 10 in 8 bits without a master: 885 us, 4.6 TB/s.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <type_traits>
#include <vector>

#include "dflare.h"
#include "elements.h"

namespace dflare {

namespace {

constexpr int kValues = 8;             // of a thread: a lane's share of a block of 256 is 1/32
constexpr int kChunk = kT * kValues;   // values of a work-group's turn
constexpr int kScaled = 256;           // values that share a scale
constexpr int kGroups = 2048;          // work-groups of a launch, at most
constexpr float kMost = 448.f, kLeast = 0.001953125f;  // of e4m3: largest, smallest above zero (2^-9)
constexpr float kPerMost = 1.f / kMost;
constexpr float kLeastScale = 1.2621774483536189e-29f;  // 2^-96: scales and their inverses stay inside fp32

struct Hyper {
  float decay, alpha, root;  // lr w, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  float b1, c1, b2, c2, eps; // c: 1 - b
};
struct Options {
  double lr, weight_decay, ln1, ln2;  // logarithms of b1, b2
  const double* lr_device;
  const int64_t* step_device;
  const double* sumsq;
  int64_t step;
  float max_norm;
  Hyper h;
};
__host__ __device__ inline void set_step(Hyper& h, double lr, double weight_decay, double ln1, double ln2, double t) {
  h.decay = (float)(lr * weight_decay);
  h.alpha = (float)(lr / (1.0 - exp(t * ln1)));
  h.root = (float)(1.0 / sqrt(1.0 - exp(t * ln2)));
}

// The tensors of a launch, as many as its arguments (4 KB) hold beside the options: 87 with masters and scales.  A tensor's addresses are
// distances of 40 bits from those of the launch's first tensor less 2^39.  The arguments come from far, and every access that
// waits for another one costs a microsecond, so a record is read as a whole, and the first chunks by a lane each (301 tensors, 8 bits: four
// launches of 7-9 us; as 57 records of whole addresses six, and with a binary search over arrays of fields six of 9).
constexpr long kReach = 1l << 39;
template <bool MASTER, bool BYTE>
struct Tab {
  static constexpr int K = 4 + MASTER + 2 * BYTE;  // parameter, gradient, m, v; master; scales
  static constexpr int N = 3840 / (4 * K + 16);
  struct Record {
    uint32_t lo[K];
    uint32_t hi[2];  // bits from 32 on of address k in byte k; byte 7: 1: fp32 parameter; 2: fp32 gradient; 4: a master; the high bits of n above
    uint32_t n;      // values, the low 32 bits
  };
  uint64_t base[K];
  Record r[N];
  int first[N + 1];  // chunks before the tensor
  int count;
};
static_assert(sizeof(Tab<true, true>) + sizeof(Options) <= 4088 && sizeof(Tab<false, false>) + sizeof(Options) <= 4088, "kernel arguments");
// a tensor of it
template <bool MASTER, bool BYTE>
struct Tensor {
  void *p, *m, *v;
  const void* g;
  float *w, *ms, *vs;
  long n;
  int tag;
  __device__ __forceinline__ Tensor(const Tab<MASTER, BYTE>& t, int i) {
    const auto r = t.r[i];
    auto address = [&](int k) {
      return (void*)(t.base[k] + ((uint64_t)((r.hi[k / 4] >> (8 * (k % 4))) & 255u) << 32 | r.lo[k]));
    };
    p = address(0);
    g = address(1);
    m = address(2);
    v = address(3);
    w = MASTER ? (float*)address(4) : nullptr;
    ms = BYTE ? (float*)address(4 + MASTER) : nullptr;
    vs = BYTE ? (float*)address(5 + MASTER) : nullptr;
    tag = (int)(r.hi[1] >> 24);
    n = (long)r.n | (long)(tag >> 3) << 32;
  }
};

// 8 values at any element
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  float a[4], b[4];
  load_n<float, 4, false>(p, a);
  load_n<float, 4, false>(p + 4, b);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&x)[8]) { load_n<bf16_t, 8, false>(p, x); }
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
  store_n<float, 4, false>(p, a);
  store_n<float, 4, false>(p + 4, b);
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8]) { store_n<bf16_t, 8, false>(p, x); }
struct e4m3_t {
  uint8_t b;
};
struct __attribute__((packed, aligned(1))) Bytes8 {
  u32x2 v;
};
__device__ __forceinline__ void unpack8(u32x2 w, float (&x)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
    x[4 * k] = lo[0];
    x[4 * k + 1] = lo[1];
    x[4 * k + 2] = hi[0];
    x[4 * k + 3] = hi[1];
  }
}
__device__ __forceinline__ u32x2 pack8(const float (&x)[8]) {  // nearest even
  u32x2 w;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * k], x[4 * k + 1], 0, false);
    w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * k + 2], x[4 * k + 3], r, true);
  }
  return w;
}
__device__ __forceinline__ void load8(const e4m3_t* p, float (&x)[8]) { unpack8(reinterpret_cast<const Bytes8*>(p)->v, x); }
__device__ __forceinline__ void store8(e4m3_t* p, const float (&x)[8]) { reinterpret_cast<Bytes8*>(p)->v = pack8(x); }

// `left` values at p, 0 to 8; zeros past them
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int left, float (&x)[8]) {
  if (left >= 8) return load8(p, x);
  if constexpr (std::is_same_v<T, e4m3_t>) {
    u32x2 w = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) w[e / 4] |= (uint32_t)p[e].b << (e % 4 * 8);
    unpack8(w, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < left ? to_f(p[e]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, int left, const float (&x)[8]) {
  if (left >= 8) return store8(p, x);
  if constexpr (std::is_same_v<T, e4m3_t>) {
    const u32x2 w = pack8(x);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e].b = (uint8_t)(w[e / 4] >> (e % 4 * 8));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = from_f<T>(x[e]);
  }
}

// x over the scale of its 256 values, which 32 lanes hold, and the scale.  A NaN among them is their largest, and so all 256 are NaN, as
// the formula has it.  ROOT: what is above zero stays at least the smallest number above zero
template <bool ROOT>
__device__ __forceinline__ float to_scale(float (&x)[8]) {
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = __builtin_elementwise_maximum(most, fabsf(x[e]));
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) most = __builtin_elementwise_maximum(most, __shfl_xor(most, off));
  const float scale = __builtin_elementwise_maximum(most * kPerMost, kLeastScale), inv = 1.f / scale;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float q = x[e] * inv;
    if (scale < INFINITY) q = fmaf(fmaf(-q, scale, x[e]), inv, q);  // the quotient, correctly rounded
    x[e] = ROOT && x[e] > 0.f && q < kLeast ? kLeast : q;
  }
  return scale;
}

// The card's roots take numbers below 2^-126 for zero: a v below 2^-90 (a gradient below 1e-13) is multiplied by 2^64 first, its root by 2^-32
struct Scaled {
  float v, back;
  __device__ __forceinline__ explicit Scaled(float x) {
    const bool small = x < 0x1p-90f;
    v = small ? x * 0x1p64f : x;
    back = small ? 0x1p-32f : 1.f;
  }
};
// The root, correctly rounded: an estimate y of 1 / sqrt(v), then both v y and y / 2 corrected by
// 1/2 - (y / 2) (v y), and the root by its remainder (Markstein, "IA-64 and elementary functions", 2000)
__device__ __forceinline__ float root_of(float v) {
  const Scaled s(v);
  const float y = __builtin_amdgcn_rsqf(s.v);
  float g = s.v * y, h = 0.5f * y;
  const float e = fmaf(-h, g, 0.5f);
  g = fmaf(g, e, g);
  h = fmaf(h, e, h);
  g = fmaf(fmaf(-g, g, s.v), h, g);
  return v > 0.f && v < INFINITY ? g * s.back : v;  // (a NaN is itself)
}
__device__ __forceinline__ float near_root_of(float v) {  // to a unit in the last place
  const Scaled s(v);
  return __builtin_amdgcn_sqrtf(s.v) * s.back;
}

template <bool MASTER, bool BYTE, typename P, typename G>
__device__ __forceinline__ void chunk(const Tensor<MASTER, BYTE>& t, int c, const Hyper& h, Factor f) {
  using S = std::conditional_t<BYTE, e4m3_t, float>;
  const long at = (long)c * kChunk + threadIdx.x * kValues;
  const int left = (int)max(min(t.n - at, 8l), 0l);
  if (!BYTE && left == 0) return;
  float p[8], g[8], m[8], v[8];
  P* param = (P*)t.p + at;
  S *pm = (S*)t.m + at, *pv = (S*)t.v + at;
  float* master = MASTER && (t.tag & 4) ? t.w + at : nullptr;
  load_some((const G*)t.g + at, left, g);
  load_some(pm, left, m);
  load_some(pv, left, v);
  if (master) load_some((const float*)master, left, p);
  else load_some((const P*)param, left, p);
  float *sm = nullptr, *sv = nullptr;
  if constexpr (BYTE) {
    if (left > 0) {
      sm = t.ms + at / kScaled;
      sv = t.vs + at / kScaled;
      const float a = *sm, b = *sv;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] *= a;
        v[e] *= b;
        v[e] *= v[e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = f.of(g[e]);
    float r;
    if constexpr (BYTE) {
      // Every operation rounded by itself: a number that lies next to a border between two of e4m3 falls to one side of it by the formula,
      // not by how a compiler forms it, and a state can be reproduced from its inputs bit by bit
#pragma clang fp contract(off)
      m[e] = h.b1 * m[e] + h.c1 * x;
      v[e] = h.b2 * v[e] + h.c2 * (x * x);
      r = root_of(v[e]);
    } else {
      m[e] = fmaf(h.c1, x, h.b1 * m[e]);
      v[e] = fmaf(h.c2 * x, x, h.b2 * v[e]);
      r = near_root_of(v[e]);  // (to a unit in the last place, as the reciprocal)
    }
    // Decay and update are taken off together, and p is rounded once: 1 - lr w in fp32 is a multiple of 2^-24, 19% off at lr w = 1e-7 and no
    // decay below 3e-8, step after step to the same side.  (An infinite p stays what it is.)
    const float kept = fabsf(p[e]) < INFINITY ? p[e] : 0.f;
    p[e] -= fmaf(h.decay, kept, h.alpha * (m[e] * __builtin_amdgcn_rcpf(fmaf(r, h.root, h.eps))));
    if constexpr (BYTE) v[e] = r;
  }
  if constexpr (BYTE) {
    const float a = to_scale<false>(m), b = to_scale<true>(v);
    if (left > 0 && threadIdx.x % 32 == 0) {
      *sm = a;
      *sv = b;
    }
  }
  store_some(pm, left, m);
  store_some(pv, left, v);
  store_some(param, left, p);
  if (master) store_some(master, left, p);
}

template <bool MASTER, bool BYTE>
__global__ __launch_bounds__(kT) void k_adamw(Tab<MASTER, BYTE> tab, Options o) {
  const int total = tab.first[tab.count];
  int c = (int)((long)total * blockIdx.x / gridDim.x);
  const int end = (int)((long)total * (blockIdx.x + 1) / gridDim.x);
  if (c >= end) return;
  const double sumsq = o.sumsq ? o.sumsq[0] : 0.0;  // (on its way beside the table)
  // the last tensor whose first chunk is not after c
  int at = -1;
  for (int k = 0; k < tab.count; k += 64) {
    const int i = k + (int)(threadIdx.x & 63);
    at += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < tab.count && tab.first[min(i, tab.count)] <= c));
  }
  Hyper h = o.h;
  if (o.lr_device || o.step_device) {
    const double lr = o.lr_device ? *o.lr_device : o.lr;
    const int64_t step = o.step_device ? *o.step_device : o.step;
    if (!(lr >= 0.0 && lr < (double)INFINITY) || step < 1) return;  // the host refuses such numbers: the step is left out
    set_step(h, lr, o.weight_decay, o.ln1, o.ln2, (double)step);
  }
  Factor f{1.f, 0};
  if (o.sumsq) {
    const double norm = sqrt(sumsq);
    if (!(norm < (double)INFINITY)) return;  // not finite: the step is left out
    if (norm > (double)o.max_norm) f.m = (float)frexp((double)o.max_norm / norm, &f.e);
  }
  while (true) {
    const Tensor<MASTER, BYTE> t(tab, at);
    const int first = tab.first[at], stop = min(tab.first[at + 1], end);
    auto walk = [&](auto p, auto g) {
      for (; c < stop; ++c) chunk<MASTER, BYTE, decltype(p), decltype(g)>(t, c - first, h, f);
    };
    switch (t.tag & 3) {
      case 0: walk(bf16_t{}, bf16_t{}); break;
      case 1: walk(float{}, bf16_t{}); break;
      case 2: walk(bf16_t{}, float{}); break;
      default: walk(float{}, float{});
    }
    if (c >= end) return;
    ++at;
  }
}

// ---- host side ----

int check(const dflare_adamw_tensor* t, int n, const dflare_adamw_options& o) {
  if (n < 0 || (n > 0 && !t)) return DFLARE_ERR_INVALID_ARG;
  if (!(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0)) return DFLARE_ERR_INVALID_ARG;
  if (!((float)o.eps >= FLT_MIN) || !isfinite((float)o.eps) || !(o.weight_decay >= 0.0) || !isfinite(o.weight_decay)) return DFLARE_ERR_INVALID_ARG;
  if (!o.lr_device && (!(o.lr >= 0.0) || !isfinite(o.lr))) return DFLARE_ERR_INVALID_ARG;
  if (!o.step_device && o.step < 1) return DFLARE_ERR_INVALID_ARG;
  if (misplaced(o.lr_device, 8) || misplaced(o.step_device, 8) || misplaced(o.sumsq, 8)) return DFLARE_ERR_INVALID_ARG;
  if (o.sumsq && !(o.max_norm >= 0.f)) return DFLARE_ERR_INVALID_ARG;
  if (o.state_bits != 8 && o.state_bits != 32) return DFLARE_ERR_INVALID_ARG;
  const bool byte = o.state_bits == 8;
  for (int i = 0; i < n; ++i) {
    const dflare_adamw_tensor& x = t[i];
    const int ps = size_of(x.param_dtype), gs = size_of(x.grad_dtype);
    if (!ps || !gs || x.n < 0 || (x.master && x.param_dtype != DFLARE_BF16)) return DFLARE_ERR_INVALID_ARG;
    if (x.n > 0 && (!x.param || !x.grad || !x.m || !x.v || (byte && (!x.m_scale || !x.v_scale)))) return DFLARE_ERR_INVALID_ARG;
    if (misplaced(x.param, ps) || misplaced(x.grad, gs) || misplaced(x.master, 4)) return DFLARE_ERR_INVALID_ARG;
    if (byte ? misplaced(x.m_scale, 4) || misplaced(x.v_scale, 4) : misplaced(x.m, 4) || misplaced(x.v, 4)) return DFLARE_ERR_INVALID_ARG;
    if (x.n > (1ll << 36)) return DFLARE_ERR_UNSUPPORTED;
  }
  return DFLARE_OK;
}

// INVALID_ARG where what is written (parameters, masters, states) overlaps anything else.  The lists of a call are mostly in the
// order of their addresses: a list is cut into ascending runs, and where these are few and lie apart as wholes (views of
// flat buffers), that is all; otherwise everything is sorted.
int all_apart(const dflare_adamw_tensor* t, int n, const dflare_adamw_options& o) try {
  struct Span {
    uintptr_t a, b;
    bool out;
  };
  const bool byte = o.state_bits == 8;
  const size_t state = byte ? 1 : 4;
  // f(address, bytes, written) for every tensor, list by list
  auto each = [&](auto f) {
    f(o.lr_device, 8, false);
    f(o.step_device, 8, false);
    f(o.sumsq, 8, false);
    for (int i = 0; i < n; ++i) f(t[i].param, (size_t)t[i].n * size_of(t[i].param_dtype), true);
    for (int i = 0; i < n; ++i) f(t[i].grad, (size_t)t[i].n * size_of(t[i].grad_dtype), false);
    for (int i = 0; i < n; ++i) f(t[i].master, (size_t)t[i].n * 4, true);
    for (int i = 0; i < n; ++i) f(t[i].m, (size_t)t[i].n * state, true);
    for (int i = 0; i < n; ++i) f(t[i].v, (size_t)t[i].n * state, true);
    if (!byte) return;
    for (int i = 0; i < n; ++i) f(t[i].m_scale, ((size_t)t[i].n + kScaled - 1) / kScaled * 4, true);
    for (int i = 0; i < n; ++i) f(t[i].v_scale, ((size_t)t[i].n + kScaled - 1) / kScaled * 4, true);
  };
  auto before = [](const Span& x, const Span& y) { return x.a < y.a; };
  auto clear = [](const Span* s, const Span* end) {
    uintptr_t end_out = 0, end_any = 0;
    for (; s != end; ++s) {
      if (s->a < end_out || (s->out && s->a < end_any)) return false;
      end_any = std::max(end_any, s->b);
      if (s->out) end_out = std::max(end_out, s->b);
    }
    return true;
  };
  constexpr int RUNS = 48;
  Span runs[RUNS];
  int count = 0;
  bool few = true;
  each([&](const void* p, size_t bytes, bool out) {
    const uintptr_t a = (uintptr_t)p;
    if (!p || !bytes || !few) return;
    if (count && runs[count - 1].out == out && a >= runs[count - 1].b) {
      runs[count - 1].b = a + bytes;
    } else if (count < RUNS) {
      runs[count++] = Span{a, a + bytes, out};
    } else {
      few = false;
    }
  });
  if (few) {
    std::sort(runs, runs + count, before);
    if (clear(runs, runs + count)) return DFLARE_OK;
  }
  std::vector<Span> all;
  all.reserve(7 * (size_t)n + 3);
  each([&](const void* p, size_t bytes, bool out) {
    if (p && bytes) all.push_back({(uintptr_t)p, (uintptr_t)p + bytes, out});
  });
  std::sort(all.begin(), all.end(), before);
  return clear(all.data(), all.data() + all.size()) ? DFLARE_OK : DFLARE_ERR_INVALID_ARG;
} catch (const std::bad_alloc&) {
  return DFLARE_ERR_OUT_OF_MEMORY;
}

template <bool MASTER, bool BYTE>
void launch(const dflare_adamw_tensor* t, int n, const Options& o, hipStream_t st) {
  using T = Tab<MASTER, BYTE>;
  T tab;
  tab.count = 0;
  tab.first[0] = 0;
  auto flush = [&] {
    if (tab.count) hipLaunchKernelGGL((k_adamw<MASTER, BYTE>), dim3(std::min(tab.first[tab.count], kGroups)), dim3(kT), 0, st, tab, o);
    tab.count = 0;
  };
  for (int i = 0; i < n; ++i) {
    const dflare_adamw_tensor& x = t[i];
    if (!x.n) continue;
    uint64_t at[7] = {(uint64_t)x.param, (uint64_t)x.grad, (uint64_t)x.m, (uint64_t)x.v};
    if (MASTER) at[4] = (uint64_t)x.master;
    if (BYTE) {
      at[4 + MASTER] = (uint64_t)x.m_scale;
      at[5 + MASTER] = (uint64_t)x.v_scale;
    }
    const long chunks = (x.n + kChunk - 1) / kChunk;
    bool fits = tab.count < T::N && (!tab.count || tab.first[tab.count] + chunks <= (1l << 30));
    for (int k = 0; tab.count && k < T::K; ++k) {
      if (MASTER && k == 4 && !x.master) continue;  // (its address is not read)
      fits = fits && at[k] - tab.base[k] < (uint64_t)(2 * kReach);
    }
    if (!fits) flush();
    if (!tab.count)
      for (int k = 0; k < T::K; ++k) tab.base[k] = at[k] - kReach;
    const int j = tab.count++;
    typename T::Record& r = tab.r[j];
    r.hi[0] = 0;
    r.hi[1] = (uint32_t)((x.param_dtype == DFLARE_F32) | (x.grad_dtype == DFLARE_F32) << 1 | (x.master != nullptr) << 2 | (x.n >> 32) << 3) << 24;
    for (int k = 0; k < T::K; ++k) {
      const uint64_t far = at[k] - tab.base[k];
      r.lo[k] = (uint32_t)far;
      r.hi[k / 4] |= (uint32_t)((far >> 32) & 255u) << (8 * (k % 4));
    }
    r.n = (uint32_t)x.n;
    tab.first[j + 1] = tab.first[j] + (int)chunks;
  }
  flush();
}

}  // namespace

}  // namespace dflare

using namespace dflare;

extern "C" {

int dflare_adamw(const dflare_adamw_tensor* tensors, int32_t n, const dflare_adamw_options* options, void* stream) {
  if (!options) return DFLARE_ERR_INVALID_ARG;
  const dflare_adamw_options& o = *options;
  int rc = check(tensors, n, o);
  if (rc != DFLARE_OK) return rc;
  if ((rc = all_apart(tensors, n, o)) != DFLARE_OK) return rc;
  if ((rc = stream_ok(stream)) != DFLARE_OK) return rc;
  Options k{};
  k.lr = o.lr;
  k.weight_decay = o.weight_decay;
  k.ln1 = log(o.beta1);
  k.ln2 = log(o.beta2);
  k.lr_device = o.lr_device;
  k.step_device = o.step_device;
  k.sumsq = o.sumsq;
  k.step = o.step;
  k.max_norm = o.max_norm;
  k.h.b1 = (float)o.beta1;
  k.h.c1 = (float)(1.0 - o.beta1);
  k.h.b2 = (float)o.beta2;
  k.h.c2 = (float)(1.0 - o.beta2);
  k.h.eps = (float)o.eps;
  if (!o.lr_device && !o.step_device) set_step(k.h, o.lr, o.weight_decay, k.ln1, k.ln2, (double)o.step);
  bool master = false;
  for (int i = 0; i < n; ++i) master |= tensors[i].master && tensors[i].n > 0;
  const hipStream_t st = (hipStream_t)stream;
  if (o.state_bits == 8) {
    if (master) launch<true, true>(tensors, n, k, st);
    else launch<false, true>(tensors, n, k, st);
  } else {
    if (master) launch<true, false>(tensors, n, k, st);
    else launch<false, false>(tensors, n, k, st);
  }
  return launched();
}

}  // extern "C"
