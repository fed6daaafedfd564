// Products of matrices on the bf16 matrix cores: tiles, their way from memory through LDS, and the loop over k that the LM head
// with its loss, the projections and the gated block share.
#pragma once

#include <limits.h>

#include "elements.h"

namespace dflare {

namespace {

constexpr int kBK = 64;     // k of a stage
// A product's output tile TM x TN and its WM x WN waves, each with MT x NT products of 32 x 32
template <int TM_, int TN_, int WM_, int WN_>
struct Shape {
  static constexpr int TM = TM_, TN = TN_, WM = WM_, WN = WN_, W = WM * WN, T = 64 * W;
  static constexpr int MT = TM / WM / 32, NT = TN / WN / 32;
  static constexpr int kABytes = TM * kBK * 2, kBBytes = TN * kBK * 2, kStageBytes = kABytes + kBBytes;
};
using Large = Shape<256, 256, 2, 4>;  // one work-group per CU
using Small = Shape<128, 128, 2, 2>;  // two
using Few = Shape<128, 64, 2, 2>;     // three

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                 0, 0);
}
__device__ __forceinline__ f32x4 unpack4(uint32_t a, uint32_t b) {
  return f32x4{__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u), __uint_as_float(b << 16),
               __uint_as_float(b & 0xFFFF0000u)};
}

// ---- products.  D[n][m] = sum over k of A[m, k] B[n, k] for a tile of m x n.  An operand lies in memory
// either with k along its rows (plain) or with k down its columns (across); both go to LDS as they lie, 16-byte
// pieces permuted by an xor so that the reads are free of bank conflicts, and the `across` ones are transposed
// by the LDS read (ds_read_b64_tr_b16):
//   plain   rows of 64 k, 128 bytes: piece c of row r at c ^ (r / 2 mod 8)
//   across  64 rows of as many columns as the tile: piece c of row k at c ^ 4 (k mod 4)
// m runs along A so that a lane holds, of one n (a token's row), 4 consecutive m at a time: sums over the words
// of a row stay within a lane. ----
struct Operand {
  const uint16_t* p;  // first element of the tile's rows (plain) or columns (across)
  long ld;
  int valid;  // rows (plain) or columns (across) of the tile that exist; past them the last is repeated
  int kend;   // k that exist (past them the stage's first again, to meet zeros of the other operand)
  // plain: 256 k lie side by side, the next 256 `block` bytes on (512: rows of any length); first stage
  long block = 512;
  int s0 = 0;
  // plain, in two parts: the rows of a tile are PART of p, then PART of `other` (of the same ld and valid), and so on in turn
  const uint16_t* other = nullptr;
};

// 1 KB from base + off (16 bytes per lane) to LDS, asynchronously.  In asm, and waited for by wait_vm_barrier: with the
// builtin the compiler waits for every such load before a transposing LDS read, which has a stage wait
// for the next one's data (dh 2.3 us a stage against 1.8).  m0 needs no saving: the compiler sets it before each
// use of its own.
__device__ __forceinline__ void load_lds(const char* base, uint32_t off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(off), "s"(base) : "memory");
}

// ROWS: rows (plain) or columns (across) of the operand's tile; W waves load it.  TURN: the whole stages of k are taken in
// turn from stage s0 on.  PART: rows of an operand's part, 0: whole
template <bool ACROSS, int ROWS, int W, bool TURN = false, int PART = 0>
struct Loader {
  static_assert(!ACROSS || ROWS % 128 == 0, "the pieces' permutation");
  static constexpr int N = ROWS * kBK * 2 / 1024 / W;  // loads of a wave and stage
  static constexpr int SB = 256 / kBK;                 // stages of a block of 256 k
  const char* at;   // of the next stage
  uint32_t off[N];  // byte offset of a lane's pieces
  long step;
  int st;
  const char* base;  // TURN: of stage 0
  int whole;
  __device__ __forceinline__ void init(const Operand& o, int w, int lane, int whole_) {
    st = o.s0;
    step = ACROSS ? o.ld * kBK * 2 : TURN ? kBK * 2 : o.block - (SB - 1) * kBK * 2;
    const uint16_t* p = o.p;
    if constexpr (PART > 0) {
      static_assert(!ACROSS && PART % (8 * N) == 0, "a wave loads rows of one part");
      if (N * w * 8 / PART & 1) p = o.other;
    }
    base = reinterpret_cast<const char*>(p);
    whole = whole_;
    if constexpr (TURN) at = base + st * step;
    else at = base + (ACROSS ? 0 : st / SB * o.block + st % SB * (kBK * 2));
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (!ACROSS) {
        const int row = (N * w + j) * 8 + (lane >> 3), c = (lane & 7) ^ ((row >> 1) & 7);
        int from = row;
        if constexpr (PART > 0) from = row / (2 * PART) * PART + row % PART;
        off[j] = (uint32_t)(min(from, o.valid - 1) * o.ld * 2 + c * 16);
      } else {
        constexpr int P = ROWS / 8;  // pieces of a row
        const int row = (N * w + j) * (64 / P) + lane / P, c = (lane % P) ^ ((row & 3) << 2);
        off[j] = (uint32_t)(row * o.ld * 2 + min(c * 8, o.valid - 8) * 2);
      }
    }
  }
  // the next stage has only `left` k: pieces past them take its first again (only before the last stage is loaded)
  __device__ __forceinline__ void cut(const Operand& o, int w, int lane, int left) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (!ACROSS) {
        const int row = (N * w + j) * 8 + (lane >> 3), c = (lane & 7) ^ ((row >> 1) & 7);
        if (c * 8 >= left) off[j] -= c * 16;
      } else {
        const int row = (N * w + j) * (512 / ROWS) + lane / (ROWS / 8);
        if (row >= left) off[j] -= (uint32_t)(row * o.ld * 2);
      }
    }
  }
  // the wave's share of the next stage
  __device__ __forceinline__ void issue(uint32_t dst) {
#pragma unroll
    for (int j = 0; j < N; ++j) load_lds(at, off[j], dst + j * 1024);
    if constexpr (TURN) {
      at += step;
      if (++st == whole) at = base;
    } else if constexpr (ACROSS) {
      at += step;
    } else {
      at += (++st % SB == 0) ? step : kBK * 2;
    }
  }
};

template <bool ACROSS, int ROWS>
struct Reader {
  uint32_t off[4];
  // tile0: first 32-row (or 32-column) tile of the wave
  __device__ __forceinline__ void init(int tile0, int lane) {
    const int h = lane >> 5;
    if constexpr (!ACROSS) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) off[ks] = (tile0 * 32 + (lane & 31)) * 128 + (((2 * ks + h) ^ ((lane >> 1) & 7)) << 4);
    } else {
      const int i = lane & 15, g = (lane >> 4) & 1, f = i >> 2;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        off[j] = (8 * h + f) * (ROWS * 2) + ((4 * ((tile0 + j) ^ f) + 2 * g + ((i & 3) >> 1)) << 4) + (i & 1) * 8;
    }
  }
  __device__ __forceinline__ u32x4 get(const char* op, int ks, int j) const {
    if constexpr (!ACROSS) return *reinterpret_cast<const u32x4*>(op + off[ks] + j * 4096);
    else {
      const char* p = op + off[j] + ks * 16 * (ROWS * 2);
      const u32x2 lo = tr(p), hi = tr(p + 4 * (ROWS * 2));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  }
  // the same for a ks that the compiler does not know
  __device__ __forceinline__ u32x4 at(const char* op, int ks, int j) const {
    if constexpr (!ACROSS) return *reinterpret_cast<const u32x4*>(op + (ks == 0 ? off[0] : ks == 1 ? off[1] : ks == 2 ? off[2] : off[3]) + j * 4096);
    else return get(op, ks, j);
  }
  static __device__ __forceinline__ u32x2 tr(const char* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDSP s16x4*)(LDSP char*)const_cast<char*>(p)));
  }
};

template <typename S>
using Acc = f32x16[S::MT][S::NT];
template <typename S>
__device__ __forceinline__ void clear(Acc<S>& acc) {
#pragma unroll
  for (int i = 0; i < S::MT; ++i)
#pragma unroll
    for (int j = 0; j < S::NT; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
}

// Two stages lie in LDS, one of them on its way; a wave reads the operands of each 16 k between the products of the 16
// before.  7,296 rows x 30,464 words x 4,096 (1,545 to 1,570 us with the epilogue, 1,170 TFLOP/s; dh of them 1,615 to 1,680): the matrix
// cores are busy 63% of the clocks, at 1.8 GHz; a library product of that shape takes 1,510 us (dh's 2,070).  The
// same with 4 waves of 128 x 128 has 13% more clocks at a higher rate of them and the same time, and so have
// work-groups that stay and load their next tile under the epilogue, 128 x 256 tiles two to a CU are 20% slower, and
// lines requested into L2 two stages ahead 6%: what is left lies outside the CUs, in the loads that miss L2 (2.3 TB/s).
// acc = A B^T over k in [0, K); K is rounded up to whole stages, of which operands past kend give zeros times
// something finite.  start(acc) runs while the first stages are on their way.
// MASK: acc += A B^T over k in [0, K) alone, kend of both operands being K; what lies past it takes no part (a stage that K
// ends in comes last, by itself, with both operands' k past the end set to zero).  The whole stages are taken in turn from s0 on,
// the same for both operands.
template <typename S, bool XA, bool XB, bool MASK = false, int PART = 0, typename F>
__device__ __forceinline__ void product(const Operand& oa, const Operand& ob, int K, char* lds, Acc<S>& acc, F&& start) {
  using LA = Loader<XA, S::TM, S::W, MASK, PART>;
  using LB = Loader<XB, S::TN, S::W, MASK>;
  constexpr int MT = S::MT, NT = S::NT, Q = MT * NT, R = MT + NT, SB = S::kStageBytes;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  LA la;
  LB lb;
  const int nk = (K + kBK - 1) / kBK, whole = MASK ? K / kBK : nk;
  la.init(oa, w, lane, whole);
  lb.init(ob, w, lane, whole);
  Reader<XA, S::TM> ra;
  Reader<XB, S::TN> rb;
  ra.init(w % S::WM * MT, lane);
  rb.init(w / S::WM * NT, lane);
  if constexpr (!MASK) clear<S>(acc);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(LDSP char*)lds);
  const uint32_t da = lds0 + w * LA::N * 1024, db = lds0 + S::kABytes + w * LB::N * 1024;
  int next = 0;  // stage to load; past the last stage nothing is
  auto issue_a = [&](uint32_t buf) {
    if (next >= nk) return;
    if (MASK && next == whole) la.at = la.base + whole * la.step;
    if (oa.kend - next * kBK < kBK) la.cut(oa, w, lane, oa.kend - next * kBK);
    la.issue(da + buf);
  };
  auto issue_b = [&](uint32_t buf) {
    if (next < nk) {
      if (MASK && next == whole) lb.at = lb.base + whole * lb.step;
      if (ob.kend - next * kBK < kBK) lb.cut(ob, w, lane, ob.kend - next * kBK);
      lb.issue(db + buf);
    }
    ++next;
  };
  struct Frags {
    u32x4 a[MT], b[NT];
  };
  auto read = [&](Frags& f, uint32_t buf, int ks, int n) {  // in the order in which the products take them
    if (n == 0 || n > MT) f.b[n == 0 ? 0 : n - MT] = rb.get(lds + S::kABytes + buf, ks, n == 0 ? 0 : n - MT);
    else f.a[n - 1] = ra.get(lds + buf, ks, n - 1);
  };
  auto multiply = [&](const Frags& f, int n) { acc[n % MT][n / MT] = mfma32(f.a[n % MT], f.b[n / MT], acc[n % MT][n / MT]); };
  auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
  // Q products, beside them the R reads for the next Q
  auto step = [&](const Frags& f, Frags& g, uint32_t buf, int ks) {
#pragma unroll
    for (int n = 0; n < Q; ++n) {
      multiply(f, n);
#pragma unroll
      for (int r = n * R / Q; r < (n + 1) * R / Q; ++r) read(g, buf, ks, r);
      fence();
    }
  };
  issue_a(0);
  issue_b(0);
  issue_a(SB);
  issue_b(SB);
  start(acc);
  wait_vm_barrier<0>();
  Frags f0, f1;
#pragma unroll
  for (int n = 0; n < R; ++n) read(f0, 0, 0, n);
  uint32_t buf = 0;
  bool late = false;  // the second operand's share of the stage after the next is still to be issued
  for (int kt = 0; kt < whole; ++kt) {
    const uint32_t other = SB - buf;
    fence();
#pragma unroll
    for (int n = 0; n < Q; ++n) {
      multiply(f0, n);
#pragma unroll
      for (int r = n * R / Q; r < (n + 1) * R / Q; ++r) read(f1, buf, 1, r);
      if (n == (Q > 4 ? Q / 4 - 1 : 0) && late) issue_b(other);
      fence();
    }
    step(f1, f0, buf, 2);
    step(f0, f1, buf, 3);
    // in the midst of the stage's last products: the next stage is here, and all waves have read this one, whose
    // buffer takes the one after the next (after a quarter of them on the large tile: at 8,192 rows, by turns, 0.2 to 3.4% faster than after half)
    constexpr int B = MASK && Q > 4 ? Q / 4 : Q / 2;
#pragma unroll
    for (int n = 0; n < Q; ++n) {
      if (n == B) wait_vm_barrier<0>();
      multiply(f1, n);
      if (n >= B) {
#pragma unroll
        for (int r = (n - B) * R / (Q - B); r < (n + 1 - B) * R / (Q - B); ++r) read(f0, other, 0, r);
        if (n == B + (Q > 4)) issue_a(buf);
      }
      fence();
    }
    late = true;
    buf = other;
  }
  if constexpr (MASK) {
    if (whole < nk) {
      const int left = K - whole * kBK, h = lane >> 5;
#pragma unroll 1
      for (int ks = 0; ks * 16 < left; ++ks) {
        const int n = left - ks * 16 - 8 * h;  // of a lane's 8 k those below n are there
        u32x4 keep;
#pragma unroll
        for (int e = 0; e < 4; ++e) keep[e] = 2 * e + 1 < n ? ~0u : 2 * e < n ? 0xFFFFu : 0u;
        u32x4 a[MT], b[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) a[i] = ra.at(lds + buf, ks, i) & keep;
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = rb.at(lds + S::kABytes + buf, ks, j) & keep;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = mfma32(a[i], b[j], acc[i][j]);
      }
    }
  }
  wait_vm_barrier<0>();
}

// Output tile t of TA x TB, so that the work-groups that run together on an XCD (ids are dealt to the 8 XCDs
// in turn) share operand tiles in its L2: an XCD takes a contiguous part of the tiles, in groups of 4 A tiles by
// all B tiles.  false past the last tile.
__device__ __forceinline__ bool tile_of(int id, int TA, int TB, int& ta, int& tb) {
  const int total = TA * TB, per = (total + 7) / 8;
  const int t = id % 8 * per + id / 8;
  if (id / 8 >= per || t >= total) return false;
  const int g = t / (4 * TB), w = min(4, TA - 4 * g), r = t - g * 4 * TB;
  ta = 4 * g + r % w;
  tb = r / w;
  return true;
}

// The tile as bf16 in LDS, TM m (in 16-byte pieces) by TN n: piece p of row n at p ^ (n mod the pieces)
template <typename S>
__device__ __forceinline__ void put_tile(char* lds, const Acc<S>& acc, int j, int n, int m_tile0, int h) {
  constexpr int P = S::TM / 8;
#pragma unroll
  for (int t = 0; t < S::MT; ++t)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x16& z = acc[t][j];
      const int p = m_tile0 * 4 + t * 4 + q;
      const uint2 v = make_uint2(pack2(z[4 * q], z[4 * q + 1]), pack2(z[4 * q + 2], z[4 * q + 3]));
      *reinterpret_cast<uint2*>(lds + n * (S::TM * 2) + ((p ^ (n & (P - 1))) << 4) + h * 8) = v;
    }
}
// and from there to rows of `to` (of which rows n < nv and columns m < mv exist; mv a multiple of 8)
template <typename S>
__device__ __forceinline__ void store_tile(const char* lds, uint16_t* to, long ld, int nv, int mv) {
  constexpr int P = S::TM / 8, RW = S::TN / S::W;  // pieces of a row, rows of a wave
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll 4
  for (int it = 0; it < RW * P / 64; ++it) {
    const int n = w * RW + it * (64 / P) + lane / P, p = lane % P;
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + n * (S::TM * 2) + ((p ^ (n & (P - 1))) << 4));
    if (n < nv && p * 8 < mv) *reinterpret_cast<u32x4*>(to + n * ld + p * 8) = v;
  }
}

}  // namespace

}  // namespace dflare
