// gfx950 kernels of the stand-alone operators: a matrix product with bias,
// activation and residual in its epilogue, the routing of rows to experts,
// and the routed experts' SwiGLU products.
//
// Arithmetic (independent of the number of rows and of the kernel that runs,
// so a row's result never depends on the other rows of a call):
//   * every product element is one fp32 accumulator that takes the reduction's
//     super-steps (32 columns in bf16, 16 in fp32: one fragment) in order; a
//     linear sums several such chains, in order, their number a function of
//     the reduction's length (linear_chains) or, for at most NARROW outputs (a
//     router), eight; the experts' in fp32 are chains of EXPERT_CHAIN super-steps
//     (their results pass through two products: with one chain each over 7168
//     columns they are 2.3e-6 off, with these 5e-7; in bf16 the rounding of z
//     hides it, and one chain it is);
//   * an experts' row is sum_j fma(w_j, y_j) over its slots in order, in fp32.

#include "operators.h"

#include <float.h>
#include <math.h>

#include <algorithm>

#include "device.h"

namespace ee {

// Bytes of a row that one super-step covers: 32 bf16 or 16 fp32 values, 16
// bytes per lane group.
constexpr int STEP = 64;
constexpr int EXPERT_CHAIN = 16;

// acc[n][m] += (16 features of wp[n]) x (16 rows of xp[m]) over S super-steps.  wp and
// xp point to the lane's own 16 bytes of step 0.  D steps are in flight: a step's
// registers are requested again as soon as it is multiplied.  Bound by the bytes
// in flight (a wave's share of the weights is one chain: nothing else may be
// multiplied meanwhile), so D is what the registers hold; whole turns of D
// have no branch between their steps, where the compiler would wait for more
// than the step needs (one decoded token through 8 experts, 2048 x 768: 25 us
// with a test per step and two alternating sets of 8, 13 us).  FOLD: every D steps
// are a chain of their own, the chains added in order.  EVERY > 1: the steps are two
// by two of every EVERY-th pair.
typedef const __attribute__((address_space(1))) unsigned char global_bytes;
typedef const __attribute__((address_space(1))) u32x4 global_u32x4;
template <int DT, int NT, int MT, int D, bool FOLD = false, int EVERY = 1>
__device__ __forceinline__ void chain(const unsigned char* const (&wptr)[NT], const unsigned char* const (&xptr)[MT], int S,
                                      f32x4 (&acc)[NT][MT]) {
  // (global pointers by type: through the loop the compiler loses that they
  // are, and a flat load's wait drains all of them)
  global_bytes *wp[NT], *xp[MT];
#pragma unroll
  for (int n = 0; n < NT; ++n) wp[n] = (global_bytes*)wptr[n];
#pragma unroll
  for (int m = 0; m < MT; ++m) xp[m] = (global_bytes*)xptr[m];
  static_assert(EVERY == 1 || D % 2 == 0, "whole pairs");
  constexpr int PAIR = 2 * STEP * EVERY;
  auto at = [](int i) { return EVERY == 1 ? i * STEP : i / 2 * PAIR + i % 2 * STEP; };
  uint4 w[D][NT], x[D][MT];
  auto load = [&](int i) {
#pragma unroll
    for (int n = 0; n < NT; ++n) w[i][n] = __builtin_bit_cast(uint4, *(global_u32x4*)(wp[n] + at(i)));
#pragma unroll
    for (int m = 0; m < MT; ++m) x[i][m] = __builtin_bit_cast(uint4, *(global_u32x4*)(xp[m] + at(i)));
    __builtin_amdgcn_sched_barrier(0);   // (requests in the order of their use: a wait then leaves the later ones out)
  };
  auto mul = [&](int i) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[n][m] = mma<DT>(w[i][n], x[i][m], acc[n][m]);
  };
  auto next = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) wp[n] += at(D);
#pragma unroll
    for (int m = 0; m < MT; ++m) xp[m] += at(D);
  };
  f32x4 tot[NT][MT];
  auto fold = [&](bool first) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        tot[n][m] = first ? f32x4{0.f, 0.f, 0.f, 0.f} + acc[n][m] : tot[n][m] + acc[n][m];
        acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
  };
  const int turns = S / D, rest = S % D;
  if (turns) {
#pragma unroll
    for (int i = 0; i < D; ++i) load(i);
    next();
    for (int g = 1; g < turns; ++g) {
#pragma unroll
      for (int i = 0; i < D; ++i) {
        mul(i);
        load(i);
      }
      if constexpr (FOLD) fold(g == 1);
      next();
    }
#pragma unroll
    for (int i = 0; i < D; ++i) {
      mul(i);
      if (i < rest) load(i);
    }
    if constexpr (FOLD)
      if (rest) fold(turns == 1);
  } else {
#pragma unroll
    for (int i = 0; i < D; ++i)
      if (i < rest) load(i);
  }
#pragma unroll
  for (int i = 0; i < D; ++i)
    if (i < rest) mul(i);
  if constexpr (FOLD)
    if (S > D) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[n][m] = tot[n][m] + acc[n][m];
    }
}

// Four consecutive values, rounded to the type, from an aligned element index.
template <int DT> __device__ __forceinline__ void store4(void* base, size_t i, f32x4 v) {
  if constexpr (DT == DT_BF16)
    *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(base) + i) =
        make_uint2(bf16x2_bits(v[0], v[1]), bf16x2_bits(v[2], v[3]));
  else
    *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(base) + i) = v;
}

// 1 / (1 + e^-v) on the hardware's exp2 and reciprocal.  The exponent's product is
// rounded once (|v| log2(e) 2^-24 of e^-v), so the result is off by at most a few
// 2^-24 where it matters (|v| e^-v / (1 + e^-v) < 0.3) and its product with v by a
// few 2^-24 |v| everywhere.  (expf and a division: the activation of an 8192 x
// 11008 output took 110 us, now 16.)
__device__ __forceinline__ float logistic(float v) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v));
}
__device__ __forceinline__ float silu(float v) { return v * logistic(v); }

__device__ __forceinline__ float activate(float v, int act) {
  switch (act) {
    case ACT_SILU: return silu(v);
    case ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
    case ACT_GELU_TANH: return v * logistic(1.5957691216057308f * (v + 0.044715f * v * v * v));
    case ACT_RELU: return v < 0.0f ? 0.0f : v;   // (NaN stays NaN)
    default: return v;
  }
}

// ----------------------------------------------------------------- epilogues --

__device__ __forceinline__ f32x4 activate4(f32x4 v, int act) {
  if (act == ACT_NONE) return v;
  f32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = activate(v[i], act);
  return u;
}

// The residual of features n .. n + 3 of row t (zeros where there is none), and
// the bias, activation, residual and store of a product.  vec: rows of y and
// residual are aligned for four values at a time.
__device__ __forceinline__ f32x4 linear_residual(const LinearArgs& a, int t, int n, bool vec) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (!a.res || t >= a.T || n >= a.N) return v;
  const size_t o = (size_t)t * a.ldr + n;
  if (a.odt == DT_BF16) {
    const uint16_t* res = reinterpret_cast<const uint16_t*>(a.res) + o;
    if (vec) {
      const uint2 r = *reinterpret_cast<const uint2*>(res);
      return f32x4{bf2f(r.x & 0xffff), bf2f(r.x >> 16), bf2f(r.y & 0xffff), bf2f(r.y >> 16)};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < a.N) v[i] = bf2f(res[i]);
  } else {
    const float* res = reinterpret_cast<const float*>(a.res) + o;
    if (vec) return *reinterpret_cast<const f32x4*>(res);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < a.N) v[i] = res[i];
  }
  return v;
}
__device__ __forceinline__ void linear_store(const LinearArgs& a, int t, int n, f32x4 v, bool vec) {
  if (t >= a.T || n >= a.N) return;
  const size_t o = (size_t)t * a.ldy + n;
  if (a.odt == DT_BF16) {
    uint16_t* y = reinterpret_cast<uint16_t*>(a.y) + o;
    if (vec) {
      *reinterpret_cast<uint2*>(y) = make_uint2(bf16x2_bits(v[0], v[1]), bf16x2_bits(v[2], v[3]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) y[i] = (uint16_t)f2bf_bits(v[i]);
    }
  } else {
    float* y = reinterpret_cast<float*>(a.y) + o;
    if (vec) {
      *reinterpret_cast<f32x4*>(y) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) y[i] = v[i];
    }
  }
}
__device__ __forceinline__ void linear_out(const LinearArgs& a, int t, int n, f32x4 v, f32x4 bias, f32x4 res, bool vec) {
  linear_store(a, t, n, activate4(v + bias, a.act) + res, vec);
}
__device__ __forceinline__ bool linear_vec(const LinearArgs& a) {
  const uintptr_t need = a.odt == DT_BF16 ? 8 : 16;
  return a.N % 4 == 0 && a.ldy % 4 == 0 && (!a.res || a.ldr % 4 == 0) && reinterpret_cast<uintptr_t>(a.y) % need == 0 &&
         reinterpret_cast<uintptr_t>(a.res) % need == 0;
}
// Eight bf16 values of a row at a time: rows of y and residual in 16-byte pieces.
__device__ __forceinline__ bool linear_wide(const LinearArgs& a) {
  return a.odt == DT_BF16 && a.N % 8 == 0 && a.ldy % 8 == 0 && (!a.res || a.ldr % 8 == 0) &&
         (reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.res)) % 16 == 0;
}
__device__ __forceinline__ void linear_store8(const LinearArgs& a, int t, int n, f32x4 v, f32x4 u) {
  if (t >= a.T || n >= a.N) return;
  *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.y) + (size_t)t * a.ldy + n) =
      make_uint4(bf16x2_bits(v[0], v[1]), bf16x2_bits(v[2], v[3]), bf16x2_bits(u[0], u[1]), bf16x2_bits(u[2], u[3]));
}
__device__ __forceinline__ f32x4 linear_bias(const LinearArgs& a, int n) {
  f32x4 b = {0.f, 0.f, 0.f, 0.f};
  if (a.bias)
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = a.bias[min(n + i, a.N - 1)];
  return b;
}

// Chains of a linear's reduction over S super-steps: one for every 64 (2048 bf16
// columns), at most eight, each a run of whole groups of four.  They let a product
// of few rows spread a long reduction over several waves; the others fold one
// accumulator into another at a chain's end.  First super-step of chain j.
constexpr int MAX_CHAINS = 8;

// At most NARROW outputs (a router): CHAINS chains, of the 128-byte stages w, w + 8, ...
constexpr int NARROW = 512, CHAINS = 8;
__host__ __device__ __forceinline__ int linear_chains(int S) {
  const int c = S / 64;
  return c < 1 ? 1 : c > MAX_CHAINS ? MAX_CHAINS : c;
}
__host__ __device__ __forceinline__ int chain_start(int j, int S, int chains) {
  return j == chains ? S : j * (S / 4) / chains * 4;   // (S <= 2^16)
}

// -------------------------------------------------------------- tile products --

// Waits until at most N of the wave's vector memory operations are outstanding.
template <int N> __device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
// Workgroup barrier that waits for no memory operation (the callers wait for
// what they need), and that the compiler moves no access across.
__device__ __forceinline__ void barrier_only() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

enum TileMode { TM_LINEAR, TM_UP, TM_DOWN };

// A run of at most BM rows of one expert, rows p0 .. p0 + n - 1 of the sorted order.
struct ExpertTile {
  int e, p0, n;
};

// What one call's experts kernels share (device memory in the workspace).
struct FfnPlan {
  int* ntile;          // row tiles in use
  ExpertTile* tile;    // [ntile]
  int* order;          // [pairs] pairs (row * k + slot) sorted by expert; skipped ones are not in it
  void* z;             // [pairs][F] dt, rows in sorted order
  float* y;            // [pairs][nc]: columns c0 .. c0 + nc - 1 of the down products, rows by pair (k > 1)
  int c0, nc;
};

struct TileArgs {
  LinearArgs l;        // TM_LINEAR
  FfnArgs f;           // the others
  FfnPlan p;
  int nrt, nft;        // row tiles (at most), feature tiles
  unsigned kmul;       // TM_UP: 2^32 / k rounded up, the factor that divides a pair's number (< 2^24) by k <= 32; 0: k is 1
  bool narrow;         // TM_LINEAR: the chains of a narrow linear; an even number of super-steps
};

// Products of BM rows with BN rows of weights, both streamed through LDS in
// stages of SPS super-steps (64 bytes of a row each), NST stages deep.  What bounds
// a large product is power, and then what shares the CU with the matrix
// cores: fragments read from LDS (a wave of RF x FF fragments reads RF + FF per RF FF
// matrix instructions) and requests written to it.  The largest tile, 128 x 256 with
// eight waves of 64 x 64, keeps two stages in flight and takes 80400 clocks for 4096
// columns where its matrix instructions alone take 65536; with all CUs at work the
// clock falls from 2.4 to 1.6 GHz (8192 x 4096 x 11008: 590 us, 1250 TFLOP/s; all
// requests left out, 540).  Tiles of 256 x 256 (four waves of 128 x 128, or eight) take
// 4 % fewer clocks over 4096 features, more over 11008, and no less time.
//   * Stages arrive by direct loads to LDS, each of whole lines (SPS = 2: eight
//     rows of 128 bytes; 4: four of 256).  The 16-byte pieces of row r stand at
//     place piece ^ (r / 2 % 8) or piece ^ (r % 16), so that the 16 rows that a
//     fragment read touches fall on all banks.
//   * Fragments are read one super-step ahead of the matrix instructions
//     that use them, across the stages' barriers too.
//   * SPS = 4 halves the barriers, which small tiles wait for most, and needs a
//     multiple of four super-steps; SPS = 2 takes any number.
// Rows past the end repeat the last one; their results are not stored.
// Whether a workgroup takes one tile after another, so that the next one's first
// stages are on their way while the last one's results are stored: where only one
// workgroup fits a CU and reductions are short (8192 rows of 128 experts, 2048 x
// 768: 942 us without, 909 so.  The down product's stores still wait for those requests:
// the pairs' numbers that they need are loaded behind them.  Linears and fp32 gain nothing, 8192 x 11008 606 us without,
// 612 so: the sums of their chains leave too few registers).
template <int DT, int MODE, int BM, int BN, int NST, int SPS> constexpr bool tile_keeps() {
  return MODE != TM_LINEAR && DT != DT_F32 && (BM + BN) * SPS * 64 * NST > 80 * 1024;
}

template <int DT, int MODE, int BM, int BN, int WR, int WF, int NST, int SPS>
__global__ __launch_bounds__(WR * WF * 64, 2) void tile_kernel(TileArgs a) {
  constexpr int ESZ = Geo<DT>::ESZ, WAVES = WR * WF, RF = BM / WR / 16, FF = BN / WF / 16;
  constexpr int PPR = 4 * SPS, RPL = 64 / PPR;   // 16-byte pieces of a row's stage, rows per load
  constexpr int LPW = (BM + BN) / RPL / WAVES;   // loads per wave and stage
  constexpr int STAGE = (BM + BN) * PPR;         // pieces of a stage
  constexpr bool KEEP = tile_keeps<DT, MODE, BM, BN, NST, SPS>();
  constexpr bool NARROWS = MODE == TM_LINEAR && SPS == 2;
  static_assert(SPS == 2 || SPS == 4, "two fragment sets in turn, rows of 8 or 16 pieces");
  static_assert((BM + BN) % (RPL * WAVES) == 0 && BM % RPL == 0, "every wave loads as much");
  static_assert(MODE != TM_UP || FF % 2 == 0, "a wave owns gate and up tiles of the same features");
  static_assert(NST == 3 || NST == 4, "buffers in turn");
  static_assert((NST - 1) * LPW < 64, "outstanding loads are counted in six bits");
  // (arrays of their own: the compiler then knows that a request into one does not touch the others)
  __shared__ uint4 b0[STAGE], b1[STAGE], b2[STAGE], b3[NST > 3 ? STAGE : 1];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, grp = lane >> 4;
  const int wr = wv / WF, wf = wv % WF;

  // Workgroups are dealt to the eight XCDs in turn: each XCD takes a run of the
  // tiles, GR row tiles side by side under one feature tile after another, so
  // that what they share stays in its L2.
  const int nrt = MODE == TM_LINEAR ? a.nrt : *a.p.ntile;
  const int ntile = nrt * a.nft, per = (ntile + 7) / 8, tile0 = (int)(blockIdx.x & 7) * per;
  const int end = min(per, ntile - tile0);   // this XCD's tiles
  int at = (int)(blockIdx.x >> 3);
  if (at >= end) return;
  constexpr int GR = BN > BM ? 4 : 8;   // (8192 x 11008, 128 x 256 tiles: 608 us with 4, 670 with 8, 680 with 32)
  const int S = (MODE == TM_LINEAR ? a.l.K : MODE == TM_UP ? a.f.d : a.f.F) / Geo<DT>::KS;   // super-steps
  const unsigned ldw = (unsigned)(MODE == TM_LINEAR ? a.l.ldw : MODE == TM_UP ? a.f.d : a.f.F) * ESZ;   // bytes between rows
  const unsigned ldx = (unsigned)(MODE == TM_LINEAR ? a.l.ldx : MODE == TM_UP ? a.f.ldx : a.f.F) * ESZ;
  const int stages = (S + SPS - 1) / SPS;
  auto swizzle = [](int r) { return SPS == 2 ? (r >> 1) & 7 : r & 15; };

  // The order of the weights' rows within a wave's tiles, where the output leaves
  // in bf16: row m of the tiles 2h and 2h + 1 is feature 32 h + 8 (m / 4) + m % 4,
  // and 4 more, so that a lane's values of both are eight in a row and a store
  // instruction writes 64 bytes of each output row instead of 32.
  constexpr int FT = MODE == TM_UP ? FF / 2 : FF;   // tiles that one store covers
  constexpr bool PAIRS = FT % 2 == 0 && DT == DT_BF16 && MODE != TM_DOWN;
  const bool wide = PAIRS && (MODE == TM_UP || linear_wide(a.l));
  auto feature = [&](int f, int m) { return wide ? (f >> 1) * 32 + (m >> 2) * 8 + (f & 1) * 4 + (m & 3) : f * 16 + m; };

  // The tile's place and, for each of the wave's loads, this lane's piece.
  const unsigned char *xb, *wb;   // the operands' tiles
  int t0 = 0, rows, f0;           // first row, rows, first feature
  ExpertTile et{};
  unsigned off[LPW];
  auto place = [&]() {
    const int tile = tile0 + at, gsz = GR * a.nft, gi = tile / gsz, gr0 = gi * GR, gh = min(GR, nrt - gr0), gj = tile - gi * gsz;
    const int rt = gr0 + gj % gh, ft = gj / gh;
    if constexpr (MODE == TM_LINEAR) {
      t0 = rt * BM;
      rows = min(BM, a.l.T - t0);
      f0 = ft * BN;
      xb = reinterpret_cast<const unsigned char*>(a.l.x) + (size_t)t0 * ldx;
      wb = reinterpret_cast<const unsigned char*>(a.l.w) + (size_t)f0 * ldw;
    } else {
      et = a.p.tile[rt];
      rows = et.n;
      if constexpr (MODE == TM_UP) {
        f0 = ft * (BN / 2);
        xb = reinterpret_cast<const unsigned char*>(a.f.x);
        wb = reinterpret_cast<const unsigned char*>(a.f.wgu) + (size_t)et.e * 2 * a.f.F * ldw;
      } else {
        f0 = a.p.c0 + ft * BN;
        xb = reinterpret_cast<const unsigned char*>(a.p.z) + (size_t)et.p0 * ldx;
        wb = reinterpret_cast<const unsigned char*>(a.f.wd) + ((size_t)et.e * a.f.d + f0) * ldw;
      }
    }
    int ln = lane;
    if constexpr (KEEP) asm volatile("" : "+v"(ln));   // (computed anew for each tile: kept, it would cost registers that the products need)
    unsigned pair[LPW];   // (requested together)
    if (MODE == TM_UP && wv * LPW < BM / RPL)
#pragma unroll
      for (int i = 0; i < LPW; ++i) pair[i] = a.p.order[et.p0 + min((wv * LPW + i) * RPL + ln / PPR, rows - 1)];
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
      const int inst = wv * LPW + i;
      int r = inst * RPL + ln / PPR;
      const unsigned piece = ((ln % PPR) ^ swizzle(r)) * 16;
      if (inst < BM / RPL) {
        r = min(r, rows - 1);
        if constexpr (MODE == TM_UP) r = a.kmul ? __umulhi(pair[i], a.kmul) : pair[i];
        off[i] = (unsigned)r * ldx + piece;
      } else {
        r -= BM;
        if constexpr (MODE == TM_LINEAR) {
          const int w = r / (FF * 16), j = r % (FF * 16);
          r = min(w * (FF * 16) + feature(j / 16, j % 16), a.l.N - 1 - f0);
        }
        if constexpr (MODE == TM_DOWN) r = min(r, a.f.d - 1 - f0);
        if constexpr (MODE == TM_UP) {   // a wave's first FF / 2 tiles are gate features, then up of the same
          const int w = r / (FF * 16), j = r % (FF * 16), up = j >= FF * 8;
          const int k = up ? j - FF * 8 : j;
          r = min(f0 + w * (FF * 8) + feature(k / 16, k % 16), a.f.F - 1) + (up ? a.f.F : 0);
        }
        off[i] = (unsigned)r * ldw + piece;
      }
    }
  };
  // Requests load i of the next stage (past the last one: that one again,
  // unused).  The second half of an odd reduction's last stage is the first half
  // again.
  int next;
  auto fetch_one = [&](uint4* buf, int i) {
    const int inst = wv * LPW + i;
    const unsigned over = SPS == 2 && 2 * next + 1 == S && (((lane >> 2) ^ inst) & 1) ? 64u : 0u;
    const unsigned char* src = (inst < BM / RPL ? xb : wb) + (size_t)next * (SPS * STEP);
    __builtin_amdgcn_global_load_lds((global_void*)(src + (off[i] - over)), (lds_void*)(buf + inst * 64), 16, 0, 0);
  };
  // (narrow: every eighth stage, then those that follow the first of them)
  const int step = NARROWS && a.narrow ? CHAINS : 1, starts = NARROWS && a.narrow ? min(CHAINS, stages) : 0;
  auto fetched = [&]() {
    const int on = next + step, start = (next & (step - 1)) + 1;
    next = on < stages ? on : start < starts ? start : next;
  };
  auto fetch = [&](uint4* buf) {
#pragma unroll
    for (int i = 0; i < LPW; ++i) fetch_one(buf, i);
    fetched();
  };
  auto first_stages = [&]() {
    next = 0;
    fetch(b0);
    fetch(b1);
    fetch(b2);
    if constexpr (NST > 3) fetch(b3);
  };

  f32x4 acc[FF][RF], tot[FF][RF];   // the chain, and the sum of the chains before it
  constexpr bool FOLD = MODE == TM_LINEAR || DT == DT_F32;
  const int chains = starts ? starts : MODE == TM_LINEAR ? linear_chains(S) : FOLD ? (S + EXPERT_CHAIN - 1) / EXPERT_CHAIN : 1;
  int ch, ch_end;   // the chain, its last super-step + 1
  const int q = grp ^ swizzle(c);
  const int xo = (wr * RF * 16 + c) * PPR + q, wo = (BM + wf * FF * 16 + c) * PPR + q;
  uint4 xs[2][RF], ws[2][FF];   // the fragments of two super-steps
  // fragment i of super-step s: weights first, then rows
  auto read_one = [&](const uint4* buf, int s, int i) {
    if (i < FF) ws[s & 1][i] = buf[(wo ^ (s * 4)) + i * (16 * PPR)];
    else xs[s & 1][i - FF] = buf[(xo ^ (s * 4)) + (i - FF) * (16 * PPR)];
  };
  constexpr int MN = FF * RF, PARTS = MN < 8 ? MN : 8;
  auto mul = [&](int set, int j0, int j1) {
#pragma unroll
    for (int j = j0; j < j1; ++j) acc[j / RF][j % RF] = mma<DT>(ws[set][j / RF], xs[set][j % RF], acc[j / RF][j % RF]);
  };
  // A super-step's matrix instructions in PARTS parts, between which the next
  // super-step's fragments are read and the requests for a later stage go out,
  // spread over the whole stage: all at once, either would hold up the wave's
  // matrix instructions for as long as all waves' reads or requests take.
  int left;
  auto others = [&](const uint4* cur, uint4* prev, auto ask) {
    --left;
#pragma unroll
    for (int s = 1; s < SPS; ++s)
#pragma unroll
      for (int j = 0; j < PARTS; ++j) {
#pragma unroll
        for (int i = j * (FF + RF) / PARTS; i < (j + 1) * (FF + RF) / PARTS; ++i) read_one(cur, s, i);
        if constexpr (decltype(ask)::value) {
#pragma unroll
          for (int i = (s * PARTS + j) * LPW / (PARTS * SPS); i < (s * PARTS + j + 1) * LPW / (PARTS * SPS); ++i) fetch_one(prev, i);
        }
        __builtin_amdgcn_sched_barrier(0);
        mul((s & 1) ^ 1, j * MN / PARTS, (j + 1) * MN / PARTS);
        __builtin_amdgcn_sched_barrier(0);
      }
    if constexpr (decltype(ask)::value) fetched();
  };
  // The stage in `cur`: the products of the stage before, in `prev`, are finished
  // while its first fragments are read; `prev`, which every wave has read by
  // now, takes the stage NST - 1 on.
  auto stage = [&](uint4* prev, uint4* cur) {
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): this wave's reads of `prev` are done
    wait_vm<(NST - 2) * LPW>();           // its part of `cur` has arrived
    barrier_only();
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
#pragma unroll
      for (int i = j * (FF + RF) / PARTS; i < (j + 1) * (FF + RF) / PARTS; ++i) read_one(cur, 0, i);
#pragma unroll
      for (int i = j * LPW / (PARTS * SPS); i < (j + 1) * LPW / (PARTS * SPS); ++i) fetch_one(prev, i);
      __builtin_amdgcn_sched_barrier(0);
      mul(1, j * MN / PARTS, (j + 1) * MN / PARTS);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (FOLD)
      if ((stages - left) * SPS == ch_end) {   // the stage before ended a chain
        ++ch;
        ch_end = starts ? ch_end + SPS * ((stages - ch + CHAINS - 1) / CHAINS)
                 : MODE == TM_LINEAR ? chain_start(ch + 1, S, chains) : ch_end + EXPERT_CHAIN;
#pragma unroll
        for (int f = 0; f < FF; ++f)
#pragma unroll
          for (int r = 0; r < RF; ++r) {
            tot[f][r] += acc[f][r];
            acc[f][r] = f32x4{0.f, 0.f, 0.f, 0.f};
          }
      }
    others(cur, prev, std::true_type{});
  };

  // One tile after another: the next one's first stages are requested before
  // the last one's results are stored.
  place();
  first_stages();
  for (;;) {
#pragma unroll
    for (int f = 0; f < FF; ++f)
#pragma unroll
      for (int r = 0; r < RF; ++r) tot[f][r] = acc[f][r] = f32x4{0.f, 0.f, 0.f, 0.f};
    ch = 0;
    ch_end = starts ? SPS * ((stages + CHAINS - 1) / CHAINS) : MODE == TM_LINEAR ? chain_start(1, S, chains) : EXPERT_CHAIN;
    left = stages;
    wait_vm<(NST - 1) * LPW>();
    barrier_only();
#pragma unroll
    for (int i = 0; i < FF + RF; ++i) read_one(b0, 0, i);
    others(b0, nullptr, std::false_type{});
    {
      // (whole turns of the buffers without an exit between them, so that the
      // compiler sees which request each read follows and adds no wait of its
      // own; then the rest)
      const int rest = (stages - 1) % NST;
      for (int g = (stages - 1) / NST; g > 0; --g) {
        stage(b0, b1);
        stage(b1, b2);
        if constexpr (NST == 3) stage(b2, b0);
        if constexpr (NST == 4) { stage(b2, b3); stage(b3, b0); }
      }
      if (rest > 0) {
        stage(b0, b1);
        if (rest > 1) {
          stage(b1, b2);
          if constexpr (NST > 3)
            if (rest > 2) stage(b2, b3);
        }
      }
    }
    if (SPS == 4 || S % 2 == 0) mul(1, 0, MN);   // (an odd reduction ends with half a stage)
    if (FOLD && chains > 1) {                            // (one chain: the sum as it is, as everywhere)
#pragma unroll
      for (int f = 0; f < FF; ++f)
#pragma unroll
        for (int r = 0; r < RF; ++r) acc[f][r] = tot[f][r] + acc[f][r];
    }
    wait_vm<0>();   // (nothing may arrive in LDS after the workgroup's end)

    const int ct0 = t0, cf0 = f0, crows = rows, cp0 = et.p0;
    int oc = c, og = 4 * grp;
    if constexpr (KEEP) asm volatile("" : "+v"(oc), "+v"(og));   // (as in place())
    bool more = false;
    if constexpr (KEEP) {
      at += (int)(gridDim.x >> 3);
      more = at < end;
      if (more) {
        __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
        barrier_only();                       // every wave has read its last fragments
        place();
        first_stages();
      }
    }
    if constexpr (MODE == TM_LINEAR) {
      // Each step over all of the wave's values under one branch of its own: with the
      // choices inside the loop its code was so long that fetching it bound it
      // (128 x 256 tiles: 10400 cycles of a workgroup, 4300 so; its 64 stages take 81000).  The residual is read before the first store (y may be
      // the residual, so the compiler keeps each load behind the stores before it).
      auto each = [&](auto fn) {
#pragma unroll
        for (int f = 0; f < FF; ++f)
#pragma unroll
          for (int r = 0; r < RF; ++r) fn(f, r, ct0 + (wr * RF + r) * 16 + oc, cf0 + wf * (FF * 16) + feature(f, og));
      };
      const bool vec = linear_vec(a.l);
      f32x4 res[FF][RF];
      each([&](int f, int r, int t, int n) { res[f][r] = f32x4{0.f, 0.f, 0.f, 0.f}; });
      if (a.l.res) each([&](int f, int r, int t, int n) { res[f][r] = linear_residual(a.l, t, n, vec); });
      f32x4 bias[FF];
#pragma unroll
      for (int f = 0; f < FF; ++f) bias[f] = linear_bias(a.l, cf0 + wf * (FF * 16) + feature(f, og));
      each([&](int f, int r, int, int) { acc[f][r] += bias[f]; });
      auto act = [&](auto kind) { each([&](int f, int r, int, int) { acc[f][r] = activate4(acc[f][r], decltype(kind)::value); }); };
      switch (a.l.act) {
        case ACT_SILU: act(std::integral_constant<int, ACT_SILU>{}); break;
        case ACT_GELU: act(std::integral_constant<int, ACT_GELU>{}); break;
        case ACT_GELU_TANH: act(std::integral_constant<int, ACT_GELU_TANH>{}); break;
        case ACT_RELU: act(std::integral_constant<int, ACT_RELU>{}); break;
        default: break;
      }
      each([&](int f, int r, int, int) { acc[f][r] += res[f][r]; });
      if (wide) {
        if constexpr (PAIRS) each([&](int f, int r, int t, int n) { if (f % 2 == 0) linear_store8(a.l, t, n, acc[f][r], acc[f + 1][r]); });
      } else if (vec) {
        each([&](int f, int r, int t, int n) { linear_store(a.l, t, n, acc[f][r], true); });
      } else {
        each([&](int f, int r, int t, int n) { linear_store(a.l, t, n, acc[f][r], false); });
      }
    } else if constexpr (MODE == TM_UP) {
#pragma unroll
      for (int f = 0; f < FT; f += PAIRS ? 2 : 1) {
        const int n = cf0 + wf * (FT * 16) + feature(f, og);
        if (n >= a.f.F) continue;
#pragma unroll
        for (int r = 0; r < RF; ++r) {
          const int row = (wr * RF + r) * 16 + oc;
          if (row >= crows) continue;
          auto glu = [&](int g) {
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = silu(acc[g][r][i]) * acc[g + FT][r][i];
            return v;
          };
          const size_t o = (size_t)(cp0 + row) * a.f.F + n;
          if constexpr (PAIRS) {   // (F is a multiple of 32)
            const f32x4 v = glu(f), u = glu(f + 1);
            *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(a.p.z) + o) =
                make_uint4(bf16x2_bits(v[0], v[1]), bf16x2_bits(v[2], v[3]), bf16x2_bits(u[0], u[1]), bf16x2_bits(u[2], u[3]));
          } else {
            store4<DT>(a.p.z, o, glu(f));
          }
        }
      }
    } else {
      int to[RF];
#pragma unroll
      for (int r = 0; r < RF; ++r) to[r] = a.p.order[cp0 + min((wr * RF + r) * 16 + oc, crows - 1)];
#pragma unroll
      for (int r = 0; r < RF; ++r) {
        const int row = (wr * RF + r) * 16 + oc;
        if (row >= crows) continue;
        if (a.f.k == 1) {   // (a row's only product: nothing to join)
          LinearArgs o{};
          o.y = a.f.out; o.res = a.f.res; o.ldy = a.f.ldo; o.ldr = a.f.ldr;
          o.T = a.f.T; o.N = a.f.d; o.odt = a.f.odt;
          const bool vec = linear_vec(o);
          const float w = a.f.weights[to[r]];
#pragma unroll
          for (int f = 0; f < FF; ++f) {
            const int n = cf0 + (wf * FF + f) * 16 + og;
            f32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf(w, acc[f][r][i], 0.f);
            if (o.res) v += linear_residual(o, to[r], n, vec);
            linear_store(o, to[r], n, v, vec);
          }
          continue;
        }
        float* y = a.p.y + (size_t)to[r] * a.p.nc;
#pragma unroll
        for (int f = 0; f < FF; ++f) {
          const int n = cf0 - a.p.c0 + (wf * FF + f) * 16 + og;
          if (n < a.p.nc) *reinterpret_cast<f32x4*>(y + n) = acc[f][r];
        }
      }
    }
    if (!KEEP || !more) break;
  }
}

template <int DT, int MODE, int BM, int BN, int WR, int WF, int NST, int SPS = 2>
static hipError_t launch_tile(TileArgs a, hipStream_t st) {
  if (MODE == TM_LINEAR) a.nrt = (a.l.T + BM - 1) / BM;
  const int cols = MODE == TM_LINEAR ? a.l.N : MODE == TM_UP ? 2 * a.f.F : a.p.nc;
  a.nft = (cols + BN - 1) / BN;
  if (MODE == TM_UP) a.kmul = a.f.k > 1 ? 0xffffffffu / a.f.k + 1 : 0;
  int64_t n = (int64_t)a.nrt * a.nft;
  if (tile_keeps<DT, MODE, BM, BN, NST, SPS>()) n = std::min<int64_t>(n, 256);   // one for each CU
  hipLaunchKernelGGL((tile_kernel<DT, MODE, BM, BN, WR, WF, NST, SPS>), dim3((unsigned)((n + 7) / 8 * 8)), dim3(WR * WF * 64), 0,
                     st, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------- linear --

// Few rows: a wave per chain of MT row tiles and NT feature tiles, operands
// straight to registers, the workgroup's chains added in order.  (D: steps in
// flight, what the registers hold.)
template <int DT, int MT, int NT, int D>
__global__ __launch_bounds__(MAX_CHAINS * 64, 2) void linear_rows_kernel(LinearArgs a, int nblk) {
  constexpr int ESZ = Geo<DT>::ESZ;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, grp = lane >> 4;
  const int t0 = blockIdx.x / nblk * (MT * 16), n0 = blockIdx.x % nblk * (NT * 16);
  const int S = a.K / Geo<DT>::KS, chains = linear_chains(S);
  const int s0 = chain_start(wv, S, chains), s1 = chain_start(wv + 1, S, chains);
  const unsigned char *wp[NT], *xp[MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
    wp[n] = reinterpret_cast<const unsigned char*>(a.w) + (size_t)min(n0 + n * 16 + c, a.N - 1) * a.ldw * ESZ + grp * 16 +
            (size_t)s0 * STEP;
#pragma unroll
  for (int m = 0; m < MT; ++m)
    xp[m] = reinterpret_cast<const unsigned char*>(a.x) + (size_t)min(t0 + m * 16 + c, a.T - 1) * a.ldx * ESZ + grp * 16 +
            (size_t)s0 * STEP;
  f32x4 acc[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  chain<DT, NT, MT, D>(wp, xp, s1 - s0, acc);
  __shared__ f32x4 red[MAX_CHAINS][NT * MT][64];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) red[wv][n * MT + m][lane] = acc[n][m];
  __syncthreads();
  const bool vec = linear_vec(a);
  for (int i = wv; i < NT * MT; i += chains) {
    f32x4 v = red[0][i][lane];
    for (int w = 1; w < chains; ++w) v += red[w][i][lane];
    const int t = t0 + i % MT * 16 + c, n = n0 + i / MT * 16 + 4 * grp;
    linear_out(a, t, n, v, linear_bias(a, n), linear_residual(a, t, n, vec), vec);
  }
}

template <int DT, int MT, int NT, int D>
static hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  const int nblk = (a.N + NT * 16 - 1) / (NT * 16);
  const int chains = linear_chains(a.K / ks_of(a.dt));
  hipLaunchKernelGGL((linear_rows_kernel<DT, MT, NT, D>), dim3((unsigned)nblk * ((a.T + MT * 16 - 1) / (MT * 16))),
                     dim3(chains * 64), 0, st, a, nblk);
  return hipGetLastError();
}

// Products of few outputs (a router): a workgroup's eight waves each sum the
// 128-byte stages w, w + 8, ... of the reduction for MT x NT tiles, and the
// eight sums are added in wave order.
template <int DT, int MT, int NT>
__global__ __launch_bounds__(CHAINS * 64) void linear_narrow_kernel(LinearArgs a, int nblk) {
  constexpr int ESZ = Geo<DT>::ESZ;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, grp = lane >> 4;
  const int n0 = blockIdx.x % nblk * (NT * 16), t0 = blockIdx.x / nblk * (MT * 16);
  const int S = a.K / Geo<DT>::KS;
  const unsigned char *wp[NT], *xp[MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
    wp[n] = reinterpret_cast<const unsigned char*>(a.w) + (size_t)min(n0 + n * 16 + c, a.N - 1) * a.ldw * ESZ + wv * (2 * STEP) + grp * 16;
#pragma unroll
  for (int m = 0; m < MT; ++m)
    xp[m] = reinterpret_cast<const unsigned char*>(a.x) + (size_t)min(t0 + m * 16 + c, a.T - 1) * a.ldx * ESZ + wv * (2 * STEP) + grp * 16;
  f32x4 acc[NT][MT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
  // (this wave's stages, less the missing half of the last one of all)
  const int stages = (S + 1) / 2, own = (stages - wv + CHAINS - 1) / CHAINS;
  chain<DT, NT, MT, (MT * NT > 4 ? 4 : 16), false, CHAINS>(wp, xp, 2 * own - (S % 2 && (stages - 1) % CHAINS == wv), acc);
  __shared__ f32x4 red[CHAINS][NT * MT][64];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int m = 0; m < MT; ++m) red[wv][n * MT + m][lane] = acc[n][m];
  __syncthreads();
  for (int i = wv; i < NT * MT; i += CHAINS) {
    f32x4 v = red[0][i][lane];
#pragma unroll
    for (int w = 1; w < CHAINS; ++w) v += red[w][i][lane];
    const int t = t0 + i % MT * 16 + c, n = n0 + i / MT * 16 + 4 * grp;
    linear_out(a, t, n, v, linear_bias(a, n), linear_residual(a, t, n, linear_vec(a)), linear_vec(a));
  }
}

template <int DT, int MT, int NT>
static hipError_t launch_narrow(const LinearArgs& a, hipStream_t st) {
  const int nblk = (a.N + NT * 16 - 1) / (NT * 16);
  hipLaunchKernelGGL((linear_narrow_kernel<DT, MT, NT>), dim3((unsigned)nblk * ((a.T + MT * 16 - 1) / (MT * 16))),
                     dim3(CHAINS * 64), 0, st, a, nblk);
  return hipGetLastError();
}

template <int DT>
static hipError_t linear_t(const LinearArgs& a, hipStream_t st) {
  const int64_t rt = (a.T + 15) / 16, nt = (a.N + 15) / 16;
  TileArgs t{};
  t.l = a;
  const bool f32 = DT == DT_F32;
  if (a.N <= NARROW) {
    // The narrow kernel's 16 x 16 tiles while there are few, LDS tiles (in the order of
    // its chains, for an even number of super-steps) where they take fewer turns of
    // the chip; us over 4096 columns, alone and per turn of the 256 CUs.  1 row 2048 -> 128
    // 4.4 us, 32 x 32 tiles 7.2; 1024 rows 2048 -> 256 19 and 8.1; 8192 rows 2048 -> 128
    // 27, 64 x 64 11.6; 8192 rows 4096 -> 512 178, 128 x 128 35.  fp32 300 rows 8192 -> 300
    // 59, 32 x 32 55; 1000 rows 2048 -> 256 33 and 18.
    t.narrow = true;
    auto cost = [&](int64_t m, int64_t n, double alone, double turn) {
      return std::max(alone, ceil((double)((a.T + m - 1) / m * ((a.N + n - 1) / n)) / 256.0) * turn);
    };
    const double c0 = f32 ? cost(16, 16, 16, 16) : cost(16, 16, 9, 9), c1 = f32 ? cost(32, 32, 28, 20) : cost(32, 32, 11, 5.5),
                 c2 = f32 ? cost(64, 64, 68, 62) : cost(64, 64, 15, 12), c3 = f32 ? cost(128, 128, 239, 240) : cost(128, 128, 25, 35);
    const double best = std::min({c0, c1, c2, c3});
    if (best < c0 && a.K / Geo<DT>::KS % 2 == 0) {
      if (best == c3) return launch_tile<DT, TM_LINEAR, 128, 128, 2, 4, 4>(t, st);
      if (best == c2) return launch_tile<DT, TM_LINEAR, 64, 64, 2, f32 ? 4 : 2, 4>(t, st);
      return launch_tile<DT, TM_LINEAR, 32, 32, 2, 2, 4, 2>(t, st);
    }
    // (odd reductions of many rows: larger tiles read the rows less often)
    return rt * nt <= 2048 ? launch_narrow<DT, 1, 1>(a, st) : launch_narrow<DT, 2, 4>(a, st);
  }
  // 4096 x 4096, weights from HBM: 9.2 us for one row, 9.6 for eight (32 x 32 tiles 11);
  // of 32256 columns 59 us (64 x 64 tiles 51)
  if (a.T <= 16 && nt <= 1024) return launch_rows<DT, 1, 1, 16>(a, st);
  // The tile that finishes first: turns of the 256 CUs times what a turn costs
  // (us over 4096 bf16 columns).  33 rows, weights from HBM, tiles of 32 x 32 /
  // 64 x 32 / 64 x 64: 4096 features 11.4 / 13.5 / 20 us, 6144 16.7 / 14.5 / 21,
  // 32256 69 / 64 / 54 (one barrier per two super-steps: 16.4 / 17.4 / 20 at
  // 4096).  256 rows x 4096: 64 x 64 14, 128 x 128 26.  513 x 4096: 64 x 64 37,
  // 128 x 128 26, 128 x 256 41.  With all CUs at work the clock falls, and the
  // large tiles' turns take 36 and 55: 8192 x 11008 128 x 128 740, 128 x 256 590;
  // 1024 x 19200 over 7168 columns 331 and 288.
  auto cost = [&](int64_t m, int64_t n, int64_t turn, int64_t full) {
    const int64_t tiles = (a.T + m - 1) / m * ((a.N + n - 1) / n);
    return std::max((tiles + 255) / 256 * turn * 256, tiles * full);
  };
  const int64_t none = INT64_MAX;   // (tiles of more than twice the rows only add reads)
  // fp32 is bound by its matrix instructions, a sixteenth as fast, and what counts
  // is that all CUs have the same work: over 4096 columns 32 x 32 25 us, 19 with
  // more than one on a CU, 64 x 64 67 and 62, 128 x 128 239.  513 x 4096: 32 x 32 169,
  // 64 x 64 188, 128 x 128 243; 2000 x 2000 over 2048 columns 153, 128, 125; 64 x 64
  // with eight waves 4 to 8 % faster than with four.
  const int64_t c0 = f32 ? cost(32, 32, 19, 19) : cost(32, 32, 9, 9), c1 = f32 ? cost(64, 32, 40, 40) : cost(64, 32, 14, 14),
                c2 = f32 ? cost(64, 64, 62, 62) : cost(64, 64, 18, 18),
                c3 = a.T <= 64 ? none : f32 ? cost(128, 128, 239, 240) : cost(128, 128, 27, 36),
                c4 = a.T <= 64 ? none : f32 ? cost(128, 256, 466, 480) : cost(128, 256, 43, 55);
  const int64_t best = std::min({c0, c1, c2, c3, c4});
  if (best == c4) return launch_tile<DT, TM_LINEAR, 128, 256, 2, 4, 3>(t, st);
  if (best == c3) return launch_tile<DT, TM_LINEAR, 128, 128, 2, 4, 4>(t, st);
  if (best == c2) return launch_tile<DT, TM_LINEAR, 64, 64, 2, DT == DT_F32 ? 4 : 2, 4>(t, st);
  const bool four = a.K / Geo<DT>::KS % 4 == 0;
  if (best == c1)
    return four ? launch_tile<DT, TM_LINEAR, 64, 32, 4, 2, 4, 4>(t, st) : launch_tile<DT, TM_LINEAR, 64, 32, 2, 2, 4, 2>(t, st);
  return four ? launch_tile<DT, TM_LINEAR, 32, 32, 2, 2, 4, 4>(t, st) : launch_tile<DT, TM_LINEAR, 32, 32, 2, 2, 4, 2>(t, st);
}

hipError_t run_linear(const LinearArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  return a.dt == DT_F32 ? linear_t<DT_F32>(a, st) : linear_t<DT_BF16>(a, st);
}

// -------------------------------------------------------------------- route --

constexpr int ROUTE_ROWS = 4;   // rows (waves) per workgroup

// x of the lane n places on in its row of 16 (a rotation), as DPP: no LDS.
template <int N> __device__ __forceinline__ uint32_t ror16(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, false);
}
template <int N> __device__ __forceinline__ double ror16d(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)ror16<N>((uint32_t)(b >> 32)) << 32 | ror16<N>((uint32_t)b));
}
// f over the wave's 64 values of x, in every lane: rotations within the rows of
// 16, then swaps of rows and of halves (both of a swap's results, in the same
// order in every lane).
template <class F> __device__ __forceinline__ uint32_t wave_all(uint32_t x, F f) {
  x = f(x, ror16<1>(x));
  x = f(x, ror16<2>(x));
  x = f(x, ror16<4>(x));
  x = f(x, ror16<8>(x));
  const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return f(q[0], q[1]);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  return wave_all(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ double lane_value(double x, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(b >> 32), lane), lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// (rotations add in another order in every lane: lane 0's sum serves all, or equal
// scores would differ in their last bit)
__device__ __forceinline__ double wave_sum(double x) {
  x += ror16d<1>(x);
  x += ror16d<2>(x);
  x += ror16d<4>(x);
  x += ror16d<8>(x);
  return ((lane_value(x, 0) + lane_value(x, 16)) + lane_value(x, 32)) + lane_value(x, 48);
}
// Unsigned integers in the order of the values (of which none is -0 or NaN).
__device__ __forceinline__ uint64_t ordered(double x) {
  const int64_t b = __builtin_bit_cast(int64_t, x);
  return (uint64_t)(b ^ ((b >> 63) | INT64_MIN));
}

// 1 / x for x >= 1 (0 for infinity): the hardware's estimate (2^-22 off or less) and two
// Newton steps.  The second one's only rounding is its last fma's, of a value 2^-86 off
// or less, so the result is the rounded quotient but for quotients that close to halfway
// between two doubles.  Near 1, where scores lie closest, sums 1 + e^-l that differ are
// 2^-52 apart at least and their quotients two steps: they neither swap nor become equal.  (A
// division that rounds right always takes three times the instructions.)
__device__ __forceinline__ double reciprocal(double x) {
  double r = __builtin_amdgcn_rcp(x);
  r = fma(fma(-x, r, 1.0), r, r);
  r = fma(fma(-x, r, 1.0), r, r);
  return x == INFINITY ? 0.0 : r;
}

// One wave per row, experts e = 64 i + lane in registers.  Scores, biased
// scores and the selection are float64 values of the logits, so which experts
// a row gets never hangs on a float32 rounding.  The k experts are taken one
// after another: every lane's best (the first of equal ones), then the wave's by
// the upper halves of the ordered keys, by the lower halves and by the
// index where those before leave several.  Bound by the vector instructions: 16384
// rows of 256 sigmoid scores in 8 groups 62 us with shuffles through LDS and a
// lane per group, 32 with 1120 instructions per row, 25 us with 830
// (keys as ordered integers and sorted per lane, scores looked up at the end).
template <int DT, int EPL>
__global__ __launch_bounds__(ROUTE_ROWS * 64) void route_kernel(RouteArgs a) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, t = blockIdx.x * ROUTE_ROWS + wv;
  __shared__ double lds[ROUTE_ROWS][EPL * 64];   // the row's keys (groups), then its scores
  const bool row = t < a.T;
  constexpr double NONE = -INFINITY;
  constexpr uint64_t ONONE = 0x000fffffffffffffull;   // ordered(NONE); no key's upper half is as small
  float l[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    l[i] = row && e < a.E ? load_elt<DT>(a.logits, (size_t)t * a.ld + e) : -INFINITY;
  }
  double s[EPL], key[EPL];
  float mx = -FLT_MAX;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    l[i] = l[i] > -INFINITY ? fminf(l[i], FLT_MAX) : -INFINITY;   // (NaN: not selectable)
    mx = fmaxf(mx, l[i]);
  }
  if (a.score == SCORE_SOFTMAX) {
    mx = __uint_as_float(wave_all(__float_as_uint(mx), [](uint32_t x, uint32_t y) {
      return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y)));
    }));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      s[i] = exp((double)l[i] - (double)mx);   // (mx is finite: 0 for -inf)
      sum += s[i];
    }
    sum = wave_sum(sum);
    const double inv = sum > 0.0 ? 1.0 / sum : 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) s[i] *= inv;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) s[i] = reciprocal(1.0 + exp(-(double)l[i]));   // (0 for -inf)
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    key[i] = l[i] == -INFINITY ? NONE : s[i];
    if (a.bias && e < a.E) {
      const float f = a.bias[e];
      key[i] = f > -INFINITY ? key[i] + (double)fminf(f, FLT_MAX) : NONE;   // (NaN: not selectable)
    }
  }
  if (a.groups > 1) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) lds[wv][i * 64 + lane] = key[i];
    __syncthreads();
    const int per = a.E / a.groups;
    int lanes = 1;   // lanes per group
    while (2 * lanes * a.groups <= 64) lanes *= 2;
    const int g = lane / lanes;
    double b1 = NONE, b2 = NONE;   // the group's best two keys
    if (g < a.groups)
      for (int i = lane % lanes; i < per; i += lanes) {
        const double v = lds[wv][g * per + i], low = v > b1 ? b1 : v;
        b2 = low > b2 ? low : b2;
        b1 = v > b1 ? v : b1;
      }
    for (int o = 1; o < lanes; o <<= 1) {
      const double c1 = __shfl_xor(b1, o), c2 = __shfl_xor(b2, o);
      const double low = c1 > b1 ? b1 : c1, two = c2 > b2 ? c2 : b2;
      b2 = low > two ? low : two;
      b1 = c1 > b1 ? c1 : b1;
    }
    const double gs = a.group_top == 2 && b2 > NONE ? b1 + b2 : b1;
    // groups that come before this one: better, or equal with a lower index
    int before = 0;
    for (int h = 0; h < a.groups; ++h) {
      const double o = lane_value(gs, h * lanes);
      before += o > gs || (o == gs && h < g);
    }
    const unsigned long long keep = __ballot(g < a.groups && before < a.top_groups);
    const unsigned inv = ((1u << 20) + per - 1) / per;   // e / per = e inv / 2^20 for e, per <= 1024
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = i * 64 + lane;
      if (e < a.E && !((keep >> ((e * inv >> 20) * lanes)) & 1ull)) key[i] = NONE;
    }
    __syncthreads();
  }
  uint64_t o[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    lds[wv][i * 64 + lane] = s[i];
    o[i] = ordered(key[i]);
  }
  // up to four keys per lane are sorted first (neighbours only, so equal ones keep
  // their order), and a winner's list moves up; more are searched every time
  constexpr bool SORTED = EPL <= 4;
  int at[SORTED ? EPL : 1];   // expert / 64 of the sorted keys
  if constexpr (SORTED) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) at[i] = i;
#pragma unroll
    for (int n = EPL - 1; n > 0; --n)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const bool sw = o[i + 1] > o[i];
        const uint64_t x = o[i], y = o[i + 1];
        const int u = at[i], v = at[i + 1];
        o[i] = sw ? y : x; o[i + 1] = sw ? x : y;
        at[i] = sw ? v : u; at[i + 1] = sw ? u : v;
      }
  }
  int id = -1;   // lane j: the expert of slot j
  for (int j = 0; j < a.k; ++j) {
    uint64_t best = o[0];
    if constexpr (!SORTED) {
      at[0] = 0;
#pragma unroll
      for (int i = 1; i < EPL; ++i)
        if (o[i] > best) { best = o[i]; at[0] = i; }
    }
    const uint32_t hi = (uint32_t)(best >> 32), lo = (uint32_t)best;
    const uint32_t top = wave_max(hi);
    if (top == (uint32_t)(ONONE >> 32)) break;   // none left
    unsigned long long m = __ballot(hi == top);
    if (m & (m - 1)) {
      const uint32_t low = wave_max(hi == top ? lo : 0u);
      m = __ballot(hi == top && lo == low);
      if (m & (m - 1)) {   // equal keys: the lowest index
        const bool in = (m >> lane) & 1ull;
        const uint32_t inv = ~(uint32_t)(at[0] * 64 + lane), last = wave_max(in ? inv : 0u);
        m = __ballot(in && inv == last);
      }
    }
    const int win = __builtin_amdgcn_readfirstlane(__ffsll(m) - 1), wi = __builtin_amdgcn_readlane(at[0], win);
    if (lane == j) id = wi * 64 + win;
    if constexpr (SORTED) {
      if (lane == win) {
#pragma unroll
        for (int i = 0; i + 1 < EPL; ++i) { o[i] = o[i + 1]; at[i] = at[i + 1]; }
        o[EPL - 1] = ONONE;
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (i == wi && lane == win) o[i] = ONONE;
    }
  }
  __syncthreads();
  double w = id >= 0 ? lds[wv][id] : 0.0;
  if (a.renorm) {
    double tot = 0.0;
    for (int j = 0; j < a.k; ++j) tot += lane_value(w, j);
    w = tot > 0.0 ? w / tot : 0.0;
  }
  if (row && lane < a.k) {
    a.ids[(size_t)t * a.k + lane] = id;
    a.weights[(size_t)t * a.k + lane] = (float)(w * (double)a.scale);
  }
}

template <int DT>
static hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
  const dim3 grid((a.T + ROUTE_ROWS - 1) / ROUTE_ROWS), block(ROUTE_ROWS * 64);
  if (a.E <= 64) hipLaunchKernelGGL((route_kernel<DT, 1>), grid, block, 0, st, a);
  else if (a.E <= 128) hipLaunchKernelGGL((route_kernel<DT, 2>), grid, block, 0, st, a);
  else if (a.E <= 256) hipLaunchKernelGGL((route_kernel<DT, 4>), grid, block, 0, st, a);
  else if (a.E <= 512) hipLaunchKernelGGL((route_kernel<DT, 8>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((route_kernel<DT, 16>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t run_route(const RouteArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  return a.dt == DT_BF16 ? launch_route<DT_BF16>(a, st) : launch_route<DT_F32>(a, st);
}

// ------------------------------------------------------------------ experts --

// z[p] = silu(x Wg^T) * (x Wu^T) of pair p = (row, slot), rounded to the model
// dtype: it is the next product's operand, as in the dense layers (in bf16 the result is
// 1.4 times as far off as with float32 there, 2.4e-3 to 1.7e-3; two bf16 parts would double
// the down product's matrix instructions).  One 16-feature tile of gate and of
// up per wave; all 16 columns of the product hold the pair's row.
template <int DT>
__global__ __launch_bounds__(64, 2) void ffn_up_kernel(FfnArgs a, void* z, int nblk) {
  constexpr int ESZ = Geo<DT>::ESZ;
  const int lane = threadIdx.x, c = lane & 15, grp = lane >> 4;
  const int p = blockIdx.x / nblk, f0 = blockIdx.x % nblk * 16;
  const int e = a.ids[p];
  if (e < 0 || e >= a.E) return;
  const size_t rb = (size_t)a.d * ESZ;
  const unsigned char* w = reinterpret_cast<const unsigned char*>(a.wgu) + ((size_t)e * 2 * a.F + f0 + c) * rb + grp * 16;
  const unsigned char* wp[2] = {w, w + (size_t)a.F * rb};
  const unsigned char* xp[1] = {reinterpret_cast<const unsigned char*>(a.x) + (size_t)(p / a.k) * a.ldx * ESZ + grp * 16};
  f32x4 acc[2][1] = {{f32x4{0.f, 0.f, 0.f, 0.f}}, {f32x4{0.f, 0.f, 0.f, 0.f}}};
  chain<DT, 2, 1, EXPERT_CHAIN, DT == DT_F32>(wp, xp, a.d / Geo<DT>::KS, acc);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = silu(acc[0][0][i]) * acc[1][0][i];
  if (c == 0) store4<DT>(z, (size_t)p * a.F + f0 + 4 * grp, v);
}

constexpr int DOWN_WAVES = 8;

// out[t] = sum_j w_j (z_j Wd^T) + res of 16 features of one row: a wave per
// slot, the slots' products joined in slot order.
template <int DT, int ODT>
__global__ __launch_bounds__(DOWN_WAVES * 64, 2) void ffn_down_kernel(FfnArgs a, const void* z, int nblk) {
  constexpr int ESZ = Geo<DT>::ESZ;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = lane & 15, grp = lane >> 4;
  const int t = blockIdx.x / nblk, n0 = blockIdx.x % nblk * 16;
  __shared__ float y[ROUTE_MAX_K][16], wj[ROUTE_MAX_K];
  __shared__ bool on[ROUTE_MAX_K];
  // (what joining needs is requested with the products' operands: one token
  // 23.0 us, 23.7 with these read slot by slot at the end)
  float res = 0.f;
  if (threadIdx.x < a.k) {
    const size_t p = (size_t)t * a.k + threadIdx.x;
    const int e = a.ids[p];
    on[threadIdx.x] = e >= 0 && e < a.E;
    wj[threadIdx.x] = a.weights[p];
  }
  if (a.res && threadIdx.x < 16) res = load_elt<ODT>(a.res, (size_t)t * a.ldr + n0 + threadIdx.x);
  for (int j = wv; j < a.k; j += DOWN_WAVES) {
    const size_t p = (size_t)t * a.k + j;
    const int e = a.ids[p];
    if (e < 0 || e >= a.E) continue;
    const size_t rb = (size_t)a.F * ESZ;
    const unsigned char* wp[1] = {reinterpret_cast<const unsigned char*>(a.wd) + ((size_t)e * a.d + n0 + c) * rb + grp * 16};
    const unsigned char* zp[1] = {reinterpret_cast<const unsigned char*>(z) + p * rb + grp * 16};
    f32x4 acc[1][1] = {{f32x4{0.f, 0.f, 0.f, 0.f}}};
    chain<DT, 1, 1, DT == DT_F32 ? EXPERT_CHAIN : 24, DT == DT_F32>(wp, zp, a.F / Geo<DT>::KS, acc);
    if (c == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[j][4 * grp + i] = acc[0][0][i];
  }
  __syncthreads();
  if (threadIdx.x < 16) {
    float o = 0.f;
    for (int j = 0; j < a.k; ++j)
      if (on[j]) o = fmaf(wj[j], y[j][threadIdx.x], o);
    const int n = n0 + threadIdx.x;
    if (a.res) o += res;
    store_elt<ODT>(a.out, (size_t)t * a.ldo + n, o);
  }
}

// ------------------------------------------------------- experts, many rows --

// Sorts the pairs by expert and cuts every expert's run into row tiles of BM.
// Workgroup b places the pairs of chunk b.  It needs the counts of all pairs and
// of those before its chunk, and counts them itself (every workgroup reads all
// ids, from L2): one launch and no wait between workgroups.  (65536 pairs: 61 us
// in a single workgroup.)  At most PLAN_BLOCKS chunks, so that the time grows with
// the pairs and not with their square (2^22 pairs, 64 experts of 32 over 32: the call 4.5 ms
// with chunks of 2048, 2.2 so; all pairs of one expert 29.8 and 10.4).  The order of the pairs within an expert may differ
// from run to run; every row's arithmetic is its own, so the results do not.
constexpr int PLAN_THREADS = 1024, PLAN_CHUNK = 2048, PLAN_BLOCKS = 256;
static_assert(PLAN_THREADS >= ROUTE_MAX_E, "a thread per expert");
int plan_chunk(int64_t P) { return (int)std::max<int64_t>(PLAN_CHUNK, (P + PLAN_BLOCKS - 1) / PLAN_BLOCKS); }
__global__ __launch_bounds__(PLAN_THREADS) void ffn_plan_kernel(const int* __restrict__ ids, int P, int chunk, int E, int BM, FfnPlan p) {
  __shared__ int cnt[ROUTE_MAX_E], first[ROUTE_MAX_E], tiles[ROUTE_MAX_E];
  const int t = threadIdx.x, lo = blockIdx.x * chunk, hi = min(P, lo + chunk);
  if (t < E) cnt[t] = 0;
  __syncthreads();
  auto count = [&](int from, int to) {
    for (int i = from + t; i < to; i += 4 * PLAN_THREADS) {
      int e[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) e[j] = i + j * PLAN_THREADS < to ? ids[i + j * PLAN_THREADS] : -1;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (e[j] >= 0 && e[j] < E) atomicAdd(&cnt[e[j]], 1);
    }
    __syncthreads();
  };
  count(0, lo);
  const int before = t < E ? cnt[t] : 0;
  __syncthreads();
  count(lo, P);
  // inclusive scans of the counts and of the tiles
  int n = 0, own = 0;
  if (t < E) {
    n = cnt[t];
    own = (n + BM - 1) / BM;
    first[t] = n;
    tiles[t] = own;
  }
  __syncthreads();
  for (int o = 1; o < E; o <<= 1) {
    int a = 0, b = 0;
    if (t >= o && t < E) { a = first[t - o]; b = tiles[t - o]; }
    __syncthreads();
    if (t >= o && t < E) { first[t] += a; tiles[t] += b; }
    __syncthreads();
  }
  if (t < E) {
    const int p0 = first[t] - n, t0 = tiles[t] - own;
    if (blockIdx.x == 0) {
      for (int i = 0; i < own; ++i) p.tile[t0 + i] = ExpertTile{t, p0 + i * BM, min(BM, n - i * BM)};
      if (t == E - 1) *p.ntile = tiles[t];
    }
    cnt[t] = p0 + before;
  }
  __syncthreads();
  for (int i = lo + t; i < hi; i += PLAN_THREADS) {
    const int e = ids[i];
    if (e >= 0 && e < E) p.order[atomicAdd(&cnt[e], 1)] = i;
  }
}

// out[t] = sum_j w_j y[t k + j] + res, slots in order, of columns c0 .. c0 + nc - 1,
// four per thread.  Eight slots are requested at once.
template <int ODT>
__global__ __launch_bounds__(256) void ffn_sum_kernel(FfnArgs a, FfnPlan p) {
  const int per = (p.nc / 4 + 255) / 256, t = blockIdx.x / per, n = (blockIdx.x % per * 256 + threadIdx.x) * 4;
  if (n >= p.nc || t >= a.T) return;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < a.k; j0 += 8) {
    f32x4 v[8];
    float w[8];
    bool on[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const size_t q = (size_t)t * a.k + min(j0 + j, a.k - 1);
      const int e = a.ids[q];
      on[j] = j0 + j < a.k && e >= 0 && e < a.E;
      w[j] = a.weights[q];
      if (on[j]) v[j] = *reinterpret_cast<const f32x4*>(p.y + q * p.nc + n);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (on[j])
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(w[j], v[j][i], o[i]);
  }
  const size_t c = p.c0 + n;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float u = o[i];
    if (a.res) u += load_elt<ODT>(a.res, (size_t)t * a.ldr + c + i);
    store_elt<ODT>(a.out, (size_t)t * a.ldo + c + i, u);
  }
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// (what the smallest row tile needs holds for all)
size_t ffn_tiles(int64_t P, int E, int BM) { return (size_t)(P / BM + std::min<int64_t>(P, E)); }
constexpr int MIN_BM = 32;

// Columns of the down products that are held at once: what stays in the 256 MB
// Infinity Cache between the product and its sum, in whole tiles.
constexpr size_t Y_BYTES = size_t(256) << 20;
int ffn_columns(int64_t P, int d) {
  const int64_t n = (int64_t)(Y_BYTES / 4) / P / 256 * 256;
  return (int)std::min<int64_t>(d, std::max<int64_t>(256, n));
}

// Bytes for the down products that are held: what any call with at most P pairs needs.
// (ffn_columns falls in steps, so that fewer pairs may hold more than P times its columns.
// A call in parts and an engine's smaller blocks lay out their own, fewer pairs in a
// workspace sized for the most.)  None with one expert per row: those are stored as they are made.
size_t ffn_held(size_t P, int k, int d) { return k == 1 ? 0 : std::min(P * d, std::max(Y_BYTES / 4, P * 256)) * 4; }

// Never falls as T grows: every part does not.
size_t ffn_workspace(int T, int E, int k, int d, int F, int dt) {
  const size_t P = (size_t)T * k;
  return align256(4) + align256(ffn_tiles(P, E, MIN_BM) * sizeof(ExpertTile)) + align256(P * 4) +
         align256(P * F * esz_of(dt)) + align256(ffn_held(P, k, d));
}

static FfnPlan ffn_plan(const FfnArgs& a) {
  const size_t P = (size_t)a.T * a.k;
  unsigned char* ws = a.ws;
  FfnPlan p;
  p.ntile = reinterpret_cast<int*>(ws); ws += align256(4);
  p.tile = reinterpret_cast<ExpertTile*>(ws); ws += align256(ffn_tiles(P, a.E, MIN_BM) * sizeof(ExpertTile));
  p.order = reinterpret_cast<int*>(ws); ws += align256(P * 4);
  p.z = ws; ws += align256(P * a.F * esz_of(a.dt));
  p.y = reinterpret_cast<float*>(ws);
  p.c0 = 0;
  p.nc = ffn_columns(P, a.d);
  return p;
}

// One expert per row: the rows that have none (the others' products are stored as
// they are made).
template <int ODT>
__global__ __launch_bounds__(256) void ffn_none_kernel(FfnArgs a) {
  const int t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.T) return;
  const int e = a.ids[t];
  if (e >= 0 && e < a.E) return;
  for (int n = threadIdx.x & 63; n < a.d; n += 64) {
    const float u = a.res ? 0.f + load_elt<ODT>(a.res, (size_t)t * a.ldr + n) : 0.f;
    store_elt<ODT>(a.out, (size_t)t * a.ldo + n, u);
  }
}

template <int DT, int ODT, int BM, int BN, int WR, int WF, int NST>
static hipError_t ffn_tiles_t(TileArgs t, hipStream_t st) {
  hipError_t e = launch_tile<DT, TM_UP, BM, BN, WR, WF, NST>(t, st);
  if (t.f.k == 1) {   // (8192 rows of 2 experts, 96 over 3776: 145 us with the products held and joined, 85 so)
    t.p.nc = t.f.d;
    if (e == hipSuccess) e = launch_tile<DT, TM_DOWN, BM, BN, WR, WF, NST>(t, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((ffn_none_kernel<ODT>), dim3((unsigned)((t.f.T + 3) / 4)), dim3(256), 0, st, t.f);
    return hipGetLastError();
  }
  const int nc = t.p.nc;
  for (t.p.c0 = 0; t.p.c0 < t.f.d && e == hipSuccess; t.p.c0 += nc) {
    t.p.nc = std::min(nc, t.f.d - t.p.c0);
    if ((e = launch_tile<DT, TM_DOWN, BM, BN, WR, WF, NST>(t, st)) != hipSuccess) break;
    hipLaunchKernelGGL((ffn_sum_kernel<ODT>), dim3((unsigned)((t.p.nc / 4 + 255) / 256) * t.f.T), dim3(256), 0, st, t.f, t.p);
    e = hipGetLastError();
  }
  return e;
}

template <int DT, int ODT>
static hipError_t ffn_t(const FfnArgs& a, hipStream_t st) {
  const int64_t P = (int64_t)a.T * a.k;
  hipError_t e;
  FfnPlan pl = ffn_plan(a);
  // Few pairs: each streams its expert's weights for itself, which spares the
  // sorting and one launch, some 10 us, unless the pairs share experts so
  // far that reading those again takes longer (64 MB of them).  With every expert
  // as likely, P pairs meet E (1 - (1 - 1 / E)^P).
  const double distinct = a.E * (1.0 - pow(1.0 - 1.0 / a.E, (double)P));
  const double again = ((double)P - distinct) * 3.0 * a.d * a.F * esz_of(DT);
  if (P <= 256 && again <= double(64 << 20)) {
    const int ub = a.F / 16, db = a.d / 16;
    hipLaunchKernelGGL((ffn_up_kernel<DT>), dim3((unsigned)ub * P), dim3(64), 0, st, a, pl.z, ub);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((ffn_down_kernel<DT, ODT>), dim3((unsigned)db * a.T), dim3(DOWN_WAVES * 64), 0, st, a, (const void*)pl.z, db);
    return hipGetLastError();
  }
  // The tile whose turns of the chip take least, as for a linear (row tiles: every
  // expert that is met ends in half a tile on average, so whether a last turn
  // is begun is even); with fewer than eight rows per expert the weights' stream
  // is all, and the smallest does best.  128 experts of 768 over 2048, 8 per row, tiles
  // of 32 x 64 / 64 x 256 / 128 x 256: 33 rows 205 / 210 / 213 us, 257 236 / 238 / 243, 513
  // 297 / 250 / 256, 1025 394 / 311 / 280, 4096 1087 / 674 / 555; 8 experts of 352 over
  // 256, 2 per row, 257 rows 18.5 / 20.4 / 21.8, 8192 59 / 52 / 44; 8 of 2048 over 1024, 1000
  // rows 81 / 67 / 70.  In fp32 the matrix instructions bound the tiles (8 experts of
  // 1024 over 512, 2 per row, 1000 rows: 64 x 256 81 us, 128 x 256 141).
  auto cost = [&](int BM, int BN, double turn) {
    const double rt = std::max(distinct, (double)P / BM + distinct / 2);
    auto turns = [&](int cols) {
      const double n = rt * ((cols + BN - 1) / BN) / 256.0;
      return std::max(1.0, (n + ceil(n)) / 2);
    };
    return turn * (turns(2 * a.F) * a.d + turns(a.d) * a.F);
  };
  const bool f32 = DT == DT_F32;
  const double c0 = cost(32, 64, f32 ? 39 : 9), c1 = cost(64, 256, f32 ? 240 : 30), c2 = cost(128, 256, f32 ? 470 : 40);
  const int BM = P < 8 * a.E || (c0 <= c1 && c0 <= c2) ? 32 : c1 <= c2 ? 64 : 128;
  TileArgs t{};
  t.f = a;
  t.p = pl;
  t.nrt = (int)ffn_tiles(P, a.E, BM);
  const int chunk = plan_chunk(P);
  hipLaunchKernelGGL(ffn_plan_kernel, dim3((unsigned)((P + chunk - 1) / chunk)), dim3(PLAN_THREADS), 0, st, a.ids, (int)P, chunk, a.E, BM, pl);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (BM == 32) return ffn_tiles_t<DT, ODT, 32, 64, 2, 2, 4>(t, st);
  if (BM == 64) return ffn_tiles_t<DT, ODT, 64, 256, 1, 8, 3>(t, st);
  return ffn_tiles_t<DT, ODT, 128, 256, 2, 4, 3>(t, st);
}

hipError_t run_ffn(const FfnArgs& a, hipStream_t st) {
  // The tile kernels gather rows of x at 32-bit offsets: inputs of 4 GiB and
  // more run in parts (on the same workspace, one after another).
  const int64_t row = a.ldx * esz_of(a.dt);
  const int most = (int)std::min<int64_t>(a.T, (int64_t(1) << 32) / row - 1);
  for (int t = 0; t < a.T; t += most) {
    FfnArgs b = a;
    b.T = std::min(most, a.T - t);
    b.x = reinterpret_cast<const unsigned char*>(a.x) + (size_t)t * row;
    b.ids = a.ids + (size_t)t * a.k;
    b.weights = a.weights + (size_t)t * a.k;
    b.out = reinterpret_cast<unsigned char*>(a.out) + (size_t)t * a.ldo * esz_of(a.odt);
    if (a.res) b.res = reinterpret_cast<const unsigned char*>(a.res) + (size_t)t * a.ldr * esz_of(a.odt);
    const hipError_t e = a.dt == DT_F32     ? ffn_t<DT_F32, DT_F32>(b, st)
                         : a.odt == DT_F32 ? ffn_t<DT_BF16, DT_F32>(b, st)
                                           : ffn_t<DT_BF16, DT_BF16>(b, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ee
