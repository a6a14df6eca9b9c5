// gfx950 kernels of the operators around a paged key-value cache of the caller's:
// appending rows to it, with the rotation of positions applied on the way, and
// attention of every sequence's newest rows over its pages.
//
// Arithmetic of attention (a row's bits depend on the row, its sequence's pages
// and its number of positions alone, not on the batch, the rows beside it or the
// tables' width):
//   * positions in chunks of 256 of four runs of 64 each, counted from position 0.
//     A run's state is m = its largest score (times log2 e), l = sum 2^(s - m) and
//     o = sum 2^(s - m) v, from nothing;
//   * a chunk's state takes its runs' in one after another: m' = max(m, m_r),
//     o' = fma(o_r, 2^(m_r - m'), o 2^(m - m')), l alike;
//   * a row's result adds its chunks' states, each times 2^(m - M) for the largest m, in a
//     fixed order.
// Scores, weights, l and o are fp32.  The matrix instruction of a bf16 cache takes
// the weights as two bf16 parts (p = hi + lo to 2^-17): as one they would add as much error as
// the rounding of a bf16 result, and half the chip's matrix rate waits on the cache anyway.

#include "operators.h"

#include <limits.h>
#include <math.h>

#include <algorithm>
#include <array>
#include <type_traits>

#include "device.h"

namespace ee {

// ------------------------------------------------------------------- append --

// One workgroup per row: rotation factors into LDS once, then the row's heads in
// pieces of 16 bytes.
constexpr int APPEND_THREADS = 256;

// The values of a 16-byte piece, and back.
template <int DT> __device__ __forceinline__ void unpack(uint4 u, float (&f)[Geo<DT>::EPL]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if constexpr (DT == DT_BF16) {
      f[2 * i] = bf2f(w[i] & 0xffffu);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      f[i] = __uint_as_float(w[i]);
    }
}
template <int DT> __device__ __forceinline__ uint4 pack(const float (&f)[Geo<DT>::EPL]) {
  if constexpr (DT == DT_BF16)
    return make_uint4(bf16x2_bits(f[0], f[1]), bf16x2_bits(f[2], f[3]), bf16x2_bits(f[4], f[5]), bf16x2_bits(f[6], f[7]));
  else
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

template <int DT>
__global__ __launch_bounds__(APPEND_THREADS) void append_kernel(AppendArgs a) {
  constexpr int EPL = Geo<DT>::EPL, ESZ = Geo<DT>::ESZ;
  __shared__ float2 cs[MAX_HEAD_DIM / 2];
  const int r = blockIdx.x, half = a.rot / 2;
  const int pos = a.positions[r];
  for (int i = threadIdx.x; i < half; i += APPEND_THREADS) {
    // (turns in float64, whole ones dropped there: a float32 angle of position 100000 is
    // off by 2^-8 of a radian)
    const double turns = (double)pos * a.inv_freq[i] * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[i] = make_float2(c, s);
  }
  // the row's slot; none where it names no sequence, position or page that there is
  const int seq = a.seqs ? a.seqs[r] : r / a.per_seq;
  const PagedCache& c = a.c;
  bool slot = seq >= 0 && seq < a.B && pos >= 0 && pos / c.page < c.max_pages;
  int page = -1;
  if (slot) page = c.tables[seq * c.ldt + pos / c.page];
  slot = slot && page >= 0 && page < c.n_pages;
  const int at = slot ? pos % c.page : 0;
  page = slot ? page : 0;
  uint8_t* kc = (uint8_t*)c.k + (page * c.kp + at * c.ks) * ESZ;
  uint8_t* vc = (uint8_t*)c.v + (page * c.vp + at * c.vs) * ESZ;
  const uint8_t* q = (const uint8_t*)a.q + r * a.ldq * ESZ;
  const uint8_t* k = (const uint8_t*)a.k + r * a.ldk * ESZ;
  const uint8_t* v = (const uint8_t*)a.v + r * a.ldv * ESZ;
  uint8_t* qo = (uint8_t*)a.q_out + r * a.ldqo * ESZ;
  __syncthreads();
  const int ppr = a.hd / EPL;                    // pieces of a head
  const int hp = half / EPL;                     // pieces of a rotated half
  const int rest = ppr - 2 * hp;                 // pieces behind the rotated ones
  const int work = hp + rest;                    // a thread rotates a piece of either half, or copies one
  const int heads = (a.q ? a.H : 0) + a.Hkv;
  for (int i = threadIdx.x; i < heads * work; i += APPEND_THREADS) {
    const int h = i / work, p = i % work;
    const bool key = h < a.Hkv;
    const uint8_t* src = key ? k + h * a.hd * ESZ : q + (h - a.Hkv) * a.hd * ESZ;
    uint8_t* dst = key ? kc + h * c.kh * ESZ : qo + (h - a.Hkv) * a.hd * ESZ;
    const bool store = !key || slot;
    if (p >= hp) {
      const int o = (p + hp) * 16;
      if (store) *(uint4*)(dst + o) = *(const uint4*)(src + o);
      continue;
    }
    // Interleaved pairs are within a piece; halves are `half` dimensions apart.
    const int o0 = (a.interleaved ? 2 * p : p) * 16, o1 = (a.interleaved ? 2 * p + 1 : p + hp) * 16;
    float x[EPL], y[EPL];
    unpack<DT>(*(const uint4*)(src + o0), x);
    unpack<DT>(*(const uint4*)(src + o1), y);
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < EPL; e += 2) {
        const float2 f = cs[p * EPL + e / 2], g = cs[p * EPL + EPL / 2 + e / 2];
        const float x0 = x[e], x1 = x[e + 1], y0 = y[e], y1 = y[e + 1];
        x[e] = x0 * f.x - x1 * f.y;
        x[e + 1] = x0 * f.y + x1 * f.x;
        y[e] = y0 * g.x - y1 * g.y;
        y[e + 1] = y0 * g.y + y1 * g.x;
      }
    } else {
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const float2 f = cs[p * EPL + e];
        const float x0 = x[e], y0 = y[e];
        x[e] = x0 * f.x - y0 * f.y;
        y[e] = x0 * f.y + y0 * f.x;
      }
    }
    if (store) {
      *(uint4*)(dst + o0) = pack<DT>(x);
      *(uint4*)(dst + o1) = pack<DT>(y);
    }
  }
  if (slot)
    for (int i = threadIdx.x; i < a.Hkv * ppr; i += APPEND_THREADS) {
      const int h = i / ppr, o = i % ppr * 16;
      *(uint4*)(vc + h * c.vh * ESZ + o) = *(const uint4*)(v + h * a.hd * ESZ + o);
    }
}

hipError_t run_append(const AppendArgs& a, hipStream_t st) {
  if (a.dt == DT_BF16) hipLaunchKernelGGL((append_kernel<DT_BF16>), dim3(a.R), dim3(APPEND_THREADS), 0, st, a);
  else hipLaunchKernelGGL((append_kernel<DT_F32>), dim3(a.R), dim3(APPEND_THREADS), 0, st, a);
  return hipGetLastError();
}

// ---------------------------------------------------------------- attention --

constexpr int RUN = 64, RUNS = 4, CHUNK = RUN * RUNS;   // positions of a run, runs of a chunk
constexpr int COLS = 16;                                // a tile's columns: (row, query head of the group) pairs
static_assert(CHUNK == ATTEND_CHUNK && RUNS * 64 == COLS * 16, "");

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Geometry of a wave over a run of HD dimensions.
//   scores: keys are the matrix instruction's A operand (16 positions, a lane has
//     16 bytes of one key), queries B; lane (grp, c) gets positions 4 grp + r of
//     each tile for column c;
//   values: the weights as they then stand are an A operand whose reduction slots of
//     lane group grp are the positions that lane holds, so V is loaded in
//     that order: lane (grp, c) takes the same positions' values of dimensions
//     c EPV ... of every pass.  bf16 values are transposed in registers, 8
//     positions by the dimensions of a piece; the output's lane (grp, c) then
//     holds columns 4 grp + r, dimensions (pass, c EPV + e).
// Keys, values and weights never pass through LDS.
template <int DT, int HD> struct AttGeo {
  static constexpr int ESZ = Geo<DT>::ESZ, EPL = Geo<DT>::EPL, KS = Geo<DT>::KS;
  static constexpr int NS = HD / KS;                         // fragments of a key
  static constexpr int EPV = HD / 16 < EPL ? HD / 16 : EPL;  // dimensions of a lane's piece of V
  static constexpr int NP = HD / 16 / EPV;                   // passes over the dimensions
  static constexpr int VK = DT == DT_BF16 ? 8 : 4;           // positions of a lane in a step of V
  static constexpr int SP = VK * 4;                          // positions of a step
  static constexpr int STEPS = RUN / SP;
  static constexpr int ND = HD / 16;                         // output tiles
  // Whether a wave's registers hold a run's keys and values beside the rest: the next
  // run's are then requested as soon as this one's are used.
  static constexpr bool AHEAD = HD * ESZ <= 256;
  using Piece = std::conditional_t<EPV * ESZ == 16, uint4, uint2>;
};
template <class P> __device__ __forceinline__ uint32_t word(const P& p, int i) { return __builtin_bit_cast(std::array<uint32_t, sizeof(P) / 4>, p)[i]; }


// A state takes in a later run's.
__device__ __forceinline__ float join_scale(float m, float M) { return M == -INFINITY ? 1.f : exp2_(m - M); }   // (of two empty ones: as they are)

// Longest sequences first, 64 at a time, so that short ones fill the gaps at the end (64
// sequences to 8192, 32 heads over 8 of 128: 228 us, 274 in their own order): the i-th to be taken.
__device__ __forceinline__ int by_length(const int* lens, int B, int i, int lane) {
  if (B == 1) return 0;
  const int b64 = i & ~63, n = min(64, B - b64), own = lane < n ? lens[b64 + lane] : INT_MIN;
  int rank = 0;
  for (int j = 0; j < n; ++j) {
    const int other = __builtin_amdgcn_readlane(own, j);
    rank += other > own || (other == own && j < lane);
  }
  return b64 + __ffsll(__ballot(lane < n && rank == (i & 63))) - 1;
}

// What a wave streams: the pages, keys and values of runs of one KV head.
template <int DT, int HD> struct Stream {
  using G = AttGeo<DT, HD>;
  static constexpr int ESZ = G::ESZ;
  const PagedCache& pc;
  const int* table;
  const uint8_t *kh, *vh;   // the head's
  uint64_t page_mul;
  int start, e_hi;          // positions that some row sees
  int lane, c, grp;
  int entries, entry0, entry_step;
  // Pages of a run's four 16-position tiles, -1 where there is none or no row sees it: lane
  // 4 i + j holds that of tile j of the run i turns on, for sixteen turns.  (As loads by
  // the whole wave in the loop they waited for the keys and values before them.)
  struct Pages {
    int page[4], at[4];
  };
  uint4 k[4][G::NS];
  typename G::Piece v[G::STEPS][G::NP][G::VK];

  __device__ __forceinline__ int page_of(int p0) const { return (int)(((uint64_t)(uint32_t)(p0 >> 4) * page_mul) >> 38); }
  // Turns are `step` positions apart, the first at p.
  __device__ __forceinline__ void entries_load(int64_t p, int64_t step, int inner, int64_t inner_step) {
    const int turn = lane >> 2;
    const int64_t p0 = p + turn / inner * step + turn % inner * inner_step + 16 * (lane & 3);
    entries = p0 < (int64_t)pc.max_pages * pc.page ? table[page_of((int)p0)] : -1;
  }
  __device__ __forceinline__ void entries_wait() { asm volatile("" : "+v"(entries)); }   // (here, not wherever they are used)
  __device__ __forceinline__ Pages pages(int turn, int base) const {
    Pages p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p0 = base + 16 * i, page = __builtin_amdgcn_readlane(entries, turn * 4 + i);
      p.page[i] = page >= 0 && page < pc.n_pages && p0 < e_hi && p0 + 16 > start ? page : -1;
      p.at[i] = p0 - page_of(p0) * pc.page;
    }
    return p;
  }
  __device__ __forceinline__ void load_k(const Pages& p) {
    const unsigned off = (unsigned)(c * (int)pc.ks * ESZ + grp * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto r = make_rsrc(kh + (max(p.page[i], 0) * pc.kp + p.at[i] * pc.ks) * ESZ, p.page[i] >= 0 ? 0x7fffffffu : 0u);
#pragma unroll
      for (int f = 0; f < G::NS; ++f) k[i][f] = bload<0>(r, off + f * 64);
    }
  }
  // Values of a lane's positions; zeros where no row sees the position (what its slot holds may
  // be no number): past the last one by the range of the tile, before the first by the offset.
  __device__ __forceinline__ void load_v(const Pages& p, int base) {
    const unsigned slot = (unsigned)((int)pc.vs * ESZ);
#pragma unroll
    for (int tile = 0; tile < 4; ++tile) {
      const unsigned last = (unsigned)min(e_hi - (base + 16 * tile), 16) - 1u;
      const auto r = make_rsrc(vh + (max(p.page[tile], 0) * pc.vp + p.at[tile] * pc.vs) * ESZ, p.page[tile] >= 0 ? last * slot + HD * ESZ : 0u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // slot j of lane group grp: position 4 grp + j of the step's first tile, then of its second
        const int st = tile / (G::SP / 16), j = tile % (G::SP / 16) * 4 + i;
        const unsigned off = ((4 * grp + i) * slot + c * G::EPV * ESZ) | ((unsigned)(base - start + 16 * tile + i + 4 * grp) & OOB);
#pragma unroll
        for (int np = 0; np < G::NP; ++np)
          if constexpr (G::EPV * ESZ == 16) v[st][np][j] = bload<0>(r, off + np * 256);
          else v[st][np][j] = bload64<0>(r, off);
      }
    }
  }
  // Scores of a lane's column, as weights: m, l and s = 2^(s - m).
  __device__ __forceinline__ void scores(const uint4 (&q)[G::NS], f32x4 (&s)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int f = 0; f < G::NS; ++f) s[i] = mma<DT>(k[i][f], q[f], s[i]);
    }
  }
  // whole: every column sees the run.
  __device__ __forceinline__ void weights(const Pages& p, int base, int first, int end, bool whole, float scale, f32x4 (&s)[4], float& m, float& l) const {
    m = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[i][r] *= scale;
    if (!whole || (p.page[0] | p.page[1] | p.page[2] | p.page[3]) < 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int pos = base + 16 * i + 4 * grp + r;
          if (!(p.page[i] >= 0 && pos < end && pos >= first)) s[i][r] = -INFINITY;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) m = fmaxf(m, s[i][r]);
    m = xmax32(xmax16(m));
    const float mu = m == -INFINITY ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[i][r] = exp2_(s[i][r] - mu);
        l += s[i][r];
      }
    l = xsum32(xsum16(l));
  }
  // Operand word j of dimension d: a pair of positions, from pairs of dimensions of one position.
  __device__ __forceinline__ uint32_t turned(int st, int d, int j) const {
    if constexpr (DT == DT_F32) {
      return word(v[st][d / 4][j], d % 4);
    } else {
      const int np = d / G::EPV, w = d % G::EPV / 2;
      const uint32_t x = word(v[st][np][2 * j], w), y = word(v[st][np][2 * j + 1], w);
      return d & 1 ? __builtin_amdgcn_perm(y, x, 0x07060302u) : __builtin_amdgcn_perm(y, x, 0x05040100u);
    }
  }
};
// The weights of a step of V as an operand: bf16 in two parts.
template <int DT> struct Weights {
  uint4 hi, lo;
};
template <int DT> __device__ __forceinline__ Weights<DT> operand_weights(const f32x4 (&s)[4], int st) {
  Weights<DT> w;
  if constexpr (DT == DT_BF16) {
    uint32_t u[4], v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = s[2 * st + (j >> 1)][2 * (j & 1)], y = s[2 * st + (j >> 1)][2 * (j & 1) + 1];
      u[j] = bf16x2_bits(x, y);
      v[j] = bf16x2_bits(x - bf2f(u[j] & 0xffffu), y - __uint_as_float(u[j] & 0xffff0000u));
    }
    w.hi = make_uint4(u[0], u[1], u[2], u[3]);
    w.lo = make_uint4(v[0], v[1], v[2], v[3]);
  } else {
    w.hi = __builtin_bit_cast(uint4, s[st]);
  }
  return w;
}
// acc[d] += weights x values of a step, x(d) the values of dimension tile d.  (A tile's two
// parts apart, so that neither waits for the other.)
template <int DT, int ND, class X> __device__ __forceinline__ void weigh(const Weights<DT>& w, X x, f32x4 (&acc)[ND]) {
#pragma unroll
  for (int d0 = 0; d0 < ND; d0 += 4) {
    uint4 y[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] = x(d0 + d);
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d0 + d] = mma<DT>(w.hi, y[d], acc[d0 + d]);
    if constexpr (DT == DT_BF16)
#pragma unroll
      for (int d = 0; d < 4; ++d) acc[d0 + d] = mma<DT>(w.lo, y[d], acc[d0 + d]);
  }
}

// Whether some sum of weights and values is no number.  Finite values leave numbers whatever the
// weights, so only then is the sum formed again with care: a weight of 0 does not remove an infinity or NaN
// that a row does not see, and an infinite value is left to the upper part of its weight, since the
// lower one may be 0 or of the other sign.  (16 instructions a run of head_dim 128; looking
// at the values instead took 33 rows of 4 sequences to 4096 43 us, 37.5 so.)
template <int ND> __device__ __forceinline__ bool no_number(const f32x4 (&o)[ND]) {
  float most = 0.f;   // (a maximum that NaN goes through)
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 4; r += 2) most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(most, o[d][r]), o[d][r + 1]);
  return __ballot(most != most) != 0;
}
// The word of a pair of bf16 values without its infinities.
__device__ __forceinline__ uint32_t without_infinities(uint32_t y) {
  return y & (((y & 0x7fffu) == 0x7f80u ? 0u : 0xffffu) | ((y & 0x7fff0000u) == 0x7f800000u ? 0u : 0xffff0000u));
}
template <int DT> __device__ __forceinline__ f32x4 weigh_careful(const Weights<DT>& w, const uint32_t (&y)[4], f32x4 acc) {   // (in the order of weigh)
  acc = mma<DT>(w.hi, make_uint4(y[0], y[1], y[2], y[3]), acc);
  if constexpr (DT == DT_BF16)
    acc = mma<DT>(w.lo, make_uint4(without_infinities(y[0]), without_infinities(y[1]), without_infinities(y[2]), without_infinities(y[3])), acc);
  return acc;
}

// One row per sequence.  What bounds it is the cache's stream (64 sequences up to 8192, 32
// heads over 8 of 128: 1.07 GB): a wave takes a KV head's chunks split, split + splits, ...
// of a sequence, run after run, and requests the next run's keys and values as soon
// as this one's are used.  The waves of a workgroup take a sequence's heads side by side, which
// stand next to each other where a position's heads do (read so 6.2 TB/s, a head per
// workgroup 5.5), and wait for nothing of each other.
// (Four waves with all of a SIMD's registers each where a run's keys and values take more.)
template <int DT, int HD> constexpr int stream_waves() { return AttGeo<DT, HD>::AHEAD ? 8 : 4; }
template <int DT, int HD>
__global__ __launch_bounds__((stream_waves<DT, HD>() * 64), (stream_waves<DT, HD>() / 4)) void attend_stream_kernel(AttendArgs a) {
  using G = AttGeo<DT, HD>;
  constexpr int ESZ = G::ESZ, STREAM_WAVES = stream_waves<DT, HD>();
  __shared__ uint4 sq[STREAM_WAVES][G::NS][64];   // the queries' fragments
  const PagedCache& pc = a.c;
  const int lane = threadIdx.x & 63, c = lane & 15, grp = lane >> 4;
  const int unit = __builtin_amdgcn_readfirstlane((int)blockIdx.x * STREAM_WAVES + (int)(threadIdx.x >> 6));
  const int per = a.Hkv * a.cgroups, share = unit / per, h = unit % per / a.cgroups, ct = unit % a.cgroups;
  if (share >= a.splits * a.B) return;
  const int split = share % a.splits, b = by_length(a.lens, a.B, share / a.splits, lane);
  const int len = max(min(max(a.lens[b], 0), pc.max_pages * pc.page) - a.behind, 0), start = a.window ? max(0, len - a.window) : 0;
  const int ch1 = (len + CHUNK - 1) / CHUNK;
  int ch = start / CHUNK + split, run0 = 0, runs = RUNS;
  // Few chunks for the waves that share them (tables much wider than the sequence): a run each, joined
  // by what reads the states (a sequence of 2048 in tables for 65536: 14 us, 27.5 by chunks).
  if (ch1 - start / CHUNK <= a.apart) {
    ch = start / CHUNK + split / RUNS;
    run0 = split % RUNS;
    runs = 1;
  }
  if (ch >= ch1) return;
  const int ncol = min(COLS, a.G - ct * COLS), col = min(ct * COLS + c, a.G - 1);   // (columns past the last repeat it)

  Stream<DT, HD> x{pc, pc.tables + b * pc.ldt, (const uint8_t*)pc.k + h * pc.kh * ESZ, (const uint8_t*)pc.v + h * pc.vh * ESZ, a.page_mul, start, len, lane, c, grp};
  auto entries = [&](int chunk) { x.entries_load((int64_t)chunk * CHUNK, (int64_t)a.splits * CHUNK, RUNS, RUN); };   // of four chunks
  entries(ch);   // (on its way with the queries)
  uint4 (&qs)[G::NS][64] = sq[threadIdx.x >> 6];   // (the wave's own: no barrier)
  const uint8_t* qp = (const uint8_t*)a.q + ((int64_t)b * a.ldq + (h * a.G + col) * HD) * ESZ + grp * 16;
#pragma unroll
  for (int f = 0; f < G::NS; ++f) qs[f][lane] = *(const uint4*)(qp + f * 64);
  x.entries_wait();
  int ahead = 0;   // chunks on since then
  typename Stream<DT, HD>::Pages now = x.pages(run0, ch * CHUNK + run0 * RUN), next;
  if constexpr (G::AHEAD) {
    x.load_k(now);
    x.load_v(now, ch * CHUNK + run0 * RUN);
  }
  // A chunk's state takes in a run's.
  auto take_in = [&](bool first, const f32x4 (&one)[G::ND], float mr, float lr, f32x4 (&o)[G::ND], float& m, float& l) {
    if (first) {
      m = mr;
      l = lr;
#pragma unroll
      for (int i = 0; i < G::ND; ++i) o[i] = one[i];
    } else {
      // m, l and the scales belong to column c, the values to columns 4 grp + r
      const float M = fmaxf(m, mr), fa = join_scale(m, M), fb = join_scale(mr, M);
      l = fmaf(lr, fb, l * fa);
      m = M;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float ra = __shfl(fa, 4 * grp + r), rb = __shfl(fb, 4 * grp + r);
#pragma unroll
        for (int i = 0; i < G::ND; ++i) o[i][r] = fmaf(one[i][r], rb, o[i][r] * ra);
      }
    }
  };
  for (; ch < ch1; ch += a.splits) {
    f32x4 o[G::ND];
    float m = -INFINITY, l = 0.f;
    for (int run = run0; run < run0 + runs; ++run) {
      const int base = ch * CHUNK + run * RUN;
      if constexpr (!G::AHEAD) {
        x.load_k(now);
        x.load_v(now, base);
      }
      // (past the last chunk there are no pages, and requests read nothing: a condition
      // around them would make the compiler wait for more than the oldest)
      int after = base + RUN;
      if (run == run0 + runs - 1) {
        after = (ch + a.splits) * CHUNK;
        if (++ahead == 4) {
          entries(ch + a.splits);
          x.entries_wait();
          ahead = 0;
        }
      }
      next = x.pages(ahead * RUNS + (run + 1) % RUNS, after);
      f32x4 s[4];
      {
        uint4 q[G::NS];
#pragma unroll
        for (int f = 0; f < G::NS; ++f) q[f] = qs[f][lane];
        x.scores(q, s);
      }
      if constexpr (G::AHEAD) x.load_k(next);
      float mr, lr;
      x.weights(now, base, start, len, base >= start && base + RUN <= len, a.scale_log2, s, mr, lr);
      f32x4 one[G::ND];
#pragma unroll
      for (int i = 0; i < G::ND; ++i) one[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < G::STEPS; ++st)
        weigh<DT>(operand_weights<DT>(s, st), [&](int d) { return make_uint4(x.turned(st, d, 0), x.turned(st, d, 1), x.turned(st, d, 2), x.turned(st, d, 3)); }, one);
      if constexpr (G::AHEAD) x.load_v(next, after);
      take_in(run == run0, one, mr, lr, o, m, l);
      now = next;
    }
    if constexpr (DT == DT_BF16)
      if (__builtin_expect(no_number(o), 0)) {   // the chunk once more, then the next one's requests
        entries(ch);
        x.entries_wait();
        for (int run = run0; run < run0 + runs; ++run) {
          const int base = ch * CHUNK + run * RUN;
          const typename Stream<DT, HD>::Pages p = x.pages(run, base);
          x.load_k(p);
          x.load_v(p, base);
          uint4 q[G::NS];
#pragma unroll
          for (int f = 0; f < G::NS; ++f) q[f] = qs[f][lane];
          f32x4 s[4];
          x.scores(q, s);
          float mr, lr;
          x.weights(p, base, start, len, false, a.scale_log2, s, mr, lr);
          f32x4 one[G::ND];
#pragma unroll
          for (int d = 0; d < G::ND; ++d) {
            one[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < G::STEPS; ++st) {
              const uint32_t y[4] = {x.turned(st, d, 0), x.turned(st, d, 1), x.turned(st, d, 2), x.turned(st, d, 3)};
              one[d] = weigh_careful<DT>(operand_weights<DT>(s, st), y, one[d]);
            }
          }
          take_in(run == run0, one, mr, lr, o, m, l);
        }
        entries(ch + a.splits * (1 - ahead));
        x.entries_wait();
        if constexpr (G::AHEAD) {
          x.load_k(now);
          x.load_v(now, (ch + a.splits) * CHUNK);
        }
      }
    const int64_t state = ((int64_t)(b * a.ring + (runs == 1 ? split : ch % a.ring)) * a.Hkv + h) * a.G + ct * COLS;
    if (grp == 0 && c < ncol) a.ml[state + c] = make_float2(m, l);
    // o[np EPV + e] of lane (grp, c): columns 4 grp + r, dimension np 16 EPV + c EPV + e
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (4 * grp + r < ncol)
#pragma unroll
        for (int np = 0; np < G::NP; ++np)
#pragma unroll
          for (int e = 0; e < G::EPV; e += 4)
            *(f32x4*)(a.o + (state + 4 * grp + r) * HD + np * 16 * G::EPV + c * G::EPV + e) =
                f32x4{o[np * G::EPV + e][r], o[np * G::EPV + e + 1][r], o[np * G::EPV + e + 2][r], o[np * G::EPV + e + 3][r]};
  }
}

// Several rows per sequence, or one where there are few chunks (8 KV heads of 128, one row of a
// sequence of 8192: 18 us so, 32 by the waves above; of 32768 37 and 39; of 65536 65 and
// 58).  The four waves of a workgroup take the runs of a chunk, whose states they
// join through LDS, and keep its keys and values in registers for all of the workgroup's
// column tiles (read anew for each, 33 rows of 4 sequences to 4096 took 88 us; so 59 as first built, 37 now).
// Some of them stand in scratch: 18 registers of a bf16 cache with head_dim 128 and several
// tiles, 6 with 256; the keys and values of an fp32 run of 256 do not fit a wave (394 registers, 132
// in the kernel above).
constexpr int att_tiles(int row_bytes) { return std::max(1, 32768 / (COLS * row_bytes)); }   // whose queries LDS holds
// For one column tile the next run's are requested ahead; for several, two workgroups share a
// CU instead, each working while the other waits (33 rows 38.7 us, 52 with one).
template <int DT, int HD, bool SEVERAL>
__global__ __launch_bounds__(RUNS * 64, SEVERAL ? 2 : 1) void attend_rows_kernel(AttendArgs a) {
  using G = AttGeo<DT, HD>;
  constexpr int ESZ = G::ESZ, BUFFERS = SEVERAL || HD > 128 ? 1 : 2;   // of runs' states
  constexpr bool AHEAD = G::AHEAD && !SEVERAL;
  const PagedCache& pc = a.c;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, grp = lane >> 4;
  __shared__ float sm[BUFFERS][RUNS][COLS], sl[BUFFERS][RUNS][COLS];
  __shared__ __attribute__((aligned(16))) float so[BUFFERS][RUNS][COLS][HD];
  __shared__ uint4 sq[att_tiles(HD * ESZ)][G::NS][64];   // the queries' fragments

  // Workgroups are dealt to the eight XCDs in turn: all heads and column tiles of a share of a
  // sequence's length go to one, whose L2 then has what several ask for.
  const int per = a.Hkv * a.cgroups, turn = (int)(blockIdx.x >> 3);
  const int share = turn / per * 8 + (int)(blockIdx.x & 7), h = turn % per / a.cgroups, cg = turn % a.cgroups;
  if (share >= a.splits * a.B) return;
  const int split = share % a.splits, b = by_length(a.lens, a.B, share / a.splits, lane);
  const int cols = a.T * a.G, len = min(max(a.lens[b], 0), pc.max_pages * pc.page) - a.behind;
  const int ct0 = cg * a.ctw, ct1 = min(ct0 + a.ctw, (cols + COLS - 1) / COLS);   // column tiles
  const int before = len - a.T + 1;                                              // the end of row 0
  const int e_lo = before + ct0 * COLS / a.G, e_hi = before + (min(ct1 * COLS, cols) - 1) / a.G;   // of the first and last row
  if (e_hi <= 0) return;
  const int start = a.window ? max(0, e_lo - a.window) : 0;
  const int ch1 = (e_hi + CHUNK - 1) / CHUNK;
  int ch = start / CHUNK + split;
  if (ch >= ch1) return;

  Stream<DT, HD> x{pc, pc.tables + b * pc.ldt, (const uint8_t*)pc.k + h * pc.kh * ESZ, (const uint8_t*)pc.v + h * pc.vh * ESZ, a.page_mul, start, e_hi, lane, c, grp};
  auto entries = [&](int chunk) { x.entries_load((int64_t)chunk * CHUNK + wv * RUN, (int64_t)a.splits * CHUNK, 1, 0); };
  entries(ch);   // (on its way with the queries)
  for (int i = wv; i < (ct1 - ct0) * G::NS; i += RUNS) {
    const int ct = i / G::NS, f = i % G::NS, col = min((ct0 + ct) * COLS + c, cols - 1);   // (columns past the last repeat it)
    sq[ct][f][lane] = *(const uint4*)((const uint8_t*)a.q + ((int64_t)(b * a.T + col / a.G) * a.ldq + (h * a.G + col % a.G) * HD) * ESZ + grp * 16 + f * 64);
  }
  x.entries_wait();
  int ahead = 0;
  typename Stream<DT, HD>::Pages now = x.pages(0, ch * CHUNK + wv * RUN), next;
  x.load_k(now);
  x.load_v(now, ch * CHUNK + wv * RUN);
  __builtin_amdgcn_s_waitcnt(0xc07f);
  barrier_only();
  int buf = 0;
  for (; ch < ch1; ch += a.splits) {
    const int base = ch * CHUNK + wv * RUN, after = base + a.splits * CHUNK;
    // (past the last chunk there are no pages, and requests read nothing)
    if (++ahead == 16) {
      entries(ch + a.splits);
      x.entries_wait();
      ahead = 0;
    }
    next = x.pages(ahead, after);
    // The values turned once for all tiles; their registers take the next run's.
    uint32_t vt[G::STEPS][G::ND][4];
#pragma unroll
    for (int st = 0; st < G::STEPS; ++st)
#pragma unroll
      for (int d = 0; d < G::ND; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) vt[st][d][j] = x.turned(st, d, j);
    if constexpr (AHEAD) x.load_v(next, after);
    const bool whole = base + RUN <= e_lo && base >= (a.window ? max(0, e_hi - a.window) : 0);
    for (int ct = ct0; ct < ct1; ++ct, buf ^= BUFFERS - 1) {
      const int ncol = min(COLS, cols - ct * COLS), t = min(ct * COLS + c, cols - 1) / a.G;
      const int end = before + t, first = a.window ? max(0, end - a.window) : 0;
      uint4 q[G::NS];
#pragma unroll
      for (int f = 0; f < G::NS; ++f) q[f] = sq[ct - ct0][f][lane];
      f32x4 s[4];
      x.scores(q, s);
      float m, l;
      x.weights(now, base, first, end, whole, a.scale_log2, s, m, l);
      f32x4 o[G::ND];
#pragma unroll
      for (int i = 0; i < G::ND; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < G::STEPS; ++st)
        weigh<DT>(operand_weights<DT>(s, st), [&](int d) { return make_uint4(vt[st][d][0], vt[st][d][1], vt[st][d][2], vt[st][d][3]); }, o);
      if (__builtin_expect(no_number(o), 0)) {   // row by row, of what it sees
        const int t_lo = ct * COLS / a.G, t_hi = (ct * COLS + ncol - 1) / a.G;
        for (int tt = t_lo; tt <= t_hi; ++tt) {
          const int to = before + tt, from = a.window ? max(0, to - a.window) : 0;
#pragma unroll
          for (int d = 0; d < G::ND; ++d) {
            f32x4 one = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < G::STEPS; ++st) {
              uint32_t y[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                auto in = [&](int i) {
                  const int p = base + st * G::SP + 16 * (i >> 2) + 4 * grp + (i & 3);
                  return p >= from && p < to;
                };
                if constexpr (DT == DT_BF16) y[j] = vt[st][d][j] & ((in(2 * j) ? 0xffffu : 0u) | (in(2 * j + 1) ? 0xffff0000u : 0u));
                else y[j] = in(j) ? vt[st][d][j] : 0u;
              }
              one = weigh_careful<DT>(operand_weights<DT>(s, st), y, one);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if ((ct * COLS + 4 * grp + r) / a.G == tt) o[d][r] = one[r];
          }
        }
      }
      if (grp == 0) {
        sm[buf][wv][c] = m;
        sl[buf][wv][c] = l;
      }
      // o[np EPV + e] of lane (grp, c): columns 4 grp + r, dimension np 16 EPV + c EPV + e
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * grp + r < ncol)
#pragma unroll
          for (int np = 0; np < G::NP; ++np)
#pragma unroll
            for (int e = 0; e < G::EPV; e += 4)
              *(f32x4*)&so[buf][wv][4 * grp + r][np * 16 * G::EPV + c * G::EPV + e] =
                  f32x4{o[np * G::EPV + e][r], o[np * G::EPV + e + 1][r], o[np * G::EPV + e + 2][r], o[np * G::EPV + e + 3][r]};
      __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
      barrier_only();                       // (the next run's requests go on)
      // Sixteen threads a column, whose factors they form once.
      if (const int y = threadIdx.x / 16; y < ncol) {
        const int d = threadIdx.x % 16 * 4;
        float M = sm[buf][0][y], L = sl[buf][0][y];
        f32x4 O[HD / 64];
#pragma unroll
        for (int p = 0; p < HD / 64; ++p) O[p] = *(const f32x4*)&so[buf][0][y][d + 64 * p];
#pragma unroll
        for (int w = 1; w < RUNS; ++w) {
          const float mw = sm[buf][w][y], N = fmaxf(M, mw), fa = join_scale(M, N), fb = join_scale(mw, N);
          L = fmaf(sl[buf][w][y], fb, L * fa);
          M = N;
#pragma unroll
          for (int p = 0; p < HD / 64; ++p) {
            const f32x4 z = *(const f32x4*)&so[buf][w][y][d + 64 * p];
#pragma unroll
            for (int e = 0; e < 4; ++e) O[p][e] = fmaf(z[e], fb, O[p][e] * fa);
          }
        }
        const int64_t state = ((int64_t)(b * a.ring + ch % a.ring) * a.Hkv + h) * cols + ct * COLS + y;
#pragma unroll
        for (int p = 0; p < HD / 64; ++p) *(f32x4*)(a.o + state * HD + d + 64 * p) = O[p];
        if (d == 0) a.ml[state] = make_float2(M, L);
      }
      if constexpr (BUFFERS == 1) {
        __builtin_amdgcn_s_waitcnt(0xc07f);
        barrier_only();
      }
    }
    x.load_k(next);
    if constexpr (!AHEAD) x.load_v(next, after);
    now = next;
  }
}

// Joins a row's chunks, each times 2^(m - M): the j-th from the row's first on is added to sum
// j % JOIN_GROUPS, then the sums in order.  HD / 4 lanes hold a sum.
constexpr int JOIN_GROUPS = 32;
// The row and head that a sum's lanes are for.
struct Joined {
  int64_t row;
  int head, c0, n;      // its first chunk and their number
  int64_t state0, step; // of the states of chunk 0 of the ring, and between chunks
};
__device__ __forceinline__ Joined joined(const AttendArgs& a, int64_t item) {
  Joined j;
  j.row = item / a.H;
  j.head = (int)(item % a.H);
  const int b = (int)(j.row / a.T), t = (int)(j.row % a.T);
  const int len = min(max(a.lens[b], 0), a.c.max_pages * a.c.page) - a.behind, end = len - a.T + 1 + t;
  j.c0 = (a.window ? max(0, end - a.window) : 0) / CHUNK;
  j.n = end > 0 ? (end + CHUNK - 1) / CHUNK - j.c0 : 0;
  j.step = (int64_t)a.T * a.H;
  j.state0 = (int64_t)b * a.ring * j.step + (int64_t)(j.head / a.G) * a.T * a.G + t * a.G + j.head % a.G;
  return j;
}
template <int HD, int ODT>
__device__ __forceinline__ void join_store(const AttendArgs& a, const Joined& j, int d, float M, float l, f32x4 o) {
  // (no position, or none with a score above -inf: zeros)
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = l == 0.f ? 0.f : o[e] / l;
  const size_t at = (size_t)j.row * a.ldo + j.head * HD + d;
  if (((a.ldo & 3) | (reinterpret_cast<uintptr_t>(a.out) & (ODT == DT_BF16 ? 7 : 15))) == 0) {
    if constexpr (ODT == DT_BF16) *(uint2*)((uint16_t*)a.out + at) = make_uint2(f2bf_bits(o[0]) | f2bf_bits(o[1]) << 16, f2bf_bits(o[2]) | f2bf_bits(o[3]) << 16);
    else *(f32x4*)((float*)a.out + at) = o;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) store_elt<ODT>(a.out, at + e, o[e]);
  }
  if (a.lse && d == 0) a.lse[(size_t)j.row * a.H + j.head] = l == 0.f ? -INFINITY : 0.69314718055994531f * (M + log2f(l));
}

// A product that no addition takes in (its rounding is part of the sums above).
__device__ __forceinline__ float product(float x, float y) {
#pragma clang fp contract(off)
  return x * y;
}

// Four states at a time, of one chunk's runs where those are apart: joined as in the kernels above.
__device__ __forceinline__ void join_runs(float2* ml, f32x4* x) {
#pragma unroll
  for (int r = 1; r < RUNS; ++r) {
    const float M = fmaxf(ml[0].x, ml[r].x), fa = join_scale(ml[0].x, M), fb = join_scale(ml[r].x, M);
    ml[0] = make_float2(M, fmaf(ml[r].y, fb, ml[0].y * fa));
#pragma unroll
    for (int e = 0; e < 4; ++e) x[0][e] = fmaf(x[r][e], fb, x[0][e] * fa);
  }
}

// At most JOIN_GROUPS chunks are held: every sum is one chunk's state.  AT_ONCE are requested together
// (64 sequences to 8192: 9.2 us, 8.5 with 16; 33 rows of 4 to 4096: 6.9 and 7.7; one of 2048: 3.8 and 4.3).
template <int HD, int ODT>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int LPS = HD / 4, AT_ONCE = 8;
  const int64_t item = (int64_t)blockIdx.x * (256 / LPS) + threadIdx.x / LPS;
  if (item >= (int64_t)a.B * a.T * a.H) return;
  const int at = threadIdx.x % LPS, d = at * 4;
  const Joined j = joined(a, item);
  const bool apart = j.n <= a.apart;
  const int n = apart ? j.n * RUNS : j.n;
  auto state = [&](int i) { return j.state0 + (apart ? i : (j.c0 + i) % a.ring) * j.step; };
  float M = -INFINITY;
  for (int i = at; i < n; i += LPS) M = fmaxf(M, a.ml[state(i)].x);
#pragma unroll
  for (int o = 1; o < LPS; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
  const float mu = M == -INFINITY ? 0.f : M;
  float l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < n; i0 += AT_ONCE) {
    float2 ml[AT_ONCE];
    f32x4 x[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int64_t s = state(min(i0 + i, n - 1));
      ml[i] = a.ml[s];
      x[i] = *(const f32x4*)(a.o + s * HD + d);
    }
    if (apart)
#pragma unroll
      for (int i = 0; i < AT_ONCE; i += RUNS) join_runs(ml + i, x + i);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (i0 + i >= n || (apart && i % RUNS)) continue;
      const float f = exp2_(ml[i].x - mu), fl = product(f, ml[i].y);
      l += fl;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += product(f, x[i][e]);
    }
  }
  join_store<HD, ODT>(a, j, d, M, l, o);
}

// More: a workgroup per row and head (512 chunks of one row in one of 256 threads: 30 us).
template <int HD, int ODT>
__global__ __launch_bounds__(1024) void attend_join_long_kernel(AttendArgs a) {
  constexpr int LPS = HD / 4, SETS = 1024 / LPS < JOIN_GROUPS ? 1024 / LPS : JOIN_GROUPS, PER = JOIN_GROUPS / SETS, AT_ONCE = RUNS;
  __shared__ float sM[16], sL[JOIN_GROUPS];
  __shared__ __attribute__((aligned(16))) float sO[JOIN_GROUPS][HD];
  const int tid = threadIdx.x, set = tid / LPS, d = tid % LPS * 4;
  const Joined j = joined(a, blockIdx.x);
  const bool apart = j.n <= a.apart;
  const int n = apart ? j.n * RUNS : j.n, per = apart ? RUNS : 1;   // states of a chunk
  auto state = [&](int i) { return j.state0 + (apart ? i : (j.c0 + i) % a.ring) * j.step; };
  float M = -INFINITY;
  for (int i = tid; i < n; i += 1024) M = fmaxf(M, a.ml[state(i)].x);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
  if ((tid & 63) == 0) sM[tid >> 6] = M;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) M = fmaxf(M, sM[i]);
  const float mu = M == -INFINITY ? 0.f : M;
  if (set < SETS)
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int g = set * PER + p;
      float l = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      // (apart: AT_ONCE / RUNS chunks of the group, the runs of each side by side)
      for (int c0 = g; c0 < j.n; c0 += AT_ONCE / per * JOIN_GROUPS) {
        float2 ml[AT_ONCE];
        f32x4 x[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          const int64_t s = state(min(apart ? (c0 + i / RUNS * JOIN_GROUPS) * RUNS + i % RUNS : c0 + i * JOIN_GROUPS, n - 1));
          ml[i] = a.ml[s];
          x[i] = *(const f32x4*)(a.o + s * HD + d);
        }
        if (apart)
#pragma unroll
          for (int i = 0; i < AT_ONCE; i += RUNS) join_runs(ml + i, x + i);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          if (c0 + i / per * JOIN_GROUPS >= j.n || (apart && i % RUNS)) continue;
          const float f = exp2_(ml[i].x - mu);
          l = fmaf(f, ml[i].y, l);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = fmaf(f, x[i][e], o[e]);
        }
      }
      *(f32x4*)&sO[g][d] = o;
      if (d == 0) sL[g] = l;
    }
  __syncthreads();
  if (set == 0) {
    float l = sL[0];
    f32x4 o = *(const f32x4*)&sO[0][d];
    // (groups that hold no chunk were left at +0, which adds nothing: no sum is -0 but one of such)
#pragma unroll 8
    for (int i = 1; i < JOIN_GROUPS; ++i) {
      l += sL[i];
      const f32x4 y = *(const f32x4*)&sO[i][d];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += y[e];
    }
    join_store<HD, ODT>(a, j, d, M, l, o);
  }
}

// Chunks whose states are held at once: a row's window reaches over that many.
int attend_ring(int64_t positions, int T, int window) {
  int64_t n = (positions + CHUNK - 1) / CHUNK;
  if (window) n = std::min<int64_t>(n, ((int64_t)window + T + CHUNK - 2) / CHUNK + 1);
  return (int)std::max<int64_t>(n, 1);
}
static size_t states_bytes(int64_t states, int hd) { return ((size_t)states * 8 + 255) / 256 * 256 + (size_t)states * hd * 4; }
static size_t states_bytes(int B, int T, int H, int hd, int64_t positions, int window) {
  return states_bytes((int64_t)B * attend_ring(positions, T, window) * T * H, hd);
}
// States take as much room as the tables are wide, whatever the sequences hold: what takes more than
// this (or one row of a sequence, where that does) is done in parts, one after another in the same room.
// (64 sequences of 33 rows, 32 heads of 128, tables for 131072 positions: 18 GB at once.  1024 rows of 8192
// positions in such tables: 1040 us at once, 766 in parts.)
constexpr size_t STATES_BYTES = size_t(2) << 30;
static size_t most_bytes(int H, int hd, int64_t positions, int window) {
  return std::max(STATES_BYTES, states_bytes(1, 1, H, hd, positions, window));
}
size_t attend_workspace(int B, int T, int H, int hd, int64_t positions, int window) {
  return std::min(states_bytes(B, T, H, hd, positions, window), most_bytes(H, hd, positions, window));
}

template <int DT, int HD, int ODT>
static hipError_t attend_t(AttendArgs a, hipStream_t st) {
  const int64_t positions = (int64_t)a.c.max_pages * a.c.page;
  a.ring = attend_ring(positions, a.T, a.window);
  const size_t states = (size_t)a.B * a.ring * a.T * a.H;
  a.ml = reinterpret_cast<float2*>(a.ws);
  a.o = reinterpret_cast<float*>(a.ws + (states * 8 + 255) / 256 * 256);
  // (positions below 2^30 and pages of at most 2^16, in units of 16: the quotient is exact
  // since 2^26 times the factor's error, less than 2^12, stays below 2^38)
  a.page_mul = ((1ull << 38) + a.c.page / 16 - 1) / (a.c.page / 16);
  const int ctiles = (a.T * a.G + COLS - 1) / COLS;
  const int64_t heads = (int64_t)a.B * a.Hkv;
  hipError_t e;
  a.apart = 0;
  if (a.T == 1 && heads * ctiles * a.ring > 1024) {
    // Some 4096 waves, twice what the chip holds at once (64 sequences to 8192: 228 us; 2048
    // waves 273, 6144 231).
    a.cgroups = ctiles;
    a.splits = (int)std::min<int64_t>(a.ring, std::max<int64_t>(1, 4096 / (heads * ctiles)));
    a.apart = a.splits / RUNS;
    const int64_t units = (int64_t)a.B * a.splits * a.Hkv * a.cgroups;
    constexpr int waves = stream_waves<DT, HD>();
    hipLaunchKernelGGL((attend_stream_kernel<DT, HD>), dim3((unsigned)((units + waves - 1) / waves)), dim3(waves * 64), 0, st, a);
  } else {
    // Splits of the length first, some 256 workgroups, or 512 of two to four column tiles, of
    // which a CU holds two; then of the column tiles to 512 (one row of 8 sequences of 2048: 21 us,
    // 24.3 from 512; 5 rows of 16 of 4096, two tiles: 78 from 512, 94 from 256; 33 rows, nine:
    // 158, 160 from 512).
    // A part of a call that fills the chip with the whole call's splits takes those (1024 rows of 16
    // sequences of 2048, in two parts: 1600 us, 1785 with twice the splits).
    const int64_t least = (ctiles + att_tiles(HD * esz_of(DT)) - 1) / att_tiles(HD * esz_of(DT)), some = ctiles > 1 && ctiles <= 4 ? 512 : 256;
    const int64_t of_all = std::max<int64_t>(1, some / ((int64_t)a.all * a.Hkv));
    a.splits = (int)std::min<int64_t>(a.ring, heads * least * of_all >= 512 ? of_all : std::max<int64_t>(1, some / heads));
    a.cgroups = (int)std::min<int64_t>(ctiles, std::max<int64_t>(least, 512 / (heads * a.splits)));
    a.ctw = (ctiles + a.cgroups - 1) / a.cgroups;
    a.cgroups = (ctiles + a.ctw - 1) / a.ctw;
    const dim3 grid((unsigned)(((int64_t)a.B * a.splits + 7) / 8 * 8 * a.Hkv * a.cgroups));
    if (AttGeo<DT, HD>::AHEAD && a.ctw > 1) hipLaunchKernelGGL((attend_rows_kernel<DT, HD, AttGeo<DT, HD>::AHEAD>), grid, dim3(RUNS * 64), 0, st, a);
    else hipLaunchKernelGGL((attend_rows_kernel<DT, HD, false>), grid, dim3(RUNS * 64), 0, st, a);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int64_t items = (int64_t)a.B * a.T * a.H, per = 256 / (HD / 4);
  if (a.ring > JOIN_GROUPS) hipLaunchKernelGGL((attend_join_long_kernel<HD, ODT>), dim3((unsigned)items), dim3(1024), 0, st, a);
  else hipLaunchKernelGGL((attend_join_kernel<HD, ODT>), dim3((unsigned)((items + per - 1) / per)), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <int HD>
static hipError_t attend_hd(const AttendArgs& a, hipStream_t st) {
  if (a.dt == DT_F32) return attend_t<DT_F32, HD, DT_F32>(a, st);
  return a.odt == DT_F32 ? attend_t<DT_BF16, HD, DT_F32>(a, st) : attend_t<DT_BF16, HD, DT_BF16>(a, st);
}

static hipError_t attend(const AttendArgs& a, hipStream_t st) {
  return a.hd == 64 ? attend_hd<64>(a, st) : a.hd == 128 ? attend_hd<128>(a, st) : attend_hd<256>(a, st);
}

// In parts of equally many sequences, or of rows of one, whose states fit (a row's bits depend on
// that row alone).
hipError_t run_attend(const AttendArgs& a, hipStream_t st) {
  const int64_t positions = (int64_t)a.c.max_pages * a.c.page;
  const size_t most = most_bytes(a.H, a.hd, positions, a.window);
  auto parts = [](int n, size_t fit) {   // of n, of at most `fit` each
    const int64_t k = std::max<int64_t>(1, std::min<int64_t>(n, (int64_t)fit)), count = (n + k - 1) / k;
    return (int)((n + count - 1) / count);
  };
  int seqs = a.B, rows = a.T;
  if (states_bytes(a.B, a.T, a.H, a.hd, positions, a.window) > most) {
    seqs = parts(a.B, most / states_bytes(1, a.T, a.H, a.hd, positions, a.window));
    if (seqs == 1) rows = parts(a.T, most / states_bytes((int64_t)attend_ring(positions, a.T, a.window) * a.H, a.hd));
  }
  for (int b = 0; b < a.B; b += seqs)
    for (int t = 0; t < a.T; t += rows) {
      AttendArgs p = a;
      const int64_t row = (int64_t)b * a.T + t;
      p.B = std::min(seqs, a.B - b);
      p.T = std::min(rows, a.T - t);
      p.behind = a.T - t - p.T;
      p.all = a.B;
      p.q = (const uint8_t*)a.q + row * a.ldq * esz_of(a.dt);
      p.out = (uint8_t*)a.out + row * a.ldo * esz_of(a.odt);
      p.lse = a.lse ? a.lse + row * a.H : nullptr;
      p.lens = a.lens + b;
      p.c.tables = a.c.tables + b * a.c.ldt;
      const hipError_t e = attend(p, st);
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

}  // namespace ee
