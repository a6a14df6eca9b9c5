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
//   * a chunk's state joins its runs, a row's result its chunks: each state times
//     2^(m - M) for the largest m, added in a fixed order.
// Scores, weights, l and o are fp32.  The matrix instruction of a bf16 cache takes
// the weights as two bf16 parts (p = hi + lo to 2^-17): as one they would add as much error as
// the rounding of a bf16 result, and half the chip's matrix rate waits on the cache anyway.

#include "operators.h"

#include <math.h>

#include <algorithm>

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
static_assert(CHUNK == ATTEND_CHUNK, "");

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
// No operand passes through LDS.
template <int DT, int HD> struct AttGeo {
  static constexpr int ESZ = Geo<DT>::ESZ, EPL = Geo<DT>::EPL, KS = Geo<DT>::KS;
  static constexpr int NS = HD / KS;                         // fragments of a key
  static constexpr int EPV = HD / 16 < EPL ? HD / 16 : EPL;  // dimensions of a lane's piece of V
  static constexpr int NP = HD / 16 / EPV;                   // passes over the dimensions
  static constexpr int VK = DT == DT_BF16 ? 8 : 4;           // positions of a lane in a step of V
  static constexpr int SP = VK * 4;                          // positions of a step
  static constexpr int STEPS = RUN / SP;
  static constexpr int ND = HD / 16;                         // output tiles
};

template <int DT, int HD>
__global__ __launch_bounds__(RUNS * 64) void attend_kernel(AttendArgs a) {
  using G = AttGeo<DT, HD>;
  constexpr int ESZ = G::ESZ;
  const PagedCache& pc = a.c;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, grp = lane >> 4;
  __shared__ float sm[RUNS][COLS], sl[RUNS][COLS];
  __shared__ __attribute__((aligned(16))) float so[RUNS][COLS][HD];

  // (heads first: workgroups are dealt to the eight XCDs in turn, and the tiles of a head then share one's L2)
  int id = blockIdx.x;
  const int h = id % a.Hkv; id /= a.Hkv;
  const int ct = id % a.ctiles; id /= a.ctiles;
  const int split = id % a.splits, b = id / a.splits;
  const int cols = a.T * a.G, len = min(max(a.lens[b], 0), pc.max_pages * pc.page);
  const int t_lo = ct * COLS / a.G, t_hi = min(ct * COLS + COLS - 1, cols - 1) / a.G;
  const int e_lo = len - a.T + 1 + t_lo, e_hi = len - a.T + 1 + t_hi;   // ends of the tile's rows
  const int start = a.window ? max(0, e_lo - a.window) : 0;
  if (e_hi <= 0) return;
  const int ncol = min(COLS, cols - ct * COLS);
  const int col = min(ct * COLS + c, cols - 1), t = col / a.G;          // (columns past the last repeat it)
  const int end = len - a.T + 1 + t, first = a.window ? max(0, end - a.window) : 0;

  uint4 qf[G::NS];
  {
    const uint8_t* q = (const uint8_t*)a.q + ((int64_t)(b * a.T + t) * a.ldq + (h * a.G + col % a.G) * HD) * ESZ + grp * 16;
#pragma unroll
    for (int s = 0; s < G::NS; ++s) qf[s] = *(const uint4*)(q + s * 64);
  }
  const int* table = pc.tables + b * pc.ldt;
  const int ch1 = (e_hi + CHUNK - 1) / CHUNK;
  for (int ch = start / CHUNK + split; ch < ch1; ch += a.splits) {
    const int base = ch * CHUNK + wv * RUN;
    f32x4 o[G::ND];
#pragma unroll
    for (int i = 0; i < G::ND; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (base < e_hi && base + RUN > start) {
      // pages of the run's four 16-position tiles
      __amdgpu_buffer_rsrc_t kr[4], vr[4];
      bool there[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p0 = base + 16 * i, pg = p0 / pc.page;
        there[i] = p0 < e_hi && p0 + 16 > start;
        int page = there[i] ? table[pg] : -1;
        page = __builtin_amdgcn_readfirstlane(page);
        there[i] = page >= 0 && page < pc.n_pages;
        const int64_t pb = there[i] ? page : 0, at = p0 - pg * pc.page;
        kr[i] = make_rsrc((const uint8_t*)pc.k + (pb * pc.kp + at * pc.ks + h * pc.kh) * ESZ, there[i] ? 0x7fffffffu : 0u);
        vr[i] = make_rsrc((const uint8_t*)pc.v + (pb * pc.vp + at * pc.vs + h * pc.vh) * ESZ, there[i] ? 0x7fffffffu : 0u);
      }
      f32x4 s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        const unsigned off = (unsigned)(c * (int)pc.ks * ESZ + grp * 16);
#pragma unroll
        for (int f = 0; f < G::NS; ++f) s[i] = mma<DT>(bload<0>(kr[i], off + f * 64), qf[f], s[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int p = base + 16 * i + 4 * grp + r;
          s[i][r] = there[i] && p < end && p >= first ? s[i][r] * a.scale_log2 : -INFINITY;
          m = fmaxf(m, s[i][r]);
        }
      m = xmax32(xmax16(m));
      const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[i][r] = exp2_(s[i][r] - mu);
          l += s[i][r];
        }
      l = xsum32(xsum16(l));

      // o += weights x values of the positions in [from, to), for a lane's columns
      auto values = [&](int from, int to, f32x4 (&acc)[G::ND]) {
#pragma unroll
        for (int st = 0; st < G::STEPS; ++st) {
          uint4 hi, lo;
          if constexpr (DT == DT_BF16) {
            uint32_t u[4], w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = s[2 * st + (j >> 1)][2 * (j & 1)], y = s[2 * st + (j >> 1)][2 * (j & 1) + 1];
              u[j] = bf16x2_bits(x, y);
              w[j] = bf16x2_bits(x - bf2f(u[j] & 0xffffu), y - __uint_as_float(u[j] & 0xffff0000u));
            }
            hi = make_uint4(u[0], u[1], u[2], u[3]);
            lo = make_uint4(w[0], w[1], w[2], w[3]);
          } else {
            hi = make_uint4(__float_as_uint(s[st][0]), __float_as_uint(s[st][1]), __float_as_uint(s[st][2]), __float_as_uint(s[st][3]));
          }
          // slot j of lane group grp: position 4 grp + j of the step's first tile, then of its second
          unsigned off[G::VK];
#pragma unroll
          for (int j = 0; j < G::VK; ++j) {
            const int p = base + st * G::SP + 16 * (j >> 2) + 4 * grp + (j & 3);
            off[j] = p >= from && p < to ? (unsigned)((4 * grp + (j & 3)) * (int)pc.vs * ESZ + c * G::EPV * ESZ) : OOB;
          }
#pragma unroll
          for (int np = 0; np < G::NP; ++np) {
            if constexpr (DT == DT_F32) {
              uint4 v[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) v[j] = bload<0>(vr[st], off[j] + np * 256);
              acc[np * 4 + 0] = mma<DT>(hi, make_uint4(v[0].x, v[1].x, v[2].x, v[3].x), acc[np * 4 + 0]);
              acc[np * 4 + 1] = mma<DT>(hi, make_uint4(v[0].y, v[1].y, v[2].y, v[3].y), acc[np * 4 + 1]);
              acc[np * 4 + 2] = mma<DT>(hi, make_uint4(v[0].z, v[1].z, v[2].z, v[3].z), acc[np * 4 + 2]);
              acc[np * 4 + 3] = mma<DT>(hi, make_uint4(v[0].w, v[1].w, v[2].w, v[3].w), acc[np * 4 + 3]);
            } else {
              uint32_t v[8][4];
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const auto& r = vr[2 * st + (j >> 2)];
                if constexpr (G::EPV == 8) {
                  const uint4 x = bload<0>(r, off[j] + np * 256);
                  v[j][0] = x.x; v[j][1] = x.y; v[j][2] = x.z; v[j][3] = x.w;
                } else {
                  const uint2 x = bload64<0>(r, off[j]);
                  v[j][0] = x.x; v[j][1] = x.y;
                }
              }
#pragma unroll
              for (int w = 0; w < G::EPV / 2; ++w) {
                uint32_t even[4], odd[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  even[j] = __builtin_amdgcn_perm(v[2 * j + 1][w], v[2 * j][w], 0x05040100u);
                  odd[j] = __builtin_amdgcn_perm(v[2 * j + 1][w], v[2 * j][w], 0x07060302u);
                }
                const uint4 ve = make_uint4(even[0], even[1], even[2], even[3]), vo = make_uint4(odd[0], odd[1], odd[2], odd[3]);
                const int d = np * G::EPV + 2 * w;
                acc[d] = mma<DT>(hi, ve, acc[d]);
                acc[d] = mma<DT>(lo, ve, acc[d]);
                acc[d + 1] = mma<DT>(hi, vo, acc[d + 1]);
                acc[d + 1] = mma<DT>(lo, vo, acc[d + 1]);
              }
            }
          }
        }
      };
      // Where some row does not see what another does, a value that it does not see
      // may be no number, and its weight of 0 would not remove it: row by row, with the others' values zeroed.
      if (a.T > 1 && (base + RUN > e_lo || (a.window && base < e_hi - a.window))) {
        for (int tt = t_lo; tt <= t_hi; ++tt) {
          const int e = len - a.T + 1 + tt;
          f32x4 one[G::ND];
#pragma unroll
          for (int i = 0; i < G::ND; ++i) one[i] = f32x4{0.f, 0.f, 0.f, 0.f};
          values(a.window ? max(0, e - a.window) : 0, e, one);
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if ((ct * COLS + 4 * grp + r) / a.G == tt)
#pragma unroll
              for (int i = 0; i < G::ND; ++i) o[i][r] = one[i][r];
        }
      } else {
        values(start, e_hi, o);
      }
    }
    if (grp == 0) {
      sm[wv][c] = m;
      sl[wv][c] = l;
    }
    // o[np EPV + e] of lane (grp, c): columns 4 grp + r, dimension np 16 EPV + c EPV + e
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (4 * grp + r < ncol)
#pragma unroll
        for (int np = 0; np < G::NP; ++np)
#pragma unroll
          for (int e = 0; e < G::EPV; e += 4)
            *(f32x4*)&so[wv][4 * grp + r][np * 16 * G::EPV + c * G::EPV + e] =
                f32x4{o[np * G::EPV + e][r], o[np * G::EPV + e + 1][r], o[np * G::EPV + e + 2][r], o[np * G::EPV + e + 3][r]};
    __syncthreads();
    for (int i = threadIdx.x; i < ncol * (HD / 4); i += RUNS * 64) {
      const int q = i / (HD / 4), d = i % (HD / 4) * 4;
      float M = sm[0][q];
#pragma unroll
      for (int w = 1; w < RUNS; ++w) M = fmaxf(M, sm[w][q]);
      const float mu = M == -INFINITY ? 0.f : M;
      float L = 0.f;
      f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < RUNS; ++w) {
        const float f = exp2_(sm[w][q] - mu);
        L += f * sl[w][q];
        const f32x4 x = *(const f32x4*)&so[w][q][d];
#pragma unroll
        for (int e = 0; e < 4; ++e) O[e] += f * x[e];
      }
      const int64_t state = ((int64_t)(b * a.ring + ch % a.ring) * a.Hkv + h) * cols + ct * COLS + q;
      *(f32x4*)(a.o + state * HD + d) = O;
      if (d == 0) a.ml[state] = make_float2(M, L);
    }
    __syncthreads();
  }
}

// Joins a row's chunks: workgroup (row, head), groups of HD / 4 threads take every
// NG-th chunk from the row's first on, then the groups in order.
constexpr int JOIN_THREADS = 256;
template <int HD, int ODT>
__global__ __launch_bounds__(JOIN_THREADS) void attend_join_kernel(AttendArgs a) {
  constexpr int LPS = HD / 4, NG = JOIN_THREADS / LPS;
  __shared__ float sM[JOIN_THREADS / 64], sL[NG];
  __shared__ __attribute__((aligned(16))) float sO[NG][HD];
  const int row = blockIdx.x / a.H, head = blockIdx.x % a.H, b = row / a.T, t = row % a.T, h = head / a.G;
  const int len = min(max(a.lens[b], 0), a.c.max_pages * a.c.page), end = len - a.T + 1 + t;
  const int c0 = (a.window ? max(0, end - a.window) : 0) / CHUNK, c1 = end > 0 ? (end + CHUNK - 1) / CHUNK : c0;
  const int cols = a.T * a.G, col = t * a.G + head % a.G;
  auto state = [&](int ch) { return ((int64_t)(b * a.ring + ch % a.ring) * a.Hkv + h) * cols + col; };
  float M = -INFINITY;
  for (int ch = c0 + threadIdx.x; ch < c1; ch += JOIN_THREADS) M = fmaxf(M, a.ml[state(ch)].x);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) M = fmaxf(M, __shfl_xor(M, o));
  if ((threadIdx.x & 63) == 0) sM[threadIdx.x >> 6] = M;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < JOIN_THREADS / 64; ++i) M = fmaxf(M, sM[i]);
  const float mu = M == -INFINITY ? 0.f : M;
  const int g = threadIdx.x / LPS, d = threadIdx.x % LPS * 4;
  float L = 0.f;
  f32x4 O = {0.f, 0.f, 0.f, 0.f};
  for (int ch = c0 + g; ch < c1; ch += NG) {
    const int64_t s = state(ch);
    const float2 ml = a.ml[s];
    const f32x4 x = *(const f32x4*)(a.o + s * HD + d);
    const float f = exp2_(ml.x - mu);
    L += f * ml.y;
#pragma unroll
    for (int e = 0; e < 4; ++e) O[e] += f * x[e];
  }
  *(f32x4*)&sO[g][d] = O;
  if (d == 0) sL[g] = L;
  __syncthreads();
  if (g) return;
#pragma unroll
  for (int i = 1; i < NG; ++i) {
    L += sL[i];
    O += *(const f32x4*)&sO[i][d];
  }
  // (no position, or none with a score above -inf: zeros)
#pragma unroll
  for (int e = 0; e < 4; ++e) store_elt<ODT>(a.out, (size_t)row * a.ldo + head * HD + d + e, L == 0.f ? 0.f : O[e] / L);
  if (a.lse && d == 0) a.lse[(size_t)row * a.H + head] = L == 0.f ? -INFINITY : 0.69314718055994531f * (M + log2f(L));
}

// Chunks whose states are held at once: a row's window reaches over that many.
int attend_ring(int64_t positions, int T, int window) {
  int64_t n = (positions + CHUNK - 1) / CHUNK;
  if (window) n = std::min<int64_t>(n, ((int64_t)window + T + CHUNK - 2) / CHUNK + 1);
  return (int)std::max<int64_t>(n, 1);
}
size_t attend_workspace(int B, int T, int H, int hd, int64_t positions, int window) {
  const size_t states = (size_t)B * attend_ring(positions, T, window) * T * H;
  return (states * 8 + 255) / 256 * 256 + states * hd * 4;
}

template <int DT, int HD, int ODT>
static hipError_t attend_t(AttendArgs a, hipStream_t st) {
  const int64_t positions = (int64_t)a.c.max_pages * a.c.page;
  a.ring = attend_ring(positions, a.T, a.window);
  const size_t states = (size_t)a.B * a.ring * a.T * a.H;
  a.ml = reinterpret_cast<float2*>(a.ws);
  a.o = reinterpret_cast<float*>(a.ws + (states * 8 + 255) / 256 * 256);
  a.ctiles = (a.T * a.G + COLS - 1) / COLS;
  a.splits = (int)std::min<int64_t>(a.ring, std::max<int64_t>(1, 4096 / ((int64_t)a.B * a.Hkv * a.ctiles)));
  hipLaunchKernelGGL((attend_kernel<DT, HD>), dim3((unsigned)((int64_t)a.Hkv * a.ctiles * a.splits * a.B)), dim3(RUNS * 64), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attend_join_kernel<HD, ODT>), dim3((unsigned)((int64_t)a.B * a.T * a.H)), dim3(JOIN_THREADS), 0, st, a);
  return hipGetLastError();
}

template <int HD>
static hipError_t attend_hd(const AttendArgs& a, hipStream_t st) {
  if (a.dt == DT_F32) return attend_t<DT_F32, HD, DT_F32>(a, st);
  return a.odt == DT_F32 ? attend_t<DT_BF16, HD, DT_F32>(a, st) : attend_t<DT_BF16, HD, DT_BF16>(a, st);
}

hipError_t run_attend(const AttendArgs& a, hipStream_t st) {
  return a.hd == 64 ? attend_hd<64>(a, st) : a.hd == 128 ? attend_hd<128>(a, st) : attend_hd<256>(a, st);
}

}  // namespace ee
