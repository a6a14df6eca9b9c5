// gfx950 kernels of the stand-alone operators: a matrix product with bias,
// activation and residual in its epilogue, the routing of rows to experts,
// and the routed experts' SwiGLU products.
//
// Arithmetic (independent of the number of rows and of the kernel that runs,
// so a row's result never depends on the other rows of a call):
//   * every product element is one fp32 accumulator that takes the reduction's
//     super-steps (32 columns in bf16, 16 in fp32: one fragment) in order;
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

// acc[n] += (16 features of wp[n]) x (16 rows of xp) over S super-steps.  wp and
// xp point to the lane's own 16 bytes of step 0.  Two buffers of D steps: the next
// D steps are requested before the current ones are multiplied.
template <int DT, int NT, int D>
__device__ __forceinline__ void chain(const unsigned char* const (&wp)[NT], const unsigned char* xp, int S,
                                      f32x4 (&acc)[NT]) {
  uint4 wa[D][NT], xa[D], wb[D][NT], xb[D];
  auto load = [&](uint4 (&w)[D][NT], uint4 (&x)[D], int s0) {
#pragma unroll
    for (int i = 0; i < D; ++i) {
      const int s = min(s0 + i, S - 1);   // (past the end: the last step again, unused)
#pragma unroll
      for (int n = 0; n < NT; ++n) w[i][n] = *reinterpret_cast<const uint4*>(wp[n] + (size_t)s * STEP);
      x[i] = *reinterpret_cast<const uint4*>(xp + (size_t)s * STEP);
    }
  };
  auto mul = [&](const uint4 (&w)[D][NT], const uint4 (&x)[D], int s0) {
#pragma unroll
    for (int i = 0; i < D; ++i)
      if (s0 + i < S)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[n] = mma<DT>(w[i][n], x[i], acc[n]);
  };
  load(wa, xa, 0);
  for (int s = 0; s < S; s += 2 * D) {
    load(wb, xb, s + D);
    mul(wa, xa, s);
    load(wa, xa, s + 2 * D);
    mul(wb, xb, s + D);
  }
}

__device__ __forceinline__ float silu(float v) { return v / (1.0f + expf(-v)); }

__device__ __forceinline__ float activate(float v, int act) {
  switch (act) {
    case ACT_SILU: return silu(v);
    case ACT_GELU: return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
    case ACT_GELU_TANH: return v / (1.0f + expf(-1.5957691216057308f * (v + 0.044715f * v * v * v)));
    case ACT_RELU: return v < 0.0f ? 0.0f : v;   // (NaN stays NaN)
    default: return v;
  }
}

// ------------------------------------------------------------------- linear --

// Bias, activation and residual of features n .. n + 3 of row t, and the store.
template <int ODT>
__device__ __forceinline__ void linear_out(const LinearArgs& a, int t, int n, f32x4 v) {
  if (t >= a.T) return;
  const size_t yo = (size_t)t * a.ldy + n, ro = (size_t)t * a.ldr + n;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n + i >= a.N) return;
    float u = v[i];
    if (a.bias) u += a.bias[n + i];
    u = activate(u, a.act);
    if (a.res) u += load_elt<ODT>(a.res, ro + i);
    store_elt<ODT>(a.y, yo + i, u);
  }
}

// One 16-feature tile per wave and 16 rows per workgroup.
template <int DT, int ODT>
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs a, int nblk) {
  constexpr int ESZ = Geo<DT>::ESZ;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = lane & 15, grp = lane >> 4;
  const int nb = blockIdx.x % nblk, t0 = blockIdx.x / nblk * 16, n0 = (nb * 4 + wv) * 16;
  if (n0 >= a.N) return;
  const unsigned char* wp[1] = {reinterpret_cast<const unsigned char*>(a.w) +
                                (size_t)min(n0 + c, a.N - 1) * a.ldw * ESZ + grp * 16};
  const unsigned char* xp =
      reinterpret_cast<const unsigned char*>(a.x) + (size_t)min(t0 + c, a.T - 1) * a.ldx * ESZ + grp * 16;
  f32x4 acc[1] = {f32x4{0.f, 0.f, 0.f, 0.f}};
  chain<DT, 1, 8>(wp, xp, a.K / Geo<DT>::KS, acc);
  linear_out<ODT>(a, t0 + c, n0 + 4 * grp, acc[0]);
}

hipError_t run_linear(const LinearArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  const int nblk = (a.N + 63) / 64;
  const dim3 grid((unsigned)nblk * ((a.T + 15) / 16)), block(256);
  if (a.dt == DT_F32) hipLaunchKernelGGL((linear_kernel<DT_F32, DT_F32>), grid, block, 0, st, a, nblk);
  else if (a.odt == DT_F32) hipLaunchKernelGGL((linear_kernel<DT_BF16, DT_F32>), grid, block, 0, st, a, nblk);
  else hipLaunchKernelGGL((linear_kernel<DT_BF16, DT_BF16>), grid, block, 0, st, a, nblk);
  return hipGetLastError();
}

// -------------------------------------------------------------------- route --

constexpr int ROUTE_ROWS = 4;   // rows (waves) per workgroup

// One wave per row, experts e = 64 i + lane in registers.  Scores, biased
// scores and the selection are float64 values of the logits, so which experts
// a row gets never hangs on a float32 rounding.  The k experts are taken one
// after another: a lane's best, then the wave's, the lowest index among equal
// ones.
template <int DT, int EPL>
__global__ __launch_bounds__(ROUTE_ROWS * 64) void route_kernel(RouteArgs a) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, t = blockIdx.x * ROUTE_ROWS + wv;
  __shared__ double gkey[ROUTE_ROWS][EPL * 64];
  const bool row = t < a.T;
  constexpr double NONE = -INFINITY;
  double s[EPL], key[EPL];
  double mx = NONE;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    float l = row && e < a.E ? load_elt<DT>(a.logits, (size_t)t * a.ld + e) : -INFINITY;
    if (!(l > -INFINITY)) l = -INFINITY;   // (NaN)
    s[i] = (double)fminf(l, FLT_MAX);
    mx = fmax(mx, s[i]);
  }
  for (int o = 32; o; o >>= 1) mx = fmax(mx, __shfl_xor(mx, o));
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const bool dead = s[i] == NONE;
    key[i] = dead ? NONE : 0.0;
    s[i] = dead ? 0.0 : a.score == SCORE_SOFTMAX ? exp(s[i] - mx) : 1.0 / (1.0 + exp(-s[i]));
    sum += s[i];
  }
  for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = i * 64 + lane;
    if (a.score == SCORE_SOFTMAX && sum > 0.0) s[i] /= sum;
    if (key[i] == NONE) continue;
    double b = 0.0;
    if (a.bias) {
      const float f = a.bias[e];
      b = f > -INFINITY ? (double)fminf(f, FLT_MAX) : NONE;   // (NaN: not selectable)
    }
    key[i] = s[i] + b;
  }
  if (a.groups > 1) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) gkey[wv][i * 64 + lane] = key[i];
    __syncthreads();
    const int per = a.E / a.groups;
    double gs = NONE;   // lane g: the score of group g
    if (lane < a.groups) {
      double b1 = NONE, b2 = NONE;
      for (int i = 0; i < per; ++i) {
        const double v = gkey[wv][lane * per + i];
        if (v > b1) { b2 = b1; b1 = v; }
        else if (v > b2) b2 = v;
      }
      gs = a.group_top == 2 && b2 > NONE ? b1 + b2 : b1;
    }
    // groups that come before this one: better, or equal with a lower index
    int before = 0;
    for (int g = 0; g < a.groups; ++g) {
      const double o = __shfl(gs, g);
      before += o > gs || (o == gs && g < lane);
    }
    const unsigned long long keep = __ballot(lane < a.groups && before < a.top_groups);
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = i * 64 + lane;
      if (e < a.E && !((keep >> (e / per)) & 1ull)) key[i] = NONE;
    }
  }
  int id = -1;        // lane j: the expert of slot j and its score
  double w = 0.0;
  for (int j = 0; j < a.k; ++j) {
    double best = NONE;
    int at = 0x7fffffff;
    double sc = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (key[i] > best) { best = key[i]; at = i * 64 + lane; sc = s[i]; }
    for (int o = 32; o; o >>= 1) {
      const double b = __shfl_xor(best, o), bs = __shfl_xor(sc, o);
      const int ba = __shfl_xor(at, o);
      if (b > best || (b == best && ba < at)) { best = b; at = ba; sc = bs; }
    }
    if (best == NONE) break;
    if (lane == j) { id = at; w = sc; }
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (at == i * 64 + lane) key[i] = NONE;
  }
  if (a.renorm) {
    double tot = 0.0;
    for (int j = 0; j < a.k; ++j) tot += __shfl(w, j);
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
// dtype: it is the down product's operand.  One 16-feature tile of gate and of
// up per wave; all 16 columns of the product hold the pair's row.
template <int DT>
__global__ __launch_bounds__(256) void ffn_up_kernel(FfnArgs a, void* z, int nblk) {
  constexpr int ESZ = Geo<DT>::ESZ;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = lane & 15, grp = lane >> 4;
  const int p = blockIdx.x / nblk, f0 = (blockIdx.x % nblk * 4 + wv) * 16;
  const int e = a.ids[p];
  if (f0 >= a.F || e < 0 || e >= a.E) return;
  const size_t rb = (size_t)a.d * ESZ;
  const unsigned char* w = reinterpret_cast<const unsigned char*>(a.wgu) + ((size_t)e * 2 * a.F + f0 + c) * rb + grp * 16;
  const unsigned char* wp[2] = {w, w + (size_t)a.F * rb};
  const unsigned char* xp = reinterpret_cast<const unsigned char*>(a.x) + (size_t)(p / a.k) * a.ldx * ESZ + grp * 16;
  f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  chain<DT, 2, 8>(wp, xp, a.d / Geo<DT>::KS, acc);
  if (c == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) store_elt<DT>(z, (size_t)p * a.F + f0 + 4 * grp + i, silu(acc[0][i]) * acc[1][i]);
}

constexpr int DOWN_WAVES = 8;

// out[t] = sum_j w_j (z_j Wd^T) + res of 16 features of one row: a wave per
// slot, the slots' products joined in slot order.
template <int DT, int ODT>
__global__ __launch_bounds__(DOWN_WAVES * 64) void ffn_down_kernel(FfnArgs a, const void* z, int nblk) {
  constexpr int ESZ = Geo<DT>::ESZ;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, c = lane & 15, grp = lane >> 4;
  const int t = blockIdx.x / nblk, n0 = blockIdx.x % nblk * 16;
  __shared__ float y[ROUTE_MAX_K][16];
  for (int j = wv; j < a.k; j += DOWN_WAVES) {
    const size_t p = (size_t)t * a.k + j;
    const int e = a.ids[p];
    if (e < 0 || e >= a.E) continue;
    const size_t rb = (size_t)a.F * ESZ;
    const unsigned char* wp[1] = {reinterpret_cast<const unsigned char*>(a.wd) + ((size_t)e * a.d + n0 + c) * rb + grp * 16};
    const unsigned char* zp = reinterpret_cast<const unsigned char*>(z) + p * rb + grp * 16;
    f32x4 acc[1] = {f32x4{0.f, 0.f, 0.f, 0.f}};
    chain<DT, 1, 8>(wp, zp, a.F / Geo<DT>::KS, acc);
    if (c == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[j][4 * grp + i] = acc[0][i];
  }
  __syncthreads();
  if (threadIdx.x < 16) {
    float o = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const size_t p = (size_t)t * a.k + j;
      const int e = a.ids[p];
      if (e >= 0 && e < a.E) o = fmaf(a.weights[p], y[j][threadIdx.x], o);
    }
    const int n = n0 + threadIdx.x;
    if (a.res) o += load_elt<ODT>(a.res, (size_t)t * a.ldr + n);
    store_elt<ODT>(a.out, (size_t)t * a.ldo + n, o);
  }
}

size_t ffn_workspace(int T, int E, int k, int d, int F, int dt) {
  (void)E; (void)d;
  return ((size_t)T * k * F * esz_of(dt) + 255) / 256 * 256;
}

template <int DT, int ODT>
static hipError_t ffn_t(const FfnArgs& a, hipStream_t st) {
  void* z = a.ws;
  const int ub = (a.F + 63) / 64, db = a.d / 16;
  hipLaunchKernelGGL((ffn_up_kernel<DT>), dim3((unsigned)ub * a.T * a.k), dim3(256), 0, st, a, z, ub);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((ffn_down_kernel<DT, ODT>), dim3((unsigned)db * a.T), dim3(DOWN_WAVES * 64), 0, st, a, (const void*)z, db);
  return hipGetLastError();
}

hipError_t run_ffn(const FfnArgs& a, hipStream_t st) {
  if (a.T == 0) return hipSuccess;
  if (a.dt == DT_F32) return ffn_t<DT_F32, DT_F32>(a, st);
  return a.odt == DT_F32 ? ffn_t<DT_BF16, DT_F32>(a, st) : ffn_t<DT_BF16, DT_BF16>(a, st);
}

}  // namespace ee
