// gfx950 kernels of the 8-bit operators: e4m3 codes with one scale per block of 128
// columns, and the matrix product of such operands.
//
// Arithmetic of the product (independent of the number of rows and of the kernel
// that runs, so a row's result never depends on the other rows of a call):
//   * a block's 128 products in the matrix instructions, from nothing: D_b;
//   * acc = fma(D_b, xs_b ws_b, acc), blocks in order, in fp32;
//   * bias, activation, residual, one rounding.
// D_b of a bf16 output is one 16 x 16 x 128 instruction on the codes themselves.  Its
// adders align the products of a few columns to their largest and drop what lies 14
// bits below that (measured); over random operands D_b is 2^-15.5 of sum |x w| off
// at worst.  A result then is a few 2^-16 off, a hundredth of what its rounding to bf16 costs.  An fp32
// output is asked for where that matters: there the codes are widened to bf16
// (exactly) and D_b is four 16 x 16 x 32 instructions, whose sums are fp32.

#include "operators.h"

#include <float.h>
#include <math.h>

#include <algorithm>

#include "device.h"
#include "epilogue.h"

namespace ee {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr float E4M3_MAX = 448.f;

// ----------------------------------------------------------------- quantise --

// Sixteen values of a row at column k (a multiple of 16), zeros past K.
template <int DT> __device__ __forceinline__ void load16(const Fp8QuantArgs& a, int t, int k, float (&f)[16]) {
  constexpr int ESZ = Geo<DT>::ESZ;
  uint4 u[ESZ];
  const bool in = t < a.T && k < a.K;
  const uint4* p = (const uint4*)((const uint8_t*)a.x + (in ? t * a.ldx + k : 0) * ESZ);
#pragma unroll
  for (int i = 0; i < ESZ; ++i) u[i] = in ? p[i] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int i = 0; i < ESZ; ++i) {
    const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if constexpr (DT == DT_BF16) {
        f[8 * i + 2 * j] = bf2f(w[j] & 0xffffu);
        f[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      } else {
        f[4 * i + j] = __uint_as_float(w[j]);
      }
  }
}
// Largest finite magnitude.
__device__ __forceinline__ float amax16(const float (&f)[16]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float v = fabsf(f[i]);
    if (v <= FLT_MAX) m = fmaxf(m, v);   // (false for NaN)
  }
  return m;
}
__device__ __forceinline__ float block_scale(float amax) { return fmaxf(amax / E4M3_MAX, FLT_MIN); }
// Codes of x / scale, the quotient as IEEE rounds it, to nearest even; past the
// largest code that one, NaN stays NaN.
__device__ __forceinline__ uint4 codes16(const float (&f)[16], float scale) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = f[4 * i + j] / scale;
      q[j] = v > E4M3_MAX ? E4M3_MAX : v < -E4M3_MAX ? -E4M3_MAX : v;
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Blocks of one row: eight lanes each, sixteen columns a lane.
constexpr int QUANT_THREADS = 256;
template <int DT>
__global__ __launch_bounds__(QUANT_THREADS) void quant_rows_kernel(Fp8QuantArgs a, int kb) {
  const int64_t i = (int64_t)blockIdx.x * (QUANT_THREADS / 8) + threadIdx.x / 8;   // block
  const int t = (int)min<int64_t>(i / kb, a.T), b = (int)(i % kb), k = b * BLOCK + (threadIdx.x & 7) * 16;
  float f[16];
  load16<DT>(a, t, k, f);
  float m = amax16(f);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float s = block_scale(m);
  if (t >= a.T) return;
  if (k < a.K) *(uint4*)(a.codes + t * a.ldc + k) = codes16(f, s);
  if ((threadIdx.x & 7) == 0) a.scales[i] = s;
}

// Blocks of 128 rows: a workgroup each.
template <int DT>
__global__ __launch_bounds__(QUANT_THREADS) void quant_block_kernel(Fp8QuantArgs a, int kb) {
  const int rb = blockIdx.x / kb, b = blockIdx.x % kb, k = b * BLOCK + (threadIdx.x & 7) * 16, t0 = rb * BLOCK + threadIdx.x / 8;
  __shared__ float sm[QUANT_THREADS / 64];
  float f[4][16], m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) load16<DT>(a, t0 + 32 * i, k, f[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, amax16(f[i]));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QUANT_THREADS / 64; ++i) m = fmaxf(m, sm[i]);
  const float s = block_scale(m);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t0 + 32 * i < a.T && k < a.K) *(uint4*)(a.codes + (t0 + 32 * i) * a.ldc + k) = codes16(f[i], s);
  if (threadIdx.x == 0) a.scales[blockIdx.x] = s;
}

template <int DT> static hipError_t quant_t(const Fp8QuantArgs& a, hipStream_t st) {
  const int kb = (a.K + BLOCK - 1) / BLOCK;
  if (a.block_rows == 1) {
    const int64_t n = ((int64_t)a.T * kb + QUANT_THREADS / 8 - 1) / (QUANT_THREADS / 8);
    hipLaunchKernelGGL((quant_rows_kernel<DT>), dim3((unsigned)n), dim3(QUANT_THREADS), 0, st, a, kb);
  } else {
    hipLaunchKernelGGL((quant_block_kernel<DT>), dim3((unsigned)((a.T + BLOCK - 1) / BLOCK * kb)), dim3(QUANT_THREADS), 0, st, a, kb);
  }
  return hipGetLastError();
}

hipError_t run_fp8_quant(const Fp8QuantArgs& a, hipStream_t st) {
  return a.dt == DT_BF16 ? quant_t<DT_BF16>(a, st) : quant_t<DT_F32>(a, st);
}

// ------------------------------------------------------------------ product --

// A lane's 32 codes of a block: pieces grp and grp + 4 of the row's eight 16-byte
// pieces.  (Which columns a lane holds is free as long as both operands agree, in all kernels:
// the instruction's sums depend on it.)
struct Codes {
  uint4 u[2];
};

// Two bf16 of codes 2 i and 2 i + 1 of a dword (exact).
template <bool HIGH> __device__ __forceinline__ uint32_t widen2(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b) {
  return make_uint4(widen2<false>(a), widen2<true>(a), widen2<false>(b), widen2<true>(b));
}

// D_b of 16 features (w) and 16 rows (x).
template <bool EXACT> __device__ __forceinline__ f32x4 block_product(Codes w, Codes x) {
  f32x4 d = {0.f, 0.f, 0.f, 0.f};
  if constexpr (EXACT) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      d = mma<DT_BF16>(widen8(w.u[i].x, w.u[i].y), widen8(x.u[i].x, x.u[i].y), d);
      d = mma<DT_BF16>(widen8(w.u[i].z, w.u[i].w), widen8(x.u[i].z, x.u[i].w), d);
    }
  } else {
    const i32x8 A = {(int)w.u[0].x, (int)w.u[0].y, (int)w.u[0].z, (int)w.u[0].w, (int)w.u[1].x, (int)w.u[1].y, (int)w.u[1].z, (int)w.u[1].w};
    const i32x8 B = {(int)x.u[0].x, (int)x.u[0].y, (int)x.u[0].z, (int)x.u[0].w, (int)x.u[1].x, (int)x.u[1].y, (int)x.u[1].z, (int)x.u[1].w};
    // (both formats e4m3; scales of 0 are the instruction without scales)
    d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, d, 0, 0, 0, 0, 0, 0);
  }
  return d;
}

// One wave per 16 x 16 tile, operands from memory.
template <bool EXACT>
__global__ __launch_bounds__(64) void fp8_tile_kernel(Fp8LinearArgs a, int nft) {
  const int lane = threadIdx.x, c = lane & 15, grp = lane >> 4;
  const int f0 = blockIdx.x % nft * 16, t0 = blockIdx.x / nft * 16, K = a.l.K, kb = (K + BLOCK - 1) / BLOCK;
  const uint8_t* w = (const uint8_t*)a.l.w + min(f0 + c, a.l.N - 1) * a.l.ldw + grp * 16;
  const uint8_t* x = (const uint8_t*)a.l.x + min(t0 + c, a.l.T - 1) * a.l.ldx + grp * 16;
  const float* xs = a.xs + (int64_t)min(t0 + c, a.l.T - 1) * kb;
  const float* ws = a.ws + (int64_t)(f0 / BLOCK) * kb;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int b = 0; b < kb; ++b) {
    Codes wf, xf;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = b * BLOCK + i * 64;
      const bool in = k + grp * 16 < K;
      wf.u[i] = in ? *(const uint4*)(w + k) : make_uint4(0u, 0u, 0u, 0u);
      xf.u[i] = in ? *(const uint4*)(x + k) : make_uint4(0u, 0u, 0u, 0u);
    }
    const f32x4 d = block_product<EXACT>(wf, xf);
    const float s = xs[b] * ws[b];
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] = fmaf(d[r], s, acc[r]);
  }
  const bool vec = linear_vec(a.l);
  const int t = t0 + c, n = f0 + 4 * grp;
  linear_out(a.l, t, n, acc, linear_bias(a.l, n), linear_residual(a.l, t, n, vec), vec);
}

hipError_t run_fp8_linear(const Fp8LinearArgs& a, hipStream_t st) {
  const int nft = (a.l.N + 15) / 16, nrt = (a.l.T + 15) / 16;
  if (a.l.odt == DT_F32) hipLaunchKernelGGL((fp8_tile_kernel<true>), dim3((unsigned)nft * nrt), dim3(64), 0, st, a, nft);
  else hipLaunchKernelGGL((fp8_tile_kernel<false>), dim3((unsigned)nft * nrt), dim3(64), 0, st, a, nft);
  return hipGetLastError();
}

}  // namespace ee
