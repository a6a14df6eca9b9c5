// Epilogue of the stand-alone products: bias, activation, residual and store of a
// tile's values, shared by the kernel sources that make them.
#pragma once

#include "device.h"
#include "operators.h"

namespace ee {

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

}  // namespace ee
