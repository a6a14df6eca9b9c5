// Device-side types and helpers shared by the kernel sources: numerics, the
// matrix instructions' fragment geometry and buffer loads.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace ee {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));


// ---------------------------------------------------------------- numerics --

__device__ __forceinline__ uint32_t f2bf_bits(float f) {
  uint32_t u = __float_as_uint(f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0u;   // NaN stays NaN
  u += 0x7fffu + ((u >> 16) & 1u);                        // nearest, ties to even
  return u >> 16;
}
__device__ __forceinline__ float bf2f(uint32_t b) { return __uint_as_float(b << 16); }
// Sum and maximum of x over the lanes l, l ^ 16 (row pairs) or l, l ^ 32
// (halves) of a wave with v_permlane16_swap / v_permlane32_swap: the swap
// leaves x[l] and x[l ^ 16] (x[l ^ 32]) in its two results of every lane, in
// the same order for both lanes of a pair, so the value is that of
// x + shfl_xor(x, 16) (32) without the LDS round trip.
__device__ __forceinline__ float xsum16(float x) {
  const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
__device__ __forceinline__ float xsum32(float x) {
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
__device__ __forceinline__ float xmax16(float x) {
  const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float xmax32(float x) {
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
// Nearest-even bf16 bits of two finite floats, a in the low half, with one
// v_cvt_pk_bf16_f32 (equal to f2bf_bits_finite of each, checked for every
// finite float bit pattern).
__device__ __forceinline__ uint32_t bf16x2_bits(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
// Nearest-even bf16 bits of a finite float (no NaN handling, no branch).
__device__ __forceinline__ uint32_t f2bf_bits_finite(float f) {
  const uint32_t u = __float_as_uint(f);
  return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

// Round a float to the storage type and return the stored value as float.
template <int DT> __device__ __forceinline__ float rnd(float x);
template <> __device__ __forceinline__ float rnd<DT_F32>(float x) { return x; }
template <> __device__ __forceinline__ float rnd<DT_BF16>(float x) { return bf2f(f2bf_bits(x)); }

template <int DT> __device__ __forceinline__ void store_elt(void* base, size_t i, float x);
template <> __device__ __forceinline__ void store_elt<DT_F32>(void* base, size_t i, float x) {
  reinterpret_cast<float*>(base)[i] = x;
}
template <> __device__ __forceinline__ void store_elt<DT_BF16>(void* base, size_t i, float x) {
  reinterpret_cast<uint16_t*>(base)[i] = (uint16_t)f2bf_bits(x);
}
template <int DT> __device__ __forceinline__ float load_elt(const void* base, size_t i);
template <> __device__ __forceinline__ float load_elt<DT_F32>(const void* base, size_t i) {
  return reinterpret_cast<const float*>(base)[i];
}
template <> __device__ __forceinline__ float load_elt<DT_BF16>(const void* base, size_t i) {
  return bf2f(reinterpret_cast<const uint16_t*>(base)[i]);
}

template <int DT> struct Geo;
template <> struct Geo<DT_BF16> { static constexpr int KS = 32, EPL = 8, ESZ = 2; };
template <> struct Geo<DT_F32> { static constexpr int KS = 16, EPL = 4, ESZ = 4; };

// D += A * B over one fragment pair (16x16 tile, KS reduction columns).
template <int DT> __device__ __forceinline__ f32x4 mma(uint4 a, uint4 b, f32x4 c);
template <> __device__ __forceinline__ f32x4 mma<DT_BF16>(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma<DT_F32>(uint4 a, uint4 b, f32x4 c) {
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
  return c;
}

// Element index, inside a packed fragment buffer with S super-steps, of
// matrix element (row, col).
template <int DT> __device__ __forceinline__ size_t frag_index(int row, int col, int S) {
  constexpr int KS = Geo<DT>::KS, EPL = Geo<DT>::EPL;
  const int tt = row >> 4, c = row & 15;
  const int s = col / KS, kk = col % KS;
  const int grp = kk / EPL, e = kk % EPL;
  return ((size_t)(tt * S + s) * 64 + grp * 16 + c) * EPL + e;
}

// ------------------------------------------------------------- buffer loads --

constexpr unsigned OOB = 0x80000000u; // buffer offset past every range: loads 0

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* p, unsigned bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}
// 16-byte buffer load; offsets beyond the resource size return zeros without
// a memory access.  AUX selects the cache policy (2 = non-temporal).
template <int AUX>
__device__ __forceinline__ uint4 bload(__amdgpu_buffer_rsrc_t r, unsigned off) {
  const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, AUX);
  return make_uint4(v.x, v.y, v.z, v.w);
}

// 8-byte buffer load (as bload).
template <int AUX>
__device__ __forceinline__ uint2 bload64(__amdgpu_buffer_rsrc_t r, unsigned off) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, AUX);
  return make_uint2(v.x, v.y);
}

}  // namespace ee
