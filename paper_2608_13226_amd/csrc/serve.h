// Types and conversions shared by the serving kernels (norm, 4-bit products,
// cache append, cache attention).  8-bit values are e4m3: 3 bits after the
// leading one, exponents down to -6, largest 448, no infinity.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace cp {

struct Bf16 { uint16_t bits; };
struct F16 { uint16_t bits; };
struct F32 { uint32_t bits; };
struct E4m3 { uint8_t bits; };

typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;
typedef __attribute__((__vector_size__(2 * sizeof(_Float16)))) _Float16 f16x2;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

constexpr float kE4m3Max = 448.f;

// Two floats as a packed pair of T, each rounded to nearest even (`a` low).
template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack2<Bf16>(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
template <>
__device__ __forceinline__ uint32_t pack2<F16>(float a, float b) {
  const f16x2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// A packed pair of T widened exactly.
template <class T>
__device__ __forceinline__ float2 unpack2(uint32_t w);
template <>
__device__ __forceinline__ float2 unpack2<Bf16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <>
__device__ __forceinline__ float2 unpack2<F16>(uint32_t w) {
  const f16x2 v = __builtin_bit_cast(f16x2, w);
  return make_float2((float)v[0], (float)v[1]);
}

// Four floats as e4m3 bytes, each clamped to +-448 and rounded to nearest
// even.  The comparisons are false for NaN, which stays NaN.
__device__ __forceinline__ float e4m3_clamp(float x) {
  x = x > kE4m3Max ? kE4m3Max : x;
  return x < -kE4m3Max ? -kE4m3Max : x;
}
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(a), e4m3_clamp(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(c), e4m3_clamp(d), w, true);
  return uint32_t(w);
}
// The same for floats that round to at most +-448 as they are.
__device__ __forceinline__ uint32_t pack4_e4m3_inside(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return uint32_t(w);
}

// Element i of an array of T as float, and back (rounded to nearest even).
template <class T>
__device__ __forceinline__ float load1(const void* p, int64_t i);
template <>
__device__ __forceinline__ float load1<Bf16>(const void* p, int64_t i) {
  return __uint_as_float(uint32_t(static_cast<const uint16_t*>(p)[i]) << 16);
}
template <>
__device__ __forceinline__ float load1<F16>(const void* p, int64_t i) {
  return float(static_cast<const _Float16*>(p)[i]);
}
template <>
__device__ __forceinline__ float load1<F32>(const void* p, int64_t i) {
  return static_cast<const float*>(p)[i];
}

template <class T>
__device__ __forceinline__ void store1(void* p, int64_t i, float x);
template <>
__device__ __forceinline__ void store1<Bf16>(void* p, int64_t i, float x) {
  static_cast<__bf16*>(p)[i] = (__bf16)x;
}
template <>
__device__ __forceinline__ void store1<F16>(void* p, int64_t i, float x) {
  static_cast<_Float16*>(p)[i] = (_Float16)x;
}
template <>
__device__ __forceinline__ void store1<F32>(void* p, int64_t i, float x) {
  static_cast<float*>(p)[i] = x;
}
template <>
__device__ __forceinline__ void store1<E4m3>(void* p, int64_t i, float x) {
  static_cast<uint8_t*>(p)[i] = uint8_t(pack4_e4m3(x, 0.f, 0.f, 0.f));
}

// Eight consecutive elements from element i on (16-byte aligned there; 8-byte
// for e4m3).
template <class T>
__device__ __forceinline__ void load8(const void* p, int64_t i, float* x) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = unpack2<T>(w[j]);
    x[2 * j] = f.x;
    x[2 * j + 1] = f.y;
  }
}
template <>
__device__ __forceinline__ void load8<F32>(const void* p, int64_t i, float* x) {
  const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
  const f32x4 a = q[0], b = q[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[j] = a[j];
    x[4 + j] = b[j];
  }
}

template <class T>
__device__ __forceinline__ void store8(void* p, int64_t i, const float* x) {
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = pack2<T>(x[2 * j], x[2 * j + 1]);
  *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + i) = w;
}
template <>
__device__ __forceinline__ void store8<F32>(void* p, int64_t i, const float* x) {
  f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + i);
  q[0] = f32x4{x[0], x[1], x[2], x[3]};
  q[1] = f32x4{x[4], x[5], x[6], x[7]};
}
template <>
__device__ __forceinline__ void store8<E4m3>(void* p, int64_t i, const float* x) {
  const u32x2 w = {pack4_e4m3(x[0], x[1], x[2], x[3]), pack4_e4m3(x[4], x[5], x[6], x[7])};
  *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(p) + i) = w;
}

// The same with four (8-byte aligned; 4-byte for e4m3), of 16-bit types.
template <class T>
__device__ __forceinline__ void load4(const void* p, int64_t i, float* x) {
  const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float2 f = unpack2<T>(w[j]);
    x[2 * j] = f.x;
    x[2 * j + 1] = f.y;
  }
}
template <class T>
__device__ __forceinline__ void store4(void* p, int64_t i, const float* x) {
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p) + i) = u32x2{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
}
template <>
__device__ __forceinline__ void store4<E4m3>(void* p, int64_t i, const float* x) {
  *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p) + i) = pack4_e4m3(x[0], x[1], x[2], x[3]);
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// The matrix products of the serving kernels: D[16 x 16] += A[16 x 32] B[32 x 16].
// Lane l holds row l % 16 of A and column l % 16 of B at the eight k of group
// l / 16, and of D column l % 16, rows 4 (l / 16) + 0..3.
template <class T>
__device__ __forceinline__ f32x4 mfma32(u32x4 a, u32x4 b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 mfma32<Bf16>(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 mfma32<F16>(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two e4m3 bytes (the low or high half of w) as a packed pair of T, exact.
template <class T, bool HIGH>
__device__ __forceinline__ uint32_t widen2(uint32_t w);
template <>
__device__ __forceinline__ uint32_t widen2<Bf16, false>(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
}
template <>
__device__ __forceinline__ uint32_t widen2<Bf16, true>(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
}
template <>
__device__ __forceinline__ uint32_t widen2<F16, false>(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
}
template <>
__device__ __forceinline__ uint32_t widen2<F16, true>(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true));
}

}  // namespace cp
