// 16-byte vectors of a caller's element type as floats, and back (device code).
#pragma once
#include "common.h"

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename V>
constexpr int kVec = 16 / (int)sizeof(V);  // values in 16 bytes

__device__ inline void widen(u32x4 w, float* v, float) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ inline void widen(u32x4 w, float* v, bf16_t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ inline void widen(u32x4 w, float* v, f16_t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = w[i];  // (the builtin takes the whole vector's first word when given w[i] itself)
    const f16_pair p = __builtin_bit_cast(f16_pair, u);
    v[2 * i] = (float)p[0];
    v[2 * i + 1] = (float)p[1];
  }
}
// rounded to nearest, ties to even; what half precision cannot hold becomes infinite, as a cast would make it
__device__ inline u32x4 narrow(const float* v, float) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(v[i]);
  return w;
}
__device__ inline u32x4 narrow(const float* v, bf16_t) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32_pair{v[2 * i], v[2 * i + 1]}), bf16_pair));
  return w;
}
__device__ inline u32x4 narrow(const float* v, f16_t) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32_pair{v[2 * i], v[2 * i + 1]}), f16_pair));
  return w;
}
__device__ inline float narrow1(float v, float) { return v; }
__device__ inline bf16_t narrow1(float v, bf16_t) { return f32_to_bf16(v); }
__device__ inline f16_t narrow1(float v, f16_t) { return f16_t{__builtin_bit_cast(uint16_t, (_Float16)v)}; }
