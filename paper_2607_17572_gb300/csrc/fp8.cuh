// e4m3 codes with one f32 scale for each group of 128 (the form include/jagg.h describes).
#pragma once

#include "common.cuh"

namespace jagg {
namespace fp8 {

constexpr int GROUP = 128;
constexpr float TOP = 448.f;  // the largest e4m3 value

// max(a, |v|) that keeps a NaN of either.
__device__ __forceinline__ float amax(float a, float v) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(fabsf(v)));
  return m;
}
// The scale of a group: the largest magnitude maps to 448.  The floor 2^-126 keeps the scale and its
// reciprocal normal numbers.  A NaN is kept, and makes every code of the group NaN; so is an infinity, whose
// reciprocal 0 makes the code of a finite element 0 and of an infinite one NaN, and times which all are NaN.
__device__ __forceinline__ float scale_of(float a) {
  const float s = a / TOP;
  return s < 1.17549435e-38f ? 1.17549435e-38f : s;
}
// Elements are multiplied by the scale's reciprocal (`inv` below), rounded to f32.  On bf16 inputs, whose quotient by
// the scale often lies next to a border between two codes, one code in 900 is the other neighbour of
// that border than the exact quotient's, and one in 770 when the quotient is rounded to f32 instead; what
// the codes stand for is as near to the inputs (relative 2-norm 0.025719 each).  That f32 quotient, from the
// product and its remainder, took 4608 x 4096 in row and column groups from 17.1 to 22.0 us.
//
// Two codes, `lo` in the low byte.  Rounds to nearest even; magnitudes over 448 (the group's largest
// element times a reciprocal that was rounded up) become 448, NaN stays NaN.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint2 pack8(const float (&v)[8], float inv) {
  const uint32_t a = pack2(v[0] * inv, v[1] * inv), b = pack2(v[2] * inv, v[3] * inv);
  const uint32_t c = pack2(v[4] * inv, v[5] * inv), d = pack2(v[6] * inv, v[7] * inv);
  return make_uint2(a | (b << 16), c | (d << 16));
}

// Eight consecutive elements as f32 (16-byte aligned), and back.
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<bf16>(const bf16* p, float (&v)[8]) {
  const uint4 a = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <>
__device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
template <>
__device__ __forceinline__ void store8<bf16>(bf16* p, const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&t);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
// f32 or bf16 by a flag (short vectors that are read once per row or column).
__device__ __forceinline__ float load_any(const void* p, int f32, int64_t i) {
  return f32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const bf16*>(p)[i]);
}
__device__ __forceinline__ void load8_any(const void* p, int f32, int64_t i, float (&v)[8]) {
  if (f32)
    load8(static_cast<const float*>(p) + i, v);
  else
    load8(static_cast<const bf16*>(p) + i, v);
}

inline bool aligned(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline int size_of(int dtype) { return dtype == JAGG_DTYPE_F32 ? 4 : 2; }
inline bool is_dtype(int dtype) { return dtype == JAGG_DTYPE_F32 || dtype == JAGG_DTYPE_BF16; }

}  // namespace fp8
}  // namespace jagg
