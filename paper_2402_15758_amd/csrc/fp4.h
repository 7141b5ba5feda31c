// The 4-bit storage format of weights and of the 4-bit KV cache: groups of 32
// consecutive values share a scale 2^(s - 127), s one byte; a code is a sign
// and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.  gfx950 converts two codes with their
// scale in one instruction, and every such value is exact in bf16 (two
// significant bits), so a product over 4-bit values is a bf16 (or fp32) MFMA
// over exact operands.
#pragma once
#include "common.h"

constexpr int FP4_GROUP = 32;

// s = 255 is a quiet NaN for every code of the group: the conversion
// instructions give that for a scale operand whose exponent is all ones.
__device__ __forceinline__ float fp4_scale(uint32_t s) { return __uint_as_float(s << 23); }

// Eight codes of one word (the first in the low four bits) as bf16.
__device__ __forceinline__ int4 fp4_to_bf16x8(uint32_t w, float scale) {
  return int4{__builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
              __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
              __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
              __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3))};
}
// Codes 4 j .. 4 j + 3 of a word as floats.
template <int J>
__device__ __forceinline__ f32x4 fp4_to_f32x4(uint32_t w, float scale) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2 * J);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2 * J + 1);
  return f32x4{a[0], a[1], b[0], b[1]};
}

// An MFMA operand of 32 reduction indices: lane (g, c16) holds indices 8 g ..
// 8 g + 7 of its row or column.  One bf16 k-block, or two fp32 ones whose i-th
// instruction takes indices 8 g + 4 j + i.
template <typename T> struct Frag32;
template <> struct Frag32<bf16_t> {
  int4 v[1];
  __device__ __forceinline__ void from_fp4(uint32_t w, float scale) { v[0] = fp4_to_bf16x8(w, scale); }
};
template <> struct Frag32<float> {
  int4 v[2];
  __device__ __forceinline__ void from_fp4(uint32_t w, float scale) {
    v[0] = __builtin_bit_cast(int4, fp4_to_f32x4<0>(w, scale));
    v[1] = __builtin_bit_cast(int4, fp4_to_f32x4<1>(w, scale));
  }
};
template <typename T>
__device__ __forceinline__ f32x4 mfma32(const Frag32<T>& a, const Frag32<T>& b, f32x4 acc) {
  acc = mfma_kb<T>(a.v[0], b.v[0], acc);
  if constexpr (sizeof(T) == 4) acc = mfma_kb<T>(a.v[1], b.v[1], acc);
  return acc;
}

// Scale byte of a group whose largest magnitude is amax (as a float's bits):
// amax's exponent minus 2, one more where amax lies above 1.75 times its power
// of two and would round past 6.  At most 252, so that 6 times the scale stays
// finite; at least 1.  255 for an infinity or a NaN.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23);
  if (e == 255) return 255;
  return (uint32_t)min(max(e - 2 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0), 1), 252);
}
// Codes of eight values, rounded to nearest even and held to 6 times the scale.
__device__ __forceinline__ uint32_t fp4_encode8(const float (&v)[8], uint32_t s) {
  if (s == 255) return 0;
  const float sc = fp4_scale(s);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], sc, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], sc, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], sc, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], sc, 3);
  return w;
}
// Magnitude bits of the largest of eight values; NaN patterns exceed every
// number's, so the integer maximum keeps them.
__device__ __forceinline__ uint32_t amax_bits8(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  return m;
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = bf2f(p[e]);
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = p[e];
}

// The caller's rows may start at any element: loads and stores of eight values
// take 4-byte (fp32) or 2-byte (bf16) alignment.
template <typename T>
__device__ __forceinline__ void store8(T* p, uint32_t w, float scale);
template <>
__device__ __forceinline__ void store8<bf16_t>(bf16_t* p, uint32_t w, float scale) {
  typedef int i4_any __attribute__((ext_vector_type(4), aligned(2)));
  const int4 v = fp4_to_bf16x8(w, scale);
  *reinterpret_cast<i4_any*>(p) = i4_any{v.x, v.y, v.z, v.w};
}
template <>
__device__ __forceinline__ void store8<float>(float* p, uint32_t w, float scale) {
  typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
  const f32x4 a = fp4_to_f32x4<0>(w, scale), b = fp4_to_f32x4<1>(w, scale);
  *reinterpret_cast<f4_any*>(p) = f4_any{a[0], a[1], a[2], a[3]};
  *reinterpret_cast<f4_any*>(p + 4) = f4_any{b[0], b[1], b[2], b[3]};
}
