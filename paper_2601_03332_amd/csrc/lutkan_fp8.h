// What the kernels on 8-bit floating point share (lutkan_fp8_norm.hip, lutkan_fp8_matmul.hip): rows of any alignment, the three
// 32- and 16-bit types, blocks of 128 that share a scale.
#pragma once

#include "lutkan_device.h"

namespace {

constexpr int kScaleBlock = 128;                  // columns (and rows of a weight) that share a scale
constexpr float kFp8Largest = 448.0f;             // the largest finite value of e4m3
constexpr float kFp8SmallestScale = 0x1p-126f;    // so that a scale and its reciprocal are normal numbers, for a block of zeros too

inline bool is_type(int t) { return t == LUTKAN_F32 || t == LUTKAN_F16 || t == LUTKAN_BF16; }
__host__ __device__ constexpr int type_bytes(int t) { return t == LUTKAN_F32 ? 4 : 2; }

// A copy of N bytes in one access whatever the alignment: gfx950 takes unaligned addresses in its global loads and stores.
template <typename V>
__device__ __forceinline__ V load_any(const void *p) {
  V v;
  __builtin_memcpy(&v, p, sizeof(V));
  return v;
}
template <typename V>
__device__ __forceinline__ void store_any(void *p, const V &v) { __builtin_memcpy(p, &v, sizeof(V)); }

__device__ __forceinline__ unsigned bf16_bits(float v) { return (unsigned)__builtin_bit_cast(unsigned short, (__bf16)v); }   // nearest, ties to even
__device__ __forceinline__ unsigned f16_bits(float v) { return (unsigned)__builtin_bit_cast(unsigned short, (_Float16)v); }
__device__ __forceinline__ float bf16_value(unsigned bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ float f16_value(unsigned bits) { return (float)__builtin_bit_cast(_Float16, (unsigned short)bits); }

template <int TYPE>
__device__ __forceinline__ float load_one(const unsigned char *p) {
  if constexpr (TYPE == LUTKAN_F32) return load_any<float>(p);
  else if constexpr (TYPE == LUTKAN_F16) return f16_value(load_any<unsigned short>(p));
  else return bf16_value(load_any<unsigned short>(p));
}
template <int TYPE>
__device__ __forceinline__ void store_one(unsigned char *p, float v) {
  if constexpr (TYPE == LUTKAN_F32) store_any(p, v);
  else store_any(p, (unsigned short)(TYPE == LUTKAN_F16 ? f16_bits(v) : bf16_bits(v)));
}

// Eight consecutive elements as they lie in memory, and their values.
template <int TYPE>
struct Raw8 {
  u32x4 v[TYPE == LUTKAN_F32 ? 2 : 1];
};
template <int TYPE>
__device__ __forceinline__ Raw8<TYPE> load_raw8(const unsigned char *p) { return load_any<Raw8<TYPE>>(p); }
template <int TYPE>
__device__ __forceinline__ void values8(const Raw8<TYPE> &r, float (&out)[8]) {
  if constexpr (TYPE == LUTKAN_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = __uint_as_float(r.v[e >> 2][e & 3]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const unsigned half = (r.v[0][e >> 1] >> ((e & 1) * 16)) & 0xffffu;
      out[e] = TYPE == LUTKAN_F16 ? f16_value(half) : bf16_value(half);
    }
  }
}
template <int TYPE>
__device__ __forceinline__ void store8(unsigned char *p, const float (&v)[8]) {
  Raw8<TYPE> r;
  if constexpr (TYPE == LUTKAN_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e >> 2][e & 3] = __float_as_uint(v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      r.v[0][e] = TYPE == LUTKAN_F16 ? f16_bits(v[2 * e]) | (f16_bits(v[2 * e + 1]) << 16) : bf16_bits(v[2 * e]) | (bf16_bits(v[2 * e + 1]) << 16);
  }
  store_any(p, r);
}

// max |v| as the bits of the absolute value: their order as whole numbers is that of the values, and a NaN is above all of them, so
// that a block that holds one gets a NaN scale.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// A block's scale from the largest magnitude in it; NaN stays NaN (the comparison fails).
__device__ __forceinline__ float block_scale(unsigned largest) {
  const float s = __uint_as_float(largest) / kFp8Largest;
  return s < kFp8SmallestScale ? kFp8SmallestScale : s;
}

// Eight codes of v / scale, rounded to nearest, ties to even.  The quotient is v * inverse corrected by its own remainder, so that it is
// rounded once: v * inverse alone can fall on the other side of a tie.  A scale that was rounded down lets it pass 448 by 2^-24 of it,
// which the conversion rounds back.  Infinities and NaN only come with a scale that is not finite either, and then every code is NaN or
// stands for it.
__device__ __forceinline__ float quotient(float v, float scale, float inverse) {
  const float q = v * inverse;
  return fmaf(fmaf(-q, scale, v), inverse, q);
}
__device__ __forceinline__ u32x2 codes8(const float (&v)[8], float scale) {
  const float inverse = 1.0f / scale;
  u32x2 c;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int word = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[4 * h], scale, inverse), quotient(v[4 * h + 1], scale, inverse), 0, false);
    word = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[4 * h + 2], scale, inverse), quotient(v[4 * h + 3], scale, inverse), word, true);
    c[h] = (unsigned)word;
  }
  return c;
}

inline int64_t scale_blocks(int64_t n) { return (n + kScaleBlock - 1) / kScaleBlock; }

}  // namespace
