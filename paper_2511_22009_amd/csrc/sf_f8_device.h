// e4m3 codes on the device: how a block's codes follow from its largest magnitude.
#pragma once

#include "sf_ops_device.h"

namespace sf {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kF8Top = 448.0f;  // the largest e4m3 number

// Largest of 2^n adjacent lanes, as the bit patterns of abs_bits.
__device__ __forceinline__ uint32_t max_of_16(uint32_t v) { return xor_max<1>(xor_max<2>(xor_max<4>(xor_max<8>(v)))); }
__device__ __forceinline__ uint32_t max_of_32(uint32_t v) { return max_of_16(xor_max<16>(v)); }

// Four codes in a word, the first in the low byte: nearest, ties to even.
__device__ __forceinline__ uint32_t pack_f8(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// A block's scale, top / 448, and what takes its values to codes.
struct BlockF8 {
  float scale;  // NaN for a block that is not finite
  float inv;    // 1 / scale; 0 where fp32 does not hold it to full precision, or scale is 0 or NaN
};
__device__ __forceinline__ BlockF8 block_f8(uint32_t top_bits) {
  const float s = __uint_as_float(top_bits) / kF8Top;
  BlockF8 b;
  b.scale = top_bits < 0x7f800000u ? s : __uint_as_float(0x7fc00000u);
  b.inv = s >= 0x1p-126f && top_bits < 0x7f800000u ? 1.0f / s : 0.0f;
  return b;
}

// The code of x in a block of scale s: the exact quotient's. The fp64 quotient of two fp32 numbers
// lies on the exact one's side of every tie: it is a tie only where that is one, since the quotient of
// two 24-bit significands that is not a number of five bits differs from one by over 2^-30 of itself.
__device__ __forceinline__ uint32_t code_f8_exact(float x, float s) {
  if (s != s) return 0x7f;
  if (s == 0.0f) return 0;
  const uint32_t sign = __float_as_uint(x) >> 31 << 7;
  const double q = fmin(fabs((double)x) / (double)s, 448.0);
  if (q < 0x1p-6) return sign | (uint32_t)(int)rint(q * 512.0);
  const uint64_t b = (uint64_t)__double_as_longlong(q);
  const uint64_t r = b + ((1ull << 48) - 1) + ((b >> 49) & 1);
  return sign | ((uint32_t)(r >> 49) - (1016u << 3));
}

// Codes of N values of a block. x inv (1 -+ 2^-22) lie on both sides of the exact quotient (inv and the
// two products add less than 2^-22 of it), and rounding is monotone, so where both give the same code
// it is the quotient's. Elsewhere, one value in some 2^16, the exact quotient decides.
template <int N>
__device__ __forceinline__ void codes_f8(const float (&x)[N], const BlockF8& b, uint32_t (&out)[N / 4]) {
  const float lo = b.inv * (1.0f - 0x1p-22f), hi = b.inv * (1.0f + 0x1p-22f);
  uint32_t differ = 0;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    out[i] = pack_f8(x[4 * i] * lo, x[4 * i + 1] * lo, x[4 * i + 2] * lo, x[4 * i + 3] * lo);
    differ |= out[i] ^ pack_f8(x[4 * i] * hi, x[4 * i + 1] * hi, x[4 * i + 2] * hi, x[4 * i + 3] * hi);
  }
  if (differ != 0 || b.inv == 0.0f) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      out[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) out[i] |= code_f8_exact(x[4 * i + e], b.scale) << (8 * e);
    }
  }
}

// N adjacent values at any element's address: `left` of them exist, the others are 0.
template <typename T, int N> struct Piece;
template <int N> struct Piece<bf16, N> {
  typedef uint32_t V __attribute__((ext_vector_type(N / 2), aligned(2)));
  uint32_t v[N / 2];
  __device__ __forceinline__ void load(const bf16* p, int left) {
    if (left >= N) {
      const V w = *(const V*)p;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) v[i] = w[i];
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        v[i] = 2 * i < left ? (uint32_t)((const uint16_t*)p)[2 * i] : 0u;
        if (2 * i + 1 < left) v[i] |= (uint32_t)((const uint16_t*)p)[2 * i + 1] << 16;
      }
    }
  }
  __device__ __forceinline__ void unpack(float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
};
template <int N> struct Piece<float, N> {
  typedef float V __attribute__((ext_vector_type(4), aligned(4)));
  float v[N];
  __device__ __forceinline__ void load(const float* p, int left) {
    if (left >= N) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        const V w = *(const V*)(p + 4 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * i + e] = w[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = e < left ? p[e] : 0.0f;
    }
  }
  __device__ __forceinline__ void unpack(float (&x)[N]) const {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = v[e];
  }
};

}  // namespace sf
