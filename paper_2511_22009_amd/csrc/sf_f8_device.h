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
  float inv;    // 1 / scale to a step, NaN too, 0 for a scale of 0, and -1 for one so small that differences are lost
};
// The quotient by the reciprocal of 448, corrected once by its remainder: correctly rounded, as the
// reciprocal is, wherever no part of it is below fp32's normal numbers. (With two divisions, 16384 x
// 1152 rows leave their norms as codes after 54 us instead of 50.)
__device__ __forceinline__ BlockF8 block_f8(uint32_t top_bits) {
  const float top = __uint_as_float(top_bits);
  constexpr float r = 1.0f / kF8Top;
  const float q = top * r, s = __builtin_fmaf(__builtin_fmaf(-q, kF8Top, top), r, q);
  BlockF8 b{s, __builtin_amdgcn_rcpf(s)};
  if (!(s >= 0x1p-90f && top_bits < 0x7f800000u)) {
    b.scale = top_bits < 0x7f800000u ? top / kF8Top : __uint_as_float(0x7fc00000u);
    b.inv = b.scale == 0.0f ? 0.0f : b.scale < 0x1p-90f ? -1.0f : b.scale;
  }
  return b;
}

// The code of x in a block of scale s > 0: the exact quotient's. The fp64 quotient of two fp32 numbers
// lies on the exact one's side of every tie: it is a tie only where that is one, since the quotient of
// two 24-bit significands that is not a number of five bits differs from one by over 2^-30 of itself.
__device__ __forceinline__ uint32_t code_f8_exact(float x, float s) {
  const uint32_t sign = __float_as_uint(x) >> 31 << 7;
  const double q = fmin(fabs((double)x) / (double)s, 448.0);
  if (q < 0x1p-6) return sign | (uint32_t)(int)rint(q * 512.0);
  const uint64_t b = (uint64_t)__double_as_longlong(q);
  const uint64_t r = b + ((1ull << 48) - 1) + ((b >> 49) & 1);
  return sign | ((uint32_t)(r >> 49) - (1016u << 3));
}

// Which of two adjacent codes, byte E of lo and of hi, is x's in a block of scale s >= 2^-90: the sign of
// |x| - tie s is the exact one's, as one fma rounds it, and where that is 0 the even code has it.
template <int E>
__device__ __forceinline__ uint32_t nearer_f8(uint32_t lo, uint32_t hi, float x, float s) {
  const float tie = 0.5f * (fabsf(__builtin_amdgcn_cvt_f32_fp8((int)lo, E)) + fabsf(__builtin_amdgcn_cvt_f32_fp8((int)hi, E)));
  const float over = __builtin_fmaf(-tie, s, fabsf(x));
  const uint32_t l = lo & (0xffu << (8 * E)), h = hi & (0xffu << (8 * E));
  return over > 0.0f || (over == 0.0f && !(h >> (8 * E) & 1)) ? h : l;
}

// Codes of N values of a block. x inv (1 -+ 2^-21) lie on both sides of the exact quotient (inv, a step off at most, and
// the two products add up to 2^-22 of it), and rounding is monotone, so where both give the same code
// it is the quotient's. Elsewhere, one value in some 2^16 and one in 16 where the scale is a power of
// two and the values are bf16, the exact quotient decides. (In fp64 it took 16384 x 1152 bf16
// from 13 to 19 us.)
template <int N>
__device__ __forceinline__ void codes_f8(const float (&x)[N], const BlockF8& b, uint32_t (&out)[N / 4]) {
  const float less = b.inv * (1.0f - 0x1p-21f), more = b.inv * (1.0f + 0x1p-21f);
  uint32_t hi[N / 4], differ = 0;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    out[i] = pack_f8(x[4 * i] * less, x[4 * i + 1] * less, x[4 * i + 2] * less, x[4 * i + 3] * less);
    hi[i] = pack_f8(x[4 * i] * more, x[4 * i + 1] * more, x[4 * i + 2] * more, x[4 * i + 3] * more);
    differ |= out[i] ^ hi[i];
  }
  if (b.inv < 0.0f) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      out[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) out[i] |= code_f8_exact(x[4 * i + e], b.scale) << (8 * e);
    }
  } else if (differ != 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      out[i] = nearer_f8<0>(out[i], hi[i], x[4 * i], b.scale) | nearer_f8<1>(out[i], hi[i], x[4 * i + 1], b.scale) |
               nearer_f8<2>(out[i], hi[i], x[4 * i + 2], b.scale) | nearer_f8<3>(out[i], hi[i], x[4 * i + 3], b.scale);
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
