// What the kernels of the 8-bit codes and of the rotated heads share on the device.
#pragma once

#include "sf_device.h"
#include "sf_ops.h"

namespace sf {

// Two bf16 in a word, a in the low half (one conversion of both).
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const bf16x2 v = {(bf16)a, (bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// ---- 8-bit codes -----------------------------------------------------------------------
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// Largest |v| of a wavefront as the bit pattern of a non-negative float: patterns of such
// floats order like the numbers, and NaN lies above infinity, so unlike fmaxf a maximum of
// patterns keeps a NaN.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
template <int M>
__device__ __forceinline__ uint32_t xor_max(uint32_t v) {
  const uint32_t o = __float_as_uint(lane_xor<M>(__uint_as_float(v)));
  return v > o ? v : o;
}
__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
  return xor_max<1>(xor_max<2>(xor_max<4>(xor_max<8>(xor_max<16>(xor_max<32>(v))))));
}

// How the codes of a row follow from its largest magnitude: rint(127 x / top).
struct RowQuant {
  float top;    // largest magnitude; 0 for a row that is zero or not finite (codes 0)
  float inv;    // 127 / top, or 0 where that is no use
  float scale;  // top / 127, NaN for a row that is not finite
};
__device__ __forceinline__ RowQuant row_quant(uint32_t top_bits) {
  const float top = __uint_as_float(top_bits);
  const bool finite = top_bits < 0x7f800000u;
  RowQuant r;
  r.top = finite ? top : 0.0f;
  // below 1e-36 the reciprocal would overflow: every code from the quotient then
  r.inv = r.top >= 1e-36f ? 127.0f / r.top : 0.0f;
  r.scale = finite ? top / 127.0f : __uint_as_float(0x7fc00000u);
  return r;
}
// The code of one element. y = x inv is within 127 (2^-23 + 2^-46) < 2^-16 of the quotient
// 127 x / top, and y - rint(y) is exact, so rint(y) is the quotient's unless y lies within
// 2^-15 of a half. Then the quotient decides, in fp64: 127 x is exact there, and a quotient
// of at least 1/2 that is not itself a half differs from one by at least 2^-33 (x and top
// have 24-bit significands, and x is at least top / 254), far above the division's rounding.
constexpr float kQuantSure = 0.5f - 0x1p-15f;
__device__ __forceinline__ int quant_code_exact(float x, const RowQuant& r) {
  return r.top > 0.0f ? (int)rint((double)x * 127.0 / (double)r.top) : 0;
}
__device__ __forceinline__ int quant_code(float x, const RowQuant& r) {
  const float y = x * r.inv, q = rintf(y);
  return fabsf(y - q) < kQuantSure && r.inv != 0.0f ? (int)q : quant_code_exact(x, r);
}
// Codes of N elements, four to a word, the first in the low byte. y + 1.5 2^23 rounds y to a
// whole number, ties to even, and has its low byte in its own.
template <int N>
__device__ __forceinline__ void quant_codes(const float (&x)[N], const RowQuant& r, uint32_t (&out)[N / 4]) {
  constexpr float kWhole = 12582912.0f;
  uint32_t b[N];
  float off = 0.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float y = x[e] * r.inv, t = y + kWhole;
    off = fmaxf(off, fabsf(y - (t - kWhole)));
    b[e] = __float_as_uint(t);
  }
  if (!(off < kQuantSure) || r.inv == 0.0f) {
#pragma unroll
    for (int e = 0; e < N; ++e) b[e] = (uint32_t)quant_code_exact(x[e], r);
  }
  // bytes: __builtin_amdgcn_perm(hi, lo, sel) takes 0..3 from lo, 4..7 from hi and 0 for 12
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    out[i] = __builtin_amdgcn_perm(b[4 * i + 1], b[4 * i], 0x0c0c0400u) |
             __builtin_amdgcn_perm(b[4 * i + 3], b[4 * i + 2], 0x04000c0cu);
}

}  // namespace sf
