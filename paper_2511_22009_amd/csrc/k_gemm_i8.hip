// Products of 8-bit codes on the matrix cores, out[m][n] = (sum_k A[m][k] B[n][k]) sa[m] sb[n]
// + bias[n]: v_mfma_i32_32x32x32_i8, whose 32-bit sums are exact for every K the entry point
// allows, on 64 x 64 tiles over 128-wide slices of K.
#include "sf_device.h"

namespace sf {

template <typename OT>
__global__ __launch_bounds__(256) void gemm_i8_kernel(GemmI8Args a) {
  constexpr int BM = 64, BN = 64, BK = 128, LD = BK + 16;
  __shared__ __attribute__((aligned(16))) char As[BM * LD];
  __shared__ __attribute__((aligned(16))) char Bs[BN * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1, l32 = lane & 31, g = lane >> 5;
  const int nbn = (a.N + BN - 1) / BN;
  const int m0 = (int)(blockIdx.x / nbn) * BM, n0 = (int)(blockIdx.x % nbn) * BN;
  i32x16 acc;
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[r] = 0;
  // 16 bytes of row `row` of X at column k; bytes of rows and columns that do not exist are 0
  auto chunk = [&](const int8_t* X, int ld, int rows, int row, int k) {
    i32x4 v = {0, 0, 0, 0};
    if (row < rows && k < a.K) {
      v = *(const i32x4*)(X + (int64_t)row * ld + k);
      const int left = a.K - k;
      if (left < 16) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int n = left - 4 * w;
          if (n < 4) v[w] = n > 0 ? (int)((uint32_t)v[w] & ((1u << (8 * n)) - 1u)) : 0;
        }
      }
    }
    return v;
  };
  for (int k0 = 0; k0 < a.K; k0 += BK) {
    __syncthreads();
    for (int c = tid; c < BM * 8; c += 256)
      *(i32x4*)&As[(c >> 3) * LD + (c & 7) * 16] = chunk(a.A, a.lda, a.M, m0 + (c >> 3), k0 + (c & 7) * 16);
    for (int c = tid; c < BN * 8; c += 256)
      *(i32x4*)&Bs[(c >> 3) * LD + (c & 7) * 16] = chunk(a.B, a.ldb, a.N, n0 + (c >> 3), k0 + (c & 7) * 16);
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const i32x4 x = *(const i32x4*)&As[(wm * 32 + l32) * LD + kk * 32 + g * 16];
      const i32x4 y = *(const i32x4*)&Bs[(wn * 32 + l32) * LD + kk * 32 + g * 16];
      acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(y, x, acc, 0, 0, 0);
    }
  }
  // lane (l32, g) holds row l32 and the columns 8 q + 4 g + e
  const int m = m0 + wm * 32 + l32;
  if (m >= a.M) return;
  const float sa = a.sa[m];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n = n0 + wn * 32 + q * 8 + g * 4 + e;
      if (n >= a.N) continue;
      const float p = (float)acc[4 * q + e] * sa * a.sb[n];
      ((OT*)a.out)[(int64_t)m * a.ldo + n] = from_f32<OT>(a.bias ? p + a.bias[n] : p);
    }
}

hipError_t launch_gemm_i8(bool out_bf16, const GemmI8Args& a, hipStream_t s) {
  const int64_t tiles = (((int64_t)a.M + 63) / 64) * (((int64_t)a.N + 63) / 64);
  if (tiles > 0x7fffffff) return hipErrorInvalidValue;
  if (out_bf16)
    launch(gemm_i8_kernel<bf16>, dim3((uint32_t)tiles), dim3(256), 0, s, a);
  else
    launch(gemm_i8_kernel<float>, dim3((uint32_t)tiles), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace sf
