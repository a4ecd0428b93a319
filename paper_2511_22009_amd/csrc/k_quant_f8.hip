// Rows and weights to e4m3 codes with a scale per block of 128 columns (of one row, or of 128):
// scale = top / 448, top the block's largest magnitude, code = the e4m3 number nearest to x / scale.
// Bandwidth bounds it: every value is read once and held in registers between the maximum and the code. 16384 x
// 1152 bf16 takes 11.6 us, 4.9 TB/s, into memory that no cache holds; a kernel that only copies that much 9.4,
// codes without the check for ties 11.0.
#include "sf_f8_device.h"

namespace sf {

// Sixteen lanes take one row of a block of columns, eight values each, a workgroup WAVES 4 ITS rows of it: eight rows
// per wavefront where there are many (four 12.6 us instead of 11.6, sixteen 12.9; a wavefront on 512 columns of
// one row 14.2). SQUARE: the workgroup's 128 rows share their scale, and sixteen wavefronts read them.
template <typename T, int WAVES, int ITS, bool SQUARE>
__global__ __launch_bounds__(WAVES * 64) void quantize_f8_kernel(QuantF8Args a, int kblocks) {
  constexpr int STEP = WAVES * 4;
  static_assert(!SQUARE || STEP * ITS == kF8Block, "a workgroup takes one block");
  const int tid = threadIdx.x, sub = tid & 15, row = tid >> 4;
  const int kb = blockIdx.x % kblocks, rb = blockIdx.x / kblocks;
  const int col = kb * kF8Block + 8 * sub, left = a.K - col;
  const int m0 = rb * STEP * ITS + row;
  Piece<T, 8> p[ITS];
  uint32_t top[ITS];
#pragma unroll
  for (int i = 0; i < ITS; ++i)  // rows past the last one are read as it
    p[i].load((const T*)a.x + (int64_t)min(m0 + STEP * i, a.M - 1) * a.ldx + col, left);
#pragma unroll
  for (int i = 0; i < ITS; ++i) {
    float x[8];
    p[i].unpack(x);
    uint32_t t = abs_bits(x[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) t = max(t, abs_bits(x[e]));
    top[i] = t;
  }
  if constexpr (SQUARE) {
    __shared__ uint32_t tops[WAVES];
#pragma unroll
    for (int i = 1; i < ITS; ++i) top[0] = max(top[0], top[i]);
    const uint32_t t = wave_max_bits(top[0]);
    if ((tid & 63) == 0) tops[tid >> 6] = t;
    __syncthreads();
    top[0] = tops[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top[0] = max(top[0], tops[w]);
    if (tid == 0) a.scale[(int64_t)rb * a.s_row + (int64_t)kb * a.s_block] = block_f8(top[0]).scale;
  }
#pragma unroll
  for (int i = 0; i < ITS; ++i) {
    const int m = m0 + STEP * i;
    const BlockF8 b = block_f8(SQUARE ? top[0] : max_of_16(top[i]));
    float x[8];
    p[i].unpack(x);
    uint32_t c[2];
    codes_f8(x, b, c);
    if (m >= a.M) continue;
    if (!SQUARE && sub == 0) a.scale[(int64_t)m * a.s_row + (int64_t)kb * a.s_block] = b.scale;
    uint8_t* const to = a.q + (int64_t)m * a.ldq + col;
    if (left >= 8) {
      __builtin_nontemporal_store(u32x2{c[0], c[1]}, (u32x2*)to);  // past the L2: 12.6 us otherwise
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) to[e] = (uint8_t)(c[e >> 2] >> (8 * (e & 3)));
    }
  }
}

template <typename T>
static hipError_t launch_f8(bool square, const QuantF8Args& a, hipStream_t s) {
  const int kblocks = (a.K + kF8Block - 1) / kF8Block;
  const auto grid = [&](int rows) { return dim3((uint32_t)(((int64_t)a.M + rows - 1) / rows * kblocks)); };
  if (square)
    launch(quantize_f8_kernel<T, 16, 2, true>, grid(128), dim3(1024), 0, s, a, kblocks);
  else if (a.M > 16)
    launch(quantize_f8_kernel<T, 4, 2, false>, grid(32), dim3(256), 0, s, a, kblocks);
  else
    launch(quantize_f8_kernel<T, 4, 1, false>, grid(16), dim3(256), 0, s, a, kblocks);
  return hipGetLastError();
}

hipError_t launch_quantize_f8(bool x_bf16, bool square, const QuantF8Args& a, hipStream_t s) {
  return x_bf16 ? launch_f8<bf16>(square, a, s) : launch_f8<float>(square, a, s);
}

}  // namespace sf
