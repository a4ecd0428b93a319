// Rows to 8-bit codes with one scale per row: codes = rint(127 x / a), scale = a / 127, a
// the row's largest magnitude.
#include "sf_device.h"

namespace sf {

template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= a.M) return;
  const T* row = (const T*)a.x + m * a.ldx;
  uint32_t top = 0;
  for (int k = lane; k < a.K; k += 64) top = max(top, abs_bits(to_f32(row[k])));
  const RowQuant rq = row_quant(wave_max_bits(top));
  int8_t* q = a.q + m * a.ldq;
  for (int k = lane; k < a.K; k += 64) q[k] = (int8_t)quant_code(to_f32(row[k]), rq);
  if (lane == 0) a.scale[m] = rq.scale;
}

hipError_t launch_quantize_rows(bool x_bf16, const QuantArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)a.M + 3) / 4));
  if (x_bf16)
    launch(quantize_rows_kernel<bf16>, grid, dim3(256), 0, s, a);
  else
    launch(quantize_rows_kernel<float>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace sf
