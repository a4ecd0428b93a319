// Rows to 8-bit codes with one scale per row: codes = rint(127 x / a), scale = a / 127, a
// the row's largest magnitude. Bandwidth bounds it (a row is read once and its codes are
// written once), so a wavefront holds its whole row in registers between the maximum and the
// codes: 16384 x 4608 bf16 takes 43.7 us, 5.2 TB/s (reading the row again for the codes, an
// element per lane, 134).
#include "sf_ops_device.h"

namespace sf {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Past the L2: 45.4 us otherwise, rows of 1152 13.0 instead of 14.0. (Loads past it as well: 41.8. They
// are as they are because the kernel of long rows shares them, which reads a row twice and loses, 2000 x
// 20000 35.8 instead of 31.1; a load of its own for the kernel that reads once was not measured.)
__device__ __forceinline__ void put_codes(int8_t* q, const uint32_t (&v)[2]) {
  __builtin_nontemporal_store(u32x2{v[0], v[1]}, (u32x2*)q);
}

// Chunks of eight elements at any element's address.
template <typename T> struct Chunk8;
template <> struct Chunk8<bf16> {
  typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2)));
  u32x4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *(const V*)p; }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      x[2 * w] = __uint_as_float(v[w] << 16);
      x[2 * w + 1] = __uint_as_float(v[w] & 0xffff0000u);
    }
  }
};
template <> struct Chunk8<float> {
  typedef uint32_t V __attribute__((ext_vector_type(4), aligned(4)));
  u32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *(const V*)p;
    b = *(const V*)(p + 4);
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      x[w] = __uint_as_float(a[w]);
      x[4 + w] = __uint_as_float(b[w]);
    }
  }
};

template <typename T>
__device__ __forceinline__ uint32_t chunk_top(const Chunk8<T>& c) {
  float x[8];
  c.unpack(x);
  uint32_t top = abs_bits(x[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) top = max(top, abs_bits(x[e]));
  return top;
}

// One wavefront per row; lane l holds chunks l, l + 64, ... (up to NC of them) and the element
// l of the part past the last whole chunk.
template <typename T, int NC>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= a.M) return;
  const T* row = (const T*)a.x + m * a.ldx;
  const int whole = a.K >> 3, rest = a.K & 7;
  Chunk8<T> c[NC];
  // unconditional at indexes that exist, so that no load waits for another
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (i * 64 < whole) c[i].load(row + 8 * min(lane + i * 64, whole - 1));
  const float last = rest ? to_f32(row[8 * whole + min(lane, rest - 1)]) : 0.0f;
  // a lane whose chunk is another lane's again does not change the maximum
  uint32_t top = abs_bits(last);
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (i * 64 < whole) top = max(top, chunk_top(c[i]));
  const RowQuant rq = row_quant(wave_max_bits(top));
  int8_t* q = a.q + m * a.ldq;
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (i * 64 < whole) {
      float x[8];
      c[i].unpack(x);
      uint32_t v[2];
      quant_codes(x, rq, v);
      if (lane + i * 64 < whole) put_codes(q + 8 * (lane + i * 64), v);
    }
  if (lane < rest) q[8 * whole + lane] = (int8_t)quant_code(last, rq);
  if (lane == 0) a.scale[m] = rq.scale;
}

// Rows too long for a wavefront's registers: one workgroup per row, which reads it again for
// the codes.
template <typename T>
__global__ __launch_bounds__(256) void quantize_long_rows_kernel(QuantArgs a) {
  __shared__ uint32_t tops[4];
  const int64_t m = blockIdx.x;
  const T* row = (const T*)a.x + m * a.ldx;
  const int whole = a.K >> 3, rest = a.K & 7;
  uint32_t top = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < whole; i += 256) {
    Chunk8<T> c;
    c.load(row + 8 * i);
    top = max(top, chunk_top(c));
  }
  const float last = (int)threadIdx.x < rest ? to_f32(row[8 * whole + threadIdx.x]) : 0.0f;
  top = wave_max_bits(max(top, abs_bits(last)));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  const RowQuant rq = row_quant(max(max(tops[0], tops[1]), max(tops[2], tops[3])));
  int8_t* q = a.q + m * a.ldq;
#pragma unroll 4
  for (int i = threadIdx.x; i < whole; i += 256) {
    Chunk8<T> c;
    c.load(row + 8 * i);
    float x[8];
    c.unpack(x);
    uint32_t v[2];
    quant_codes(x, rq, v);
    put_codes(q + 8 * i, v);
  }
  if ((int)threadIdx.x < rest) q[8 * whole + threadIdx.x] = (int8_t)quant_code(last, rq);
  if (threadIdx.x == 0) a.scale[m] = rq.scale;
}

template <typename T>
static hipError_t launch_quantize(const QuantArgs& a, hipStream_t s) {
  const dim3 grid((uint32_t)(((int64_t)a.M + 3) / 4)), block(256);
  if (a.K <= 1024)
    launch(quantize_rows_kernel<T, 2>, grid, block, 0, s, a);
  else if (a.K <= 4096)
    launch(quantize_rows_kernel<T, 8>, grid, block, 0, s, a);
  else if (a.K <= 8192)
    launch(quantize_rows_kernel<T, 16>, grid, block, 0, s, a);
  else
    launch(quantize_long_rows_kernel<T>, dim3((uint32_t)a.M), block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_quantize_rows(bool x_bf16, const QuantArgs& a, hipStream_t s) {
  return x_bf16 ? launch_quantize<bf16>(a, s) : launch_quantize<float>(a, s);
}

}  // namespace sf
