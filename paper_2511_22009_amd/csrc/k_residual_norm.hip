// A block's output into the residual stream and the next block's input in one pass:
//   u = post(y) post_gain,  h' = r h + gate u,  a = pre(h') pre_gain (1 + scale) + shift,
// each norm the division by the root mean square, or that of what the mean leaves, or none. Bandwidth
// bounds it: h and y are read once, h' and a written once, and a row stays in registers between its
// two norms.
#include "sf_f8_device.h"

namespace sf {

// Four elements out at any element's address: `left` of them exist.
template <typename T> struct Out4;
template <> struct Out4<float> {
  typedef float V __attribute__((ext_vector_type(4), aligned(4)));
  __device__ static void run(float* p, const float (&x)[4], int left) {
    if (left >= 4) {
      *(V*)p = V{x[0], x[1], x[2], x[3]};
    } else {
      for (int e = 0; e < 4; ++e)
        if (e < left) p[e] = x[e];
    }
  }
};
template <> struct Out4<bf16> {
  typedef uint32_t V __attribute__((ext_vector_type(2), aligned(2)));
  __device__ static void run(bf16* p, const float (&x)[4], int left) {
    if (left >= 4) {
      *(V*)p = V{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    } else {
      for (int e = 0; e < 4; ++e)
        if (e < left) p[e] = (bf16)x[e];
    }
  }
};

// Sum, and largest bit pattern, over the WAVES wavefronts of a row.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  v = wave_sum(v);
  if constexpr (WAVES > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += lds[w];
  }
  return v;
}
template <int WAVES>
__device__ __forceinline__ uint32_t row_max(uint32_t v, float* lds) {
  v = wave_max_bits(v);
  if constexpr (WAVES > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = __uint_as_float(v);
    __syncthreads();
    v = __float_as_uint(lds[0]);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = max(v, __float_as_uint(lds[w]));
  }
  return v;
}

// x of a row (pieces of four, zeros past D, also afterwards) becomes its norm without a gain. Where the squares or the sum leave
// what fp32 holds to full precision, the row is scaled by a power of two first, so finite rows of
// every size are normalised.
template <int NV, int WAVES>
__device__ __forceinline__ void normalise(float (&x)[NV][4], int kind, const ResidualNormArgs& a, int first, float* lds) {
  constexpr int STEP = WAVES * 256;
  float eps = a.eps;
  for (int again = 0;; ++again) {
    float mean = 0.0f, sum = 0.0f;
    if (kind == NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < NV; ++i) sum += (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
      sum = row_sum<WAVES>(sum, lds);
      mean = sum / (float)a.D;
    }
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float c = first + i * STEP + e < a.D ? x[i][e] - mean : 0.0f;
        q = __builtin_fmaf(c, c, q);
      }
    q = row_sum<WAVES>(q, lds);
    if (again == 0 && !(q < 1e37f && q > 1e-28f && fabsf(sum) < 1e37f)) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, abs_bits(x[i][e]));
      top = row_max<WAVES>(top, lds);
      if (top > 0 && top < 0x7f800000u) {
        int e = __builtin_amdgcn_frexp_expf(__uint_as_float(top));
        if (eps > 0.0f) e = max(e, __builtin_amdgcn_frexp_expf(eps) / 2);  // next to eps, smaller rows are as good as zeros
        const int by = -e;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) x[i][c] = __builtin_amdgcn_ldexpf(x[i][c], by);
        eps = __builtin_amdgcn_ldexpf(__builtin_amdgcn_ldexpf(eps, by), by);
        continue;
      }
    }
    const float by = 1.0f / sqrtf(q / (float)a.D + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = first + i * STEP + e < a.D ? (x[i][e] - mean) * by : 0.0f;
    return;
  }
}

// WAVES wavefronts per row, NV pieces of four per lane (D <= 256 WAVES NV).
template <typename TH, typename TY, NormOut OUT, int NV, int WAVES>
__global__ __launch_bounds__(256) void residual_norm_kernel(ResidualNormArgs a, FastDiv div_tokens, int64_t row0, int rows) {
  __shared__ float lds[4];
  constexpr int STEP = WAVES * 256;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = blockIdx.x * (4 / WAVES) + wave / WAVES;
  if (part >= rows) return;  // whole wavefronts, and with several to a row whole workgroups
  const uint32_t row = (uint32_t)(row0 + part);
  const uint32_t sample = fdiv(row, div_tokens), token = row - sample * div_tokens.d;
  const int first = 4 * ((wave % WAVES) * 64 + (threadIdx.x & 63));
  const TH* const h = (const TH*)a.h + sample * a.h_sample + token * a.h_token;
  const TY* const y = (const TY*)a.y + sample * a.y_sample + token * a.y_token;
  Piece<TH, 4> hp[NV];
  Piece<TY, 4> yp[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = first + i * STEP;
    yp[i].load(y + c, a.D - c);
    hp[i].load(h + c, a.D - c);
  }
  float x[NV][4];
#pragma unroll
  for (int i = 0; i < NV; ++i) yp[i].unpack(x[i]);
  if (a.post != NORM_NONE) normalise<NV, WAVES>(x, a.post, a, first, lds);
  const float* const gate = a.gate ? a.gate + sample * a.gate_sample : nullptr;
  TH* const h_out = (TH*)a.h_out + sample * a.ho_sample + token * a.ho_token;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = first + i * STEP, left = a.D - c;
    Piece<float, 4> p;
    float v[4];
    if (a.post_gain) {
      p.load(a.post_gain + c, left);
      p.unpack(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] *= v[e];
    }
    if (gate) {
      p.load(gate + c, left);
      p.unpack(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] *= v[e];
    }
    float hv[4];
    hp[i].unpack(hv);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i][e] = __builtin_fmaf(a.r, hv[e], x[i][e]);
    Out4<TH>::run(h_out + c, x[i], left);
  }
  if (!a.out) return;
  if (a.pre != NORM_NONE) normalise<NV, WAVES>(x, a.pre, a, first, lds);
  const float* const scale = a.scale ? a.scale + sample * a.scale_sample : nullptr;
  const float* const shift = a.shift ? a.shift + sample * a.shift_sample : nullptr;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = first + i * STEP, left = a.D - c;
    Piece<float, 4> p;
    float v[4];
    if (a.pre_gain) {
      p.load(a.pre_gain + c, left);
      p.unpack(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] *= v[e];
    }
    if (scale) {
      p.load(scale + c, left);
      p.unpack(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = __builtin_fmaf(x[i][e], v[e], x[i][e]);
    }
    if (shift) {
      p.load(shift + c, left);
      p.unpack(v);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] += v[e];
    }
    const int64_t at = sample * a.out_sample + token * a.out_token + c;
    if constexpr (OUT == NORM_CODES) {
      // 32 lanes hold a block
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) top = max(top, e < left ? abs_bits(x[i][e]) : 0u);
      const BlockF8 b = block_f8(max_of_32(top));
      uint32_t q[1];
      codes_f8(x[i], b, q);
      uint8_t* const to = (uint8_t*)a.out + at;
      if (left >= 4) {
        *(uint32_t*)to = q[0];
      } else {
        for (int e = 0; e < 4; ++e)
          if (e < left) to[e] = (uint8_t)(q[0] >> (8 * e));
      }
      if ((threadIdx.x & 31) == 0 && left > 0)
        a.out_scale[sample * a.os_sample + token * a.os_token + (int64_t)(c / kF8Block) * a.os_block] = b.scale;
    } else if constexpr (OUT == NORM_F32) {
      Out4<float>::run((float*)a.out + at, x[i], left);
    } else {
      Out4<bf16>::run((bf16*)a.out + at, x[i], left);
    }
  }
}

template <typename TH, typename TY, NormOut OUT, int NV, int WAVES>
static void launch_rows(const ResidualNormArgs& a, hipStream_t s) {
  const FastDiv div = make_fastdiv((uint32_t)a.tokens);
  constexpr int64_t kMost = 1 << 23;  // a grid holds less than 2^32 threads
  const int64_t rows = (int64_t)a.samples * a.tokens;
  for (int64_t r = 0; r < rows; r += kMost) {
    const int n = (int)(rows - r < kMost ? rows - r : kMost);
    launch(residual_norm_kernel<TH, TY, OUT, NV, WAVES>, dim3((uint32_t)((n + 4 / WAVES - 1) / (4 / WAVES))), dim3(256), 0, s, a, div, r, n);
  }
}

template <typename TH, typename TY, NormOut OUT>
static hipError_t launch_t(const ResidualNormArgs& a, hipStream_t s) {
  if (a.D <= 256) launch_rows<TH, TY, OUT, 1, 1>(a, s);
  else if (a.D <= 768) launch_rows<TH, TY, OUT, 3, 1>(a, s);
  else if (a.D <= 1280) launch_rows<TH, TY, OUT, 5, 1>(a, s);
  else if (a.D <= 2048) launch_rows<TH, TY, OUT, 8, 1>(a, s);
  else if (a.D <= 4096) launch_rows<TH, TY, OUT, 4, 4>(a, s);
  else if (a.D <= 8192) launch_rows<TH, TY, OUT, 8, 4>(a, s);
  else launch_rows<TH, TY, OUT, 16, 4>(a, s);
  return hipGetLastError();
}

template <typename TH, typename TY>
static hipError_t launch_ty(NormOut out, const ResidualNormArgs& a, hipStream_t s) {
  switch (out) {
    case NORM_BF16: return launch_t<TH, TY, NORM_BF16>(a, s);
    case NORM_F32: return launch_t<TH, TY, NORM_F32>(a, s);
    case NORM_CODES: return launch_t<TH, TY, NORM_CODES>(a, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_residual_norm(bool h_bf16, bool y_bf16, NormOut out, const ResidualNormArgs& a, hipStream_t s) {
  if (h_bf16) return y_bf16 ? launch_ty<bf16, bf16>(out, a, s) : launch_ty<bf16, float>(out, a, s);
  return y_bf16 ? launch_ty<float, bf16>(out, a, s) : launch_ty<float, float>(out, a, s);
}

}  // namespace sf
