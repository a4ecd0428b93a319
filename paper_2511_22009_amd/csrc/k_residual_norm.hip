// A block's output into the residual stream and the next block's input in one pass:
//   u = post(y) post_gain,  h' = r h + gate u,  a = pre(h') pre_gain (1 + scale) + shift,
// each norm the division by the root mean square, or that of what the mean leaves, or none. Bandwidth
// bounds it: h and y are read once, h' and a written once, and a row stays in registers between its
// two norms. 4 x 4096 rows of 1152 dims, h fp32, y bf16, a as codes: 49 us, 4.2 TB/s (a as bf16 46, 4.9 TB/s; the rate
// of a large copy 41); 2760 rows of 771 dims in fp32 9.9; eight rows of 1152 4.5 in the kernel.
#include "sf_f8_device.h"
#include "sf_ops_rules.h"

namespace sf {

// Four elements out at any element's address: `left` of them exist.
template <typename T> struct Out4;
template <> struct Out4<float> {
  typedef float V __attribute__((ext_vector_type(4), aligned(4)));
  __device__ static void run(float* p, const float (&x)[4], int left) {
    if (left >= 4) {
      __builtin_nontemporal_store(V{x[0], x[1], x[2], x[3]}, (V*)p);
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
      __builtin_nontemporal_store(V{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])}, (V*)p);
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
// every size are normalised. A mean that is rounded stays in every deviation; where it is over 16 deviations large, what it
// left (of nearly one value, small multiples of one step, exactly) is normalised in the row's place, so a
// row of one value becomes 0. With that done always, 2760 x 771 rows took 10.9 us instead of 9.8.
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
      if (again > 0 || fabsf(sum) < 1e30f) mean = sum / (float)a.D;  // fp32's largest numbers stay so without it
    }
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[i][e] = first + i * STEP + e < a.D ? x[i][e] - mean : 0.0f;
        q = __builtin_fmaf(x[i][e], x[i][e], q);
      }
    q = row_sum<WAVES>(q, lds);
    if (again == 0 && !(q < 1e37f && q > 1e-28f && fabsf(sum) < 1e30f)) {
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
        // of large rows it would become 0, and a deviation of 0 times 1 / sqrt(0) NaN; next to another one this is nothing
        if (eps > 0.0f) eps = fmaxf(__builtin_amdgcn_ldexpf(__builtin_amdgcn_ldexpf(eps, by), by), 0x1p-126f);
        continue;
      }
      if (kind == NORM_LAYER && top >= 0x7f800000u) q = __uint_as_float(0x7fc00000u);  // as a mean that is not finite leaves it
    }
    q /= (float)a.D;
    if (again < 3 && q < 0x1p-8f * mean * mean) continue;
    const float by = 1.0f / sqrtf(q + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] *= by;
    return;
  }
}

// A piece of four of a row from column c on. WHOLE (D is a multiple of four): a lane past the row reads its last piece,
// unconditionally, since a load under a lane's condition is waited for at once; what is past D is cleared
// in use. Otherwise it is read element by element where D ends in it, and is 0 past D (reading the row's last
// four there and moving them to their places took 2760 x 771 from 9.8 to 12.9 us).
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_piece(Piece<T, 4>& p, const T* row, int c, int D) {
  if constexpr (WHOLE)
    p.load(row + min(c, D - 4), 4);
  else
    p.load(row + c, D - c);
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void take_piece(float (&x)[4], const Piece<T, 4>& p, int c, int D) {
  p.unpack(x);
  if constexpr (WHOLE) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = c < D ? x[e] : 0.0f;
  }
}

// A vector's pieces of a lane, `other` where there is none.
template <bool WHOLE, int NV, int STEP>
__device__ __forceinline__ void load_vector(float (&v)[NV][4], const float* p, int first, int D, float other) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = first + i * STEP;
    if (p) {
      Piece<float, 4> q;
      load_piece<WHOLE>(q, p, c, D);
      q.unpack(v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = other;
    }
  }
}

constexpr int threads_of(int waves) { return waves > 4 ? waves * 64 : 256; }

// WAVES wavefronts per row, NV pieces of four per lane (D <= 256 WAVES NV). A workgroup takes `span` rows of one
// sample in turn, fetches the next before it works on one, and keeps the sample's vectors, folded into
// three, in registers, fetched with its first row.
template <typename TH, typename TY, NormOut OUT, int NV, int WAVES, bool WHOLE>
__global__ __launch_bounds__(threads_of(WAVES)) void residual_norm_kernel(ResidualNormArgs a, FastDiv div_spans, int span) {
  __shared__ float lds[WAVES];
  constexpr int STEP = WAVES * 256, ROWS = threads_of(WAVES) / 64 / WAVES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t sample = fdiv(blockIdx.x, div_spans);
  const int start = (int)(blockIdx.x - sample * div_spans.d) * span, end = span_end(start, span, a.tokens);
  if (wave / WAVES >= end - start) return;  // whole wavefronts, and with several to a row whole workgroups
  int token = start + wave / WAVES;
  const int first = 4 * ((wave % WAVES) * 64 + (threadIdx.x & 63));
  const TH* const h = (const TH*)a.h + sample * a.h_sample;
  const TY* const y = (const TY*)a.y + sample * a.y_sample;
  Piece<TH, 4> hp[NV];
  Piece<TY, 4> yp[NV];
  auto fetch_y = [&](int t) {
#pragma unroll
    for (int i = 0; i < NV; ++i) load_piece<WHOLE>(yp[i], y + (int64_t)t * a.y_token, first + i * STEP, a.D);
  };
  auto fetch_h = [&](int t) {
#pragma unroll
    for (int i = 0; i < NV; ++i) load_piece<WHOLE>(hp[i], h + (int64_t)t * a.h_token, first + i * STEP, a.D);
  };
  // gate post_gain, pre_gain (1 + scale) and shift
  const float* const gate = a.gate ? a.gate + sample * a.gate_sample : nullptr;
  const float* const scale = a.scale ? a.scale + sample * a.scale_sample : nullptr;
  const float* const shift = a.shift ? a.shift + sample * a.shift_sample : nullptr;
  float vg[NV][4], vs[NV][4], vb[NV][4];
  fetch_y(token);
  fetch_h(token);
  {
    float w[NV][4];
    load_vector<WHOLE, NV, STEP>(vg, gate, first, a.D, 1.0f);
    load_vector<WHOLE, NV, STEP>(w, a.post_gain, first, a.D, 1.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) vg[i][e] *= w[i][e];
    if (a.out) {
      load_vector<WHOLE, NV, STEP>(vs, scale, first, a.D, 0.0f);
      load_vector<WHOLE, NV, STEP>(w, a.pre_gain, first, a.D, 1.0f);
      load_vector<WHOLE, NV, STEP>(vb, shift, first, a.D, 0.0f);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) vs[i][e] = w[i][e] * (1.0f + vs[i][e]);
    }
  }
  for (;;) {
    float x[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i) take_piece<WHOLE>(x[i], yp[i], first + i * STEP, a.D);
    const bool more = ROWS < end - token;
    fetch_y(row_ahead(token, ROWS, end));
    if (a.post != NORM_NONE) normalise<NV, WAVES>(x, a.post, a, first, lds);
    TH* const h_out = (TH*)a.h_out + sample * a.ho_sample + (int64_t)token * a.ho_token + first;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float hv[4];
      take_piece<WHOLE>(hv, hp[i], first + i * STEP, a.D);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][e] = __builtin_fmaf(a.r, hv[e], x[i][e] * vg[i][e]);
    }
    // before this row's h' leaves: over h itself, the last row is read again
    if (more) fetch_h(token + ROWS);
#pragma unroll
    for (int i = 0; i < NV; ++i) Out4<TH>::run(h_out + i * STEP, x[i], a.D - first - i * STEP);
    if (a.out) {
      if (a.pre != NORM_NONE) normalise<NV, WAVES>(x, a.pre, a, first, lds);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = first + i * STEP, left = a.D - c;
        const int64_t at = sample * a.out_sample + (int64_t)token * a.out_token + c;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = __builtin_fmaf(x[i][e], vs[i][e], vb[i][e]);
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
            __builtin_nontemporal_store(q[0], (uint32_t*)to);
          } else {
            for (int e = 0; e < 4; ++e)
              if (e < left) to[e] = (uint8_t)(q[0] >> (8 * e));
          }
          if ((threadIdx.x & 31) == 0 && left > 0)
            a.out_scale[sample * a.os_sample + (int64_t)token * a.os_token + (int64_t)(c / kF8Block) * a.os_block] = b.scale;
        } else if constexpr (OUT == NORM_F32) {
          Out4<float>::run((float*)a.out + at, x[i], left);
        } else {
          Out4<bf16>::run((bf16*)a.out + at, x[i], left);
        }
      }
    }
    if (!more) break;
    token += ROWS;
  }
}

template <typename TH, typename TY, NormOut OUT, int NV, int WAVES, bool WHOLE>
static void launch_rows(ResidualNormArgs a, hipStream_t s) {
  constexpr int ROWS = threads_of(WAVES) / 64 / WAVES;
  // as many workgroups as a CU holds at once, each as many rows of its sample as that takes (4096 x 1152 to codes: two
  // 17.9 us, four, which take turns, 21.3; 16384 x 768: three 32.6, four 27.9)
  constexpr int64_t kGroups = NV > 4 ? 512 : NV > 3 && WAVES == 1 ? 768 : 1024;
  const NormSpans p = norm_spans(a.samples, a.tokens, ROWS, kGroups);
  const FastDiv div = make_fastdiv(p.spans);
  in_parts(a.samples, p.most, [&](int64_t, int64_t n) {
    launch(residual_norm_kernel<TH, TY, OUT, NV, WAVES, WHOLE>, dim3((uint32_t)n * p.spans), dim3(threads_of(WAVES)), 0, s, a, div, p.span);
    a.h += n * a.h_sample * (int64_t)sizeof(TH);
    a.y += n * a.y_sample * (int64_t)sizeof(TY);
    a.h_out += n * a.ho_sample * (int64_t)sizeof(TH);
    if (a.out) a.out += n * a.out_sample * (OUT == NORM_CODES ? 1 : OUT == NORM_F32 ? 4 : 2);
    if (a.out_scale) a.out_scale += n * a.os_sample;
    if (a.gate) a.gate += n * a.gate_sample;
    if (a.scale) a.scale += n * a.scale_sample;
    if (a.shift) a.shift += n * a.shift_sample;
  });
}

#define SF_NORM_TILES(X) X(1, 1) X(3, 1) X(4, 1) X(5, 1) X(1, 4) X(2, 4) X(4, 4) X(2, 16) X(4, 16)

template <typename TH, typename TY, NormOut OUT>
static hipError_t launch_t(const ResidualNormArgs& a, hipStream_t s) {
  const NormTile t = choose_norm_tile((int64_t)a.samples * a.tokens, a.D);
#define SF_NORM_CASE(nv, w)                                                                            \
  if (t.pieces == nv && t.waves == w) {                                                                \
    if (a.D % 4 == 0)                                                                                  \
      launch_rows<TH, TY, OUT, nv, w, true>(a, s);                                                     \
    else if constexpr (norm_has_tile(NormTile{nv, w}, false))                                          \
      launch_rows<TH, TY, OUT, nv, w, false>(a, s);                                                    \
    else                                                                                               \
      return hipErrorInvalidValue;                                                                     \
    return hipGetLastError();                                                                          \
  }
  SF_NORM_TILES(SF_NORM_CASE)
#undef SF_NORM_CASE
  return hipErrorInvalidValue;
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
