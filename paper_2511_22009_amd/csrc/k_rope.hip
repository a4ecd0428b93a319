// Heads turned by positions with several axes, alone or after the norm of queries and keys
// per head, in one pass over the data.
//
// A pair (x, y) of a head's dims turns by u = p f, p its token's position on the pair's axis:
// (x cos u - y sin u, x sin u + y cos u). The angle of a pair is the same in every head, so
// a wavefront takes 64 / G tokens (G lanes to a head, each with the same E pairs of every
// head), forms its lanes' angles once and runs over heads with the cosines and sines in
// registers. The sum of squares of a head is a butterfly over its G lanes.
#include <cmath>

#include "sf_device.h"
#include "streamflow.h"

namespace sf {

// cos and sin of 2 pi turns. turns arrives in fp64, so that far positions keep their digits;
// 4 turns = n + f with |f| <= 1/2 leaves an angle of at most pi / 4, where the Taylor sums
// to x^9 and x^10 end 2e-9 and 2e-10 short, below fp32's rounding.
__device__ __forceinline__ void turn_angle(double turns, float& c, float& s) {
  const double t4 = turns * 4.0, n = rint(t4);
  const float x = (float)(t4 - n) * 1.57079632679489662f, x2 = x * x;
  const float sx = x * (1.0f + x2 * (-1.0f / 6 + x2 * (1.0f / 120 + x2 * (-1.0f / 5040 + x2 * (1.0f / 362880)))));
  const float cx =
      1.0f + x2 * (-0.5f + x2 * (1.0f / 24 + x2 * (-1.0f / 720 + x2 * (1.0f / 40320 + x2 * (-1.0f / 3628800)))));
  const double quarter = n - 4.0 * floor(n * 0.25);  // 0..3; NaN for a position that is not finite
  const bool odd = quarter == 1.0 || quarter == 3.0;
  const float a = odd ? sx : cx, b = odd ? cx : sx;
  c = quarter == 1.0 || quarter == 2.0 ? -a : a;
  s = quarter >= 2.0 ? -b : b;
}

#ifndef ROPE_WAVES
#define ROPE_WAVES 8192
#endif

// Vectors of E adjacent elements at any element's address.
template <typename T, int E> struct Piece;
template <> struct Piece<bf16, 8> { typedef uint32_t V __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Piece<bf16, 4> { typedef uint32_t V __attribute__((ext_vector_type(2), aligned(2))); };
template <> struct Piece<bf16, 1> { typedef uint16_t V; };
template <> struct Piece<float, 4> { typedef uint32_t V __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Piece<float, 1> { typedef uint32_t V; };

// E pairs of a head as they lie in memory: E elements at lo and E at hi (or, for adjacent
// bf16 pairs, the 8 elements at lo at once).
template <typename T, int E>
struct Pairs {
  typename Piece<T, E>::V lo, hi;
  __device__ __forceinline__ void load(const T* p, int l, int h) {
    lo = *(const typename Piece<T, E>::V*)(p + l);
    hi = *(const typename Piece<T, E>::V*)(p + h);
  }
};

template <typename T>
__device__ __forceinline__ float bits_f32(uint32_t b) {
  return sizeof(T) == 2 ? __uint_as_float(b << 16) : __uint_as_float(b);
}

template <typename T, int E>
__device__ __forceinline__ void unpack(const typename Piece<T, E>::V& v, float (&f)[E]) {
  if constexpr (E == 1) {
    f[0] = bits_f32<T>((uint32_t)v);
  } else if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      f[e] = __uint_as_float(v[e / 2] << 16);
      f[e + 1] = __uint_as_float(v[e / 2] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = __uint_as_float(v[e]);
  }
}

template <typename T, int E>
__device__ __forceinline__ void store(T* p, const float (&f)[E]) {
  if constexpr (E == 1) {
    *p = from_f32<T>(f[0]);
  } else if constexpr (sizeof(T) == 2) {
    typename Piece<T, E>::V v;
#pragma unroll
    for (int e = 0; e < E; e += 2)
      v[e / 2] = (uint32_t)__builtin_bit_cast(uint16_t, (bf16)f[e]) |
                 ((uint32_t)__builtin_bit_cast(uint16_t, (bf16)f[e + 1]) << 16);
    *(typename Piece<T, E>::V*)p = v;
  } else {
    typename Piece<T, E>::V v;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = __float_as_uint(f[e]);
    *(typename Piece<T, E>::V*)p = v;
  }
}

// E pairs per unit, U units per lane. E = 4 where a unit's elements are adjacent in memory,
// else 1. ADJ: the layout of adjacent pairs. blockIdx.y picks heads of q or of k, never of both.
template <typename T, int E, int U, bool ADJ, bool NORM, bool ROT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  constexpr int HB = 4;  // heads whose loads are in flight together
  const int lane = threadIdx.x & 63;
  const int G = 1 << a.group_log2, li = lane & (G - 1);
  const int per_wave = 64 >> a.group_log2;
  const uint32_t total = (uint32_t)a.rows * (uint32_t)a.tokens;
  const uint32_t first = ((uint32_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (uint32_t)per_wave;
  if (first >= total) return;  // uniform across the wavefront
  const uint32_t want = first + (uint32_t)(lane >> a.group_log2);
  const bool here = want < total;
  const uint32_t tt = here ? want : total - 1;
  const uint32_t row = fdiv(tt, a.div_tok), tok = tt - row * (uint32_t)a.tokens;
  const int which = (int)blockIdx.y >= a.splits0;
  const RopeHeads& t = a.t[which];
  const int h0 = ((int)blockIdx.y - (which ? a.splits0 : 0)) * a.head_step;
  const int h1 = min(h0 + a.head_step, which ? a.heads - a.heads0 : a.heads0);

  // this lane's units: where their elements are, and what takes a pair (x, y) of the head to
  // (x xx + y xy, x yx + y yy): the gains and the turn
  const int units = a.dh / (2 * E);
  int lo[U], hi[U];
  bool on[U], turns[U];
  float xx[U][E], xy[U][E], yx[U][E], yy[U][E];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int unit = li + u * G;
    on[u] = unit < units;
    const int j0 = on[u] ? unit * E : 0;
    turns[u] = ROT && j0 < a.pairs;
    lo[u] = 2 * j0;  // adjacent pairs, and the dims that stay
    hi[u] = lo[u] + E;
#pragma unroll
    for (int e = 0; e < E; ++e) xx[u][e] = yy[u][e] = 1.0f, xy[u][e] = yx[u][e] = 0.0f;
    if (turns[u]) {
      const float* p = a.pos + (int64_t)row * a.pos_row + (int64_t)tok * a.axes;
      int was = -1;
      double f = 0.0, step = 0.0, at = 0.0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int j = j0 + e;
        int ax = 0;
#pragma unroll
        for (int i = 1; i < kRopeAxes; ++i) ax += i < a.axes && j >= a.first[i];
        if (ax == was) {
          f *= step;  // the next pair of the axis
        } else {
          // the arrays by a dynamic index would go through memory
          int s0 = a.first[0], s1 = a.first[1];
          double rate = a.rate[0];
          step = a.step[0];
#pragma unroll
          for (int i = 1; i < kRopeAxes; ++i)
            if (ax == i) s0 = a.first[i], s1 = a.first[i + 1], rate = a.rate[i], step = a.step[i];
          f = exp2(-rate * (double)(a.spread ? j : j - s0)) * 0.15915494309189534;  // turns per position
          at = (double)p[ax];
          was = ax;
          if (e == 0 && !ADJ) {
            if (a.layout == SF_ROPE_HALVES) lo[u] = j0, hi[u] = j0 + a.pairs;
            if (a.layout == SF_ROPE_AXIS_HALVES) lo[u] = s0 + j0, hi[u] = s1 + j0;  // 2 s0 + (j0 - s0), + (s1 - s0)
          }
        }
        float c, s;
        turn_angle(at * f, c, s);
        xx[u][e] = yy[u][e] = c;
        xy[u][e] = a.inverse ? s : -s;
        yx[u][e] = -xy[u][e];
      }
    }
    if constexpr (NORM) {
      if (t.gain) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float gx = t.gain[ADJ && E == 4 ? lo[u] + 2 * e : lo[u] + e];
          const float gy = t.gain[ADJ && E == 4 ? lo[u] + 2 * e + 1 : hi[u] + e];
          xx[u][e] *= gx;
          yx[u][e] *= gx;
          xy[u][e] *= gy;
          yy[u][e] *= gy;
        }
      }
    }
  }
  const float inv_dh = 1.0f / (float)a.dh;
  const T* const in = (const T*)t.in + (int64_t)row * t.in_row + (int64_t)tok * t.in_tok;
  T* const out = (T*)t.out + (int64_t)row * t.out_row + (int64_t)tok * t.out_tok;
  for (int hb = h0; hb < h1; hb += HB) {
    Pairs<T, E> raw[HB][U];
#pragma unroll
    for (int b = 0; b < HB; ++b) {
      const T* p = in + (int64_t)min(hb + b, h1 - 1) * t.in_head;
#pragma unroll
      for (int u = 0; u < U; ++u) raw[b][u].load(p, lo[u], hi[u]);
    }
#pragma unroll
    for (int b = 0; b < HB; ++b) {
      const int h = hb + b;
      if (h >= h1) break;
      float x[U][E], y[U][E];
      float ss = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float p[E], q[E];
        unpack<T, E>(raw[b][u].lo, p);
        unpack<T, E>(raw[b][u].hi, q);
        if constexpr (ADJ && E == 4) {
          x[u][0] = p[0]; y[u][0] = p[1]; x[u][1] = p[2]; y[u][1] = p[3];
          x[u][2] = q[0]; y[u][2] = q[1]; x[u][3] = q[2]; y[u][3] = q[3];
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) x[u][e] = p[e], y[u][e] = q[e];
        }
        if constexpr (NORM) {
          float mine = 0.0f;
#pragma unroll
          for (int e = 0; e < E; ++e) mine += x[u][e] * x[u][e] + y[u][e] * y[u][e];
          ss += on[u] ? mine : 0.0f;
        }
      }
      float r = 1.0f;
      if constexpr (NORM) {
        if (G > 1) ss += lane_xor<1>(ss);
        if (G > 2) ss += lane_xor<2>(ss);
        if (G > 4) ss += lane_xor<4>(ss);
        if (G > 8) ss += lane_xor<8>(ss);
        if (G > 16) ss += lane_xor<16>(ss);
        if (G > 32) ss += lane_xor<32>(ss);
        r = 1.0f / sqrtf(ss * inv_dh + a.eps);
      }
      T* const o = out + (int64_t)h * t.out_head;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float p[E], q[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if constexpr (NORM) x[u][e] *= r, y[u][e] *= r;
          // a dim that stays is not touched by its neighbour, which may be infinite
          p[e] = turns[u] ? x[u][e] * xx[u][e] + y[u][e] * xy[u][e] : x[u][e] * xx[u][e];
          q[e] = turns[u] ? x[u][e] * yx[u][e] + y[u][e] * yy[u][e] : y[u][e] * yy[u][e];
        }
        if constexpr (ADJ && E == 4) {
          const float lo4[4] = {p[0], q[0], p[1], q[1]}, hi4[4] = {p[2], q[2], p[3], q[3]};
#pragma unroll
          for (int e = 0; e < 4; ++e) p[e] = lo4[e], q[e] = hi4[e];
        }
        if (here && on[u]) {
          if constexpr (ADJ && E == 4 && sizeof(T) == 2) {
            const float all[8] = {p[0], p[1], p[2], p[3], q[0], q[1], q[2], q[3]};
            store<T, 8>(o + lo[u], all);
          } else {
            store<T, E>(o + lo[u], p);
            store<T, E>(o + hi[u], q);
          }
        }
      }
    }
  }
}

template <typename T, bool NORM, bool ROT>
static hipError_t launch_rope_as(const RopeArgs& a, bool whole, dim3 grid, hipStream_t s) {
  if (!whole)
    launch(rope_kernel<T, 1, 2, false, NORM, ROT>, grid, dim3(256), 0, s, a);
  else if (!ROT || a.layout == SF_ROPE_ADJACENT)
    launch(rope_kernel<T, 4, 1, true, NORM, ROT>, grid, dim3(256), 0, s, a);
  else
    launch(rope_kernel<T, 4, 1, false, NORM, ROT>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_rope(bool is_bf16, bool norm, bool rotate, RopeArgs a, hipStream_t s) {
  // units of four pairs where every unit's elements are adjacent: whole units in the head, in
  // the part that turns and, where each axis has halves of its own, in each axis
  bool whole = a.dh % 8 == 0;
  if (rotate) {
    whole = whole && a.pairs % 4 == 0;
    if (a.layout == SF_ROPE_AXIS_HALVES)
      for (int i = 1; i < a.axes; ++i) whole = whole && a.first[i] % 4 == 0;
  }
  const int lanes = whole ? a.dh / 8 : (a.dh / 2 + 1) / 2;
  a.group_log2 = 0;
  while ((1 << a.group_log2) < lanes) ++a.group_log2;
  for (int i = 0; i < a.axes; ++i) {
    // frequencies fall by 2^rate from pair to pair
    const int n = a.spread ? a.pairs : a.first[i + 1] - a.first[i];
    a.rate[i] = n > 0 ? a.log2_theta / n : 0.0;
    a.step[i] = exp2(-a.rate[i]);
  }
  const int64_t per_wave = 64 >> a.group_log2;
  const int64_t waves = ((int64_t)a.rows * a.tokens + per_wave - 1) / per_wave;
  // heads are split over wavefronts while there are fewer than kWaves of them
  int64_t splits = (ROPE_WAVES + waves - 1) / waves;
  if (splits > a.heads) splits = a.heads;
  a.head_step = (int)((a.heads + splits - 1) / splits);
  a.splits0 = (a.heads0 + a.head_step - 1) / a.head_step;
  const int splits1 = (a.heads - a.heads0 + a.head_step - 1) / a.head_step;
  const dim3 grid((uint32_t)((waves + 3) / 4), (uint32_t)(a.splits0 + splits1));
  if (is_bf16) {
    if (norm) return rotate ? launch_rope_as<bf16, true, true>(a, whole, grid, s) : launch_rope_as<bf16, true, false>(a, whole, grid, s);
    return launch_rope_as<bf16, false, true>(a, whole, grid, s);
  }
  if (norm) return rotate ? launch_rope_as<float, true, true>(a, whole, grid, s) : launch_rope_as<float, true, false>(a, whole, grid, s);
  return launch_rope_as<float, false, true>(a, whole, grid, s);
}

}  // namespace sf
