// Heads turned by positions with several axes, alone or after the norm of queries and keys
// per head, in one pass over the data.
//
// A pair (x, y) of a head's dims turns by u = p f, p its token's position on the pair's axis:
// (x cos u - y sin u, x sin u + y cos u). The angle of a pair is the same in every head, so a
// workgroup forms the angles of its tokens once, in fp64, and shares them over the heads; G
// lanes hold a head, and its sum of squares is a butterfly over them.
//
// Bandwidth bounds it: the 8 x 30 x 52 tokens of a clip with 16 heads of 128 dims (102 MB) take
// 16 us, 6.4 TB/s; q and k of 16384 tokens with 32 heads of 64 dims (134 MB, adjacent pairs) 22.5
// us, 6.0, as halves 28. With 72 dims a head fills 9 of its 16 lanes, and halves move in pieces of
// 8 bytes: 30 us for 151 MB, 5.1 TB/s; heads next to each other in packed rows 43. (Groups of 9 lanes,
// their sums in thirds through the LDS crossbar, made 4 % there and cost 5 where q and k lie
// packed; pieces of 16 bytes, eight pairs to a lane, nothing for 128 dims and 4.5 instead of 3.6 us
// for a single token; 12 pairs to a lane, wavefronts by tokens throughout and angles per wavefront
// lost 3 to 10 %.)
#include <algorithm>
#include <cmath>

#include "sf_ops_device.h"
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

// N adjacent elements at any element's address, moved in pieces of 16 and 8 bytes.
template <typename T, int N>
struct Run {
  static constexpr int WORDS = N * (int)sizeof(T) / 4;
  static_assert(WORDS % 2 == 0, "whole pieces of 8 bytes");
  typedef uint32_t V4 __attribute__((ext_vector_type(4), aligned(2)));
  typedef uint32_t V2 __attribute__((ext_vector_type(2), aligned(2)));
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i + 4 <= WORDS; i += 4) {
      const V4 v = *(const V4*)((const char*)p + 4 * i);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[i + k] = v[k];
    }
    if constexpr (WORDS % 4 == 2) {
      const V2 v = *(const V2*)((const char*)p + 4 * (WORDS - 2));
      w[WORDS - 2] = v[0];
      w[WORDS - 1] = v[1];
    }
  }
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 2)
      return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    else
      return __uint_as_float(w[e]);
  }
  template <bool PAST>
  __device__ static __forceinline__ void put(void* p, V4 v) {
    if constexpr (PAST) __builtin_nontemporal_store(v, (V4*)p);
    else *(V4*)p = v;
  }
  template <bool PAST>
  __device__ static __forceinline__ void put(void* p, V2 v) {
    if constexpr (PAST) __builtin_nontemporal_store(v, (V2*)p);
    else *(V2*)p = v;
  }
  template <bool PAST>
  __device__ static __forceinline__ void store(T* p, const float (&f)[N]) {
    uint32_t o[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(T) == 2)
        o[i] = pack_bf16(f[2 * i], f[2 * i + 1]);
      else
        o[i] = __float_as_uint(f[i]);
    }
#pragma unroll
    for (int i = 0; i + 4 <= WORDS; i += 4) put<PAST>((char*)p + 4 * i, V4{o[i], o[i + 1], o[i + 2], o[i + 3]});
    if constexpr (WORDS % 4 == 2) put<PAST>((char*)p + 4 * (WORDS - 2), V2{o[WORDS - 2], o[WORDS - 1]});
  }
};
template <typename T>
struct Run<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ float at(int) const { return to_f32(v); }
  template <bool PAST>
  __device__ static __forceinline__ void store(T* p, const float (&f)[1]) { *p = from_f32<T>(f[0]); }
};

// E pairs of a head as they lie in memory: E elements at lo and E at hi, or, adjacent pairs, 2 E
// elements at lo.
template <typename T, int E, bool ADJ>
struct Pairs {
  Run<T, E> lo, hi;
  __device__ __forceinline__ void load(const T* p, int l, int h) {
    lo.load(p + l);
    hi.load(p + h);
  }
  __device__ __forceinline__ float x(int e) const { return lo.at(e); }
  __device__ __forceinline__ float y(int e) const { return hi.at(e); }
  template <bool PAST>
  __device__ static __forceinline__ void store(T* p, int l, int h, const float (&x)[E], const float (&y)[E]) {
    Run<T, E>::template store<PAST>(p + l, x);
    Run<T, E>::template store<PAST>(p + h, y);
  }
};
template <typename T, int E>
struct Pairs<T, E, true> {
  Run<T, 2 * E> run;
  __device__ __forceinline__ void load(const T* p, int l, int) { run.load(p + l); }
  __device__ __forceinline__ float x(int e) const { return run.at(2 * e); }
  __device__ __forceinline__ float y(int e) const { return run.at(2 * e + 1); }
  template <bool PAST>
  __device__ static __forceinline__ void store(T* p, int l, int, const float (&x)[E], const float (&y)[E]) {
    float f[2 * E];
#pragma unroll
    for (int e = 0; e < E; ++e) f[2 * e] = x[e], f[2 * e + 1] = y[e];
    Run<T, 2 * E>::template store<PAST>(p + l, f);
  }
};

// Where a lane's heads lie and how outputs leave (the choice is at launch_rope): a wavefront takes a
// head of several tokens, through the L2 or past it, or several heads of one token, past it.
enum RopeOut { ROPE_PLAIN, ROPE_PAST, ROPE_BY_HEADS };

constexpr int kMostHeads = 32;  // of a lane's in a run, which has a bit for each

// A workgroup of four wavefronts takes 64 / G tokens (by heads: four); its first threads form a
// pair's angle of a token each and leave cosine and sine in LDS, under the wavefronts' first loads.
// A wavefront takes a run of heads of q or of k.
// E pairs per unit, U units per lane: one unit of four pairs whose elements are adjacent in
// memory, or two of one pair each (an element at a time: 98 dims 2.4 to 3.2 TB/s, 36 dims 2.3).
// ADJ: the layout of adjacent pairs. PART: some dims stay as they are.
// One pass over a workgroup's heads; FAR: over those alone that the first pass leaves, whose squares fp32
// does not hold. Returns which of the lane's heads it left, a bit each (what memory holds does not
// tell: results over their inputs may be such heads).
template <typename T, int E, int U, bool ADJ, bool NORM, bool ROT, bool PART, RopeOut OUT, bool FAR>
__device__ __forceinline__ uint32_t rope_pass(const RopeArgs& a, int tid, float2* angles, uint32_t far) {
  constexpr int HB = 2;  // heads (of each lane) whose loads are in flight together
  constexpr bool kByHeads = OUT == ROPE_BY_HEADS;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = 1 << a.group_log2, li = lane & (G - 1);
  const uint32_t total = (uint32_t)a.rows * (uint32_t)a.tokens;
  // each of the eight XCDs (workgroup b goes to XCD b % 8) takes a contiguous range of tokens:
  // a cache line that two workgroups' tokens share is read and written in one L2
  const uint32_t xcd = blockIdx.x % 8, base = gridDim.x / 8, rem = gridDim.x % 8;
  const int slots = 64 >> a.group_log2, in_slot = lane >> a.group_log2;
  const uint32_t first = (xcd * base + min(xcd, rem) + blockIdx.x / 8) * (uint32_t)(kByHeads ? 4 : slots);
  // a lane's token of the workgroup's, the heads a wavefront takes at once, and the lane's of them
  const int slot = kByHeads ? wave : in_slot, abreast = kByHeads ? slots : 1, mine = kByHeads ? in_slot : 0;
  const bool here = first + slot < total;
  const uint32_t tt = here ? first + slot : total - 1;
  const uint32_t row = fdiv(tt, a.div_tok), tok = tt - row * (uint32_t)a.tokens;
  const int chunk = kByHeads ? (int)blockIdx.y : (int)blockIdx.y * 4 + wave;
  const int which = chunk >= a.chunks0;
  const RopeHeads& t = a.t[which];
  const int heads = which ? a.heads - a.heads0 : a.heads0, step = a.step[which];
  const int h0 = (which ? chunk - a.chunks0 : chunk) * step, h1 = min(h0 + step, heads);

  // where this lane's units are
  const int units = a.dh / (2 * E);
  int lo[U], hi[U], pair[U];
  bool on[U], turns[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int unit = li + u * G;
    on[u] = unit < units;
    const int j0 = pair[u] = on[u] ? unit * E : 0;
    turns[u] = ROT && (!PART || j0 < a.pairs);
    lo[u] = 2 * j0;  // adjacent pairs, and the dims that stay
    hi[u] = lo[u] + E;
    if (ROT && !ADJ && turns[u]) {
      if (a.layout == SF_ROPE_HALVES) lo[u] = j0, hi[u] = j0 + a.pairs;
      if (a.layout == SF_ROPE_AXIS_HALVES) {
        int s0 = a.first[0], s1 = a.first[1];
#pragma unroll
        for (int i = 1; i < kRopeAxes; ++i)
          if (j0 >= a.first[i]) s0 = a.first[i], s1 = a.first[i + 1];
        lo[u] = s0 + j0, hi[u] = s1 + j0;  // 2 s0 + (j0 - s0), + (s1 - s0)
      }
    }
  }
  const T* const in = (const T*)t.in + (int64_t)row * t.in_row + (int64_t)tok * t.in_tok;
  T* const out = (T*)t.out + (int64_t)row * t.out_row + (int64_t)tok * t.out_tok;
  Pairs<T, E, ADJ> raw[HB][U];
  auto load = [&](int h) {
#pragma unroll
    for (int b = 0; b < HB; ++b)
#pragma unroll
      for (int u = 0; u < U; ++u) raw[b][u].load(in + (int64_t)min(h + b * abreast + mine, h1 - 1) * t.in_head, lo[u], hi[u]);
  };
  if (h0 < h1) load(h0);

  if constexpr (ROT && !FAR) {
    const int here_pairs = (int)min((uint32_t)(kByHeads ? 4 : slots), total - first) * a.pairs;
    for (int c = tid; c < here_pairs; c += 256) {
      const int at = (int)fdiv((uint32_t)c, a.div_pairs), j = c - at * a.pairs;
      const uint32_t r = fdiv(first + at, a.div_tok), k = first + at - r * (uint32_t)a.tokens;
      int ax = 0, s0 = a.first[0];
      double rate = a.rate[0];
#pragma unroll
      for (int i = 1; i < kRopeAxes; ++i)  // the arrays by a dynamic index would go through memory
        if (i < a.axes && j >= a.first[i]) ax = i, s0 = a.first[i], rate = a.rate[i];
      const double f = exp2(-rate * (double)(a.spread ? j : j - s0)) * 0.15915494309189534;  // turns per position
      float c1, s1;
      turn_angle((double)a.pos[(int64_t)r * a.pos_row + (int64_t)k * a.axes + ax] * f, c1, s1);
      angles[c] = make_float2(c1, a.inverse ? -s1 : s1);
    }
    __syncthreads();
  }
  if (h0 >= h1) return 0;

  // what takes a pair (x, y) to (x xx + y xy, x yx + y yy): the gains and the turn
  float xx[U][E], xy[U][E], yx[U][E], yy[U][E];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float2 w = make_float2(1.0f, 0.0f);
      if (ROT && turns[u] && here) w = angles[slot * a.pairs + pair[u] + e];
      xx[u][e] = yy[u][e] = w.x;
      xy[u][e] = -w.y;
      yx[u][e] = w.y;
      if constexpr (NORM) {
        if (t.gain) {
          const float gx = t.gain[ADJ ? lo[u] + 2 * e : lo[u] + e];
          const float gy = t.gain[ADJ ? lo[u] + 2 * e + 1 : hi[u] + e];
          xx[u][e] *= gx;
          yx[u][e] *= gx;
          xy[u][e] *= gy;
          yy[u][e] *= gy;
        }
      }
      // a dim that stays has no part in its neighbour, whatever its gain
      if (PART && !turns[u]) xy[u][e] = yx[u][e] = 0.0f;
    }
  const float inv_dh = 1.0f / (float)a.dh;
  uint32_t left = 0, bit = 1;
  for (int hb = h0; hb < h1; hb += HB * abreast, bit <<= HB) {
    float x[HB][U][E], y[HB][U][E];
#pragma unroll
    for (int b = 0; b < HB; ++b)
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[b][u][e] = raw[b][u].x(e), y[b][u][e] = raw[b][u].y(e);
      }
    if (hb + HB * abreast < h1) load(hb + HB * abreast);
    float r[HB];
    bool put[HB];
    if constexpr (NORM) {
      // reciprocal roots of the mean squares and eps of the batch's heads, times the square of s(b)
      auto roots = [&](auto s) {
#pragma unroll
        for (int b = 0; b < HB; ++b) {
          r[b] = 0.0f;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float mine = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float xe = x[b][u][e] * s(b), ye = y[b][u][e] * s(b);
              mine += __builtin_fmaf(xe, xe, ye * ye);
            }
            r[b] += on[u] ? mine : 0.0f;
          }
        }
        // the sums of the batch's heads over their G lanes
        auto add = [&](auto m) {
#pragma unroll
          for (int b = 0; b < HB; ++b) r[b] += lane_xor<decltype(m)::value>(r[b]);
        };
        if (G > 1) add(std::integral_constant<int, 1>{});
        if (G > 2) add(std::integral_constant<int, 2>{});
        if (G > 4) add(std::integral_constant<int, 4>{});
        if (G > 8) add(std::integral_constant<int, 8>{});
        if (G > 16) add(std::integral_constant<int, 16>{});
        if (G > 32) add(std::integral_constant<int, 32>{});
#pragma unroll
        for (int b = 0; b < HB; ++b) r[b] = __builtin_amdgcn_rsqf(r[b] * inv_dh + a.eps * s(b) * s(b));  // within 1 ulp
      };
      roots([](int) { return 1.0f; });
#pragma unroll
      for (int b = 0; b < HB; ++b) {
        // no root: 0, of a sum that overflows, or infinity, of 0 and of subnormal numbers, which the
        // instruction takes for 0
        put[b] = FAR ? (far & (bit << b)) != 0 : !__builtin_amdgcn_classf(r[b], 0x240);
        left |= put[b] ? 0 : bit << b;
      }
      if constexpr (FAR) {
        // Times a power of two, which rounds nothing. What overflows has a mean (with eps) of 2^120 and more:
        // times 2^-70, that is a normal number, and every square is below 2^116. A mean below 2^-126
        // has elements below 2^-59: times 2^100, every square is a normal number. (A mean that is
        // one has lost at most 2^-150 to subnormal squares, half a step of itself.) Heads of zeros with
        // eps 0 and heads that hold an infinity keep a root of infinity and 0: 0 / 0, inf / inf.
        constexpr float kDown = 0x1p-70f, kUp = 0x1p100f;
        const bool down[HB] = {r[0] < 1.0f, r[1] < 1.0f};  // 0, not infinity
        roots([&](int b) { return down[b] ? kDown : kUp; });
#pragma unroll
        for (int b = 0; b < HB; ++b) {
          // x (s / root), as x s would lose bits of small elements; upwards (x s) / root, as s / root
          // would overflow
          r[b] *= down[b] ? kDown : 1.0f;
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) x[b][u][e] *= down[b] ? 1.0f : kUp, y[b][u][e] *= down[b] ? 1.0f : kUp;
        }
      }
    }
#pragma unroll
    for (int b = 0; b < HB; ++b) {
      const int h = hb + b * abreast + mine;
      if (hb + b * abreast >= h1) break;
      T* const o = out + (int64_t)h * t.out_head;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float p[E], q[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          float xe = x[b][u][e], ye = y[b][u][e];
          if constexpr (NORM) xe *= r[b], ye *= r[b];
          if constexpr (ROT) {
            // a dim that stays is not touched by its neighbour, which may be infinite
            const float xt = PART && !turns[u] ? 0.0f : xe, yt = PART && !turns[u] ? 0.0f : ye;
            // (which of the two products is not rounded is written out, so that no build changes a bit)
            p[e] = __builtin_fmaf(xe, xx[u][e], yt * xy[u][e]);
            q[e] = NORM && PART ? __builtin_fmaf(ye, yy[u][e], xt * yx[u][e]) : __builtin_fmaf(xt, yx[u][e], ye * yy[u][e]);
          } else {
            p[e] = xe * xx[u][e];
            q[e] = ye * yy[u][e];
          }
        }
        if (here && on[u] && h < h1 && (!NORM || put[b])) Pairs<T, E, ADJ>::template store<OUT != ROPE_PLAIN>(o, lo[u], hi[u], p, q);
      }
    }
  }
  return left;
}

template <typename T, int E, int U, bool ADJ, bool NORM, bool ROT, bool PART, RopeOut OUT>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  __shared__ __attribute__((aligned(16))) float2 angles[ROT ? (OUT == ROPE_BY_HEADS ? 512 : 64 * E * U) : 1];  // [token][pair]
  typedef const __attribute__((address_space(4))) RopeArgs* Kernarg;  // where `a` lies
  Kernarg args = (Kernarg)__builtin_amdgcn_kernarg_segment_ptr();
  uint32_t left;
  // Through the pointer the arguments are loaded where they are used, as `a` all at the start: by heads
  // 31.4 and 32.8 us (q and k of 16384 tokens in packed rows, 16 heads of 72 dims), the others 6.2 and
  // 6.0 (the same of 4096 tokens, 12 heads of 64).
  if constexpr (OUT == ROPE_BY_HEADS)
    left = rope_pass<T, E, U, ADJ, NORM, ROT, PART, OUT, false>(*(const RopeArgs*)args, (int)threadIdx.x, angles, 0);
  else
    left = rope_pass<T, E, U, ADJ, NORM, ROT, PART, OUT, false>(a, (int)threadIdx.x, angles, 0);
  if constexpr (NORM) {
    if (!__any(left != 0)) return;
    // The heads that were left, in a pass of their own, which finds its places again (the empty asm
    // hides that it has them, so that no register is kept for it): a branch to the scaling within
    // the loop cost 2 to 4 %.
    int tid = (int)threadIdx.x;
    asm volatile("" : "+v"(tid), "+s"(args));
    rope_pass<T, E, U, ADJ, NORM, ROT, PART, OUT, true>(*(const RopeArgs*)args, tid, angles, left);
  }
}

template <typename T, bool NORM, bool ROT, bool PART>
static hipError_t launch_rope_as(const RopeArgs& a, bool whole, RopeOut out, dim3 grid, hipStream_t s) {
  const auto go = [&](auto out) {
    constexpr RopeOut O = decltype(out)::value;
    if constexpr (ROT) {
      if (a.layout != SF_ROPE_ADJACENT) return launch(rope_kernel<T, 4, 1, false, NORM, ROT, PART, O>, grid, dim3(256), 0, s, a);
    }
    launch(rope_kernel<T, 4, 1, true, NORM, ROT, PART, O>, grid, dim3(256), 0, s, a);
  };
  if (!whole)
    launch(rope_kernel<T, 1, 2, false, NORM, ROT, PART, ROPE_PLAIN>, grid, dim3(256), 0, s, a);
  else if (out == ROPE_BY_HEADS)
    go(std::integral_constant<RopeOut, ROPE_BY_HEADS>{});
  else if (out == ROPE_PAST)
    go(std::integral_constant<RopeOut, ROPE_PAST>{});
  else
    go(std::integral_constant<RopeOut, ROPE_PLAIN>{});
  return hipGetLastError();
}

template <typename T>
static hipError_t launch_rope_type(const RopeArgs& a, bool norm, bool rotate, bool whole, RopeOut out, dim3 grid, hipStream_t s) {
  const bool part = 2 * a.pairs < a.dh;
  if (!rotate) return launch_rope_as<T, true, false, false>(a, whole, out, grid, s);
  if (norm) return part ? launch_rope_as<T, true, true, true>(a, whole, out, grid, s) : launch_rope_as<T, true, true, false>(a, whole, out, grid, s);
  return part ? launch_rope_as<T, false, true, true>(a, whole, out, grid, s) : launch_rope_as<T, false, true, false>(a, whole, out, grid, s);
}

// norm without rotation, rotation without norm, or both.
hipError_t launch_rope(bool is_bf16, bool norm, bool rotate, RopeArgs a, hipStream_t s) {
  if (!norm && !rotate) return hipErrorInvalidValue;
  // units of four pairs where each lies in one piece: whole units in the head, in the part that
  // turns and, where each axis has halves of its own, in each axis
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
  }
  a.div_pairs = make_fastdiv(a.pairs > 0 ? a.pairs : 1);
  const int heads1 = a.heads - a.heads0, slots = 64 >> a.group_log2;
  // Outputs past the L2 where a head's tokens follow each other, or its dims are whole pieces of 64
  // bytes: q and k of 16384 tokens with 16 heads of 72 dims 30.5 instead of 42.7 us, a clip's 16.2
  // instead of 21. Where a token's heads follow each other instead, and only several of them are whole
  // pieces, a wavefront takes several heads of one token, past the L2 too: q and k of 16384 tokens in
  // packed rows with 16 heads of 72 dims 43 instead of 47 us, with 28 heads of 40 dims 39 instead of 55
  // (a head of several tokens past the L2, its ends sharing pieces: 52 at 72 dims).
  const int64_t size = is_bf16 ? 2 : 4;
  bool past = true, runs = whole && size * a.dh * slots % 64 == 0;
  for (int i = 0; i < 2; ++i) {
    const RopeHeads& t = a.t[i];
    if (i ? heads1 == 0 : a.heads0 == 0) continue;
    const int64_t at = (int64_t)(uintptr_t)t.out | size * (t.out_tok | t.out_row);
    past = past && (t.out_tok == a.dh || (at | size * (a.dh | t.out_head)) % 64 == 0);
    runs = runs && t.out_head == a.dh && at % 64 == 0;
  }
  const RopeOut out = past ? ROPE_PAST : runs ? ROPE_BY_HEADS : ROPE_PLAIN;
  const bool by_heads = out == ROPE_BY_HEADS;
  const int per = by_heads ? 4 : slots, abreast = by_heads ? slots : 1, waves = by_heads ? 1 : 4;
  const int64_t groups = ((int64_t)a.rows * a.tokens + per - 1) / per;
  // heads are split over workgroups too while there are fewer than that of them
  int64_t splits = (1024 + groups - 1) / groups;
  const int most = (a.heads + 3) / 4;
  if (splits > most) splits = most;
  if (by_heads && a.heads0 > 0 && heads1 > 0 && splits < 2) splits = 2;
  const auto run = [&](int heads, int n) { return n > 0 ? ((heads + n - 1) / n + abreast - 1) / abreast * abreast : 1; };
  const int longest = kMostHeads * abreast;
  splits = std::max(splits, (int64_t)a.heads / (waves * longest));
  for (;; ++splits) {
    // q and k share the runs of heads
    const int chunks = (int)splits * waves;
    a.chunks0 = (int)(((int64_t)chunks * a.heads0 + a.heads / 2) / a.heads);
    if (heads1 > 0 && a.chunks0 == chunks) --a.chunks0;
    if (a.heads0 > 0 && a.chunks0 == 0) a.chunks0 = 1;
    a.step[0] = run(a.heads0, a.chunks0);
    a.step[1] = run(heads1, chunks - a.chunks0);
    if (a.step[0] <= longest && a.step[1] <= longest) break;
  }
  const dim3 grid((uint32_t)groups, (uint32_t)splits);
  return is_bf16 ? launch_rope_type<bf16>(a, norm, rotate, whole, out, grid, s) : launch_rope_type<float>(a, norm, rotate, whole, out, grid, s);
}

}  // namespace sf
