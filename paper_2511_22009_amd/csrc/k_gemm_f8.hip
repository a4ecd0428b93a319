// Products of e4m3 codes with a scale per block of 128 on the matrix cores,
//   out[m][n] = sum_b (sum_{k in b} A[m][k] B[n][k]) sa[m][b] sb[n / 128][b] + bias[n],
// and of gated projections act(gate) up, both such products of the same rows.
//
// A block's products are summed by two v_mfma_f32_32x32x64_f8f6f4 from zero, then one fma per output
// multiplies by sa sb (rounded once) and adds to the sum over blocks, in fp32. The weights are the first
// operand, so a lane holds sixteen columns of ONE row: one scale per lane and block of rows, and the
// scale of the weights' block is the same for the whole wavefront.
//
// That instruction adds eight products of adjacent k to each other first, and cuts each off below 2^-13 of the
// largest one's power of two (measured with pairs of products 2^-2 to 2^-17 apart: 2^-13 is kept, 2^-14
// lost, 15/8 2^-11 becomes 7/4 2^-11; products eight apart are added in fp32): 1.5e-5 of the result on codes of
// a bell, a hundredth of what rounding it to bf16 costs. Outputs in fp32, and the fp32 scales of outputs that
// are codes, are for what comes after to see more than that: the operands' codes are converted to fp16, which holds
// every one, and multiplied by v_mfma_f32_32x32x16_f16 at half the rate (1e-8 on the same codes).
#include "sf_f8_device.h"
#include "sf_ops_rules.h"

namespace sf {

// Workgroup -> tile: each of the eight XCDs (workgroup b goes to XCD b % 8) takes a contiguous
// range of tiles, in groups of eight tile rows with M fastest, so that the rows and columns
// that a group touches are read from one L2.
__device__ __forceinline__ void f8_tile(int nbm, int nbn, int& mt, int& nt) {
  const int T = nbm * nbn, b = blockIdx.x;
  const int xcd = b % 8, local = b / 8, base = T / 8, rem = T % 8;
  const int logical = xcd * base + min(xcd, rem) + local;
  const int per_group = 8 * nbn;
  const int group = logical / per_group;
  const int first_m = group * 8, gsize = min(8, nbm - first_m);
  const int in = logical - group * per_group;
  mt = first_m + in % gsize;
  nt = in / gsize;
}

__device__ __forceinline__ void buffer_load4_lds(__amdgpu_buffer_rsrc_t r, char* lds, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 4, off, 0, 0, 0);
}
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
// Eight codes in two words as fp16.
__device__ __forceinline__ f16x8 f16_of(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// c plus the products of 64 k (32 in each half of the wavefront).
template <bool EXACT>
__device__ __forceinline__ f32x16 mfma_f8(const i32x8& n, const i32x8& m, f32x16 c) {
  if constexpr (EXACT) {
#pragma unroll
    for (int w = 0; w < 8; w += 2) c = __builtin_amdgcn_mfma_f32_32x32x16_f16(f16_of(n[w], n[w + 1]), f16_of(m[w], m[w + 1]), c, 0, 0, 0);
    return c;
  } else {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(n, m, c, 0, 0, 0, 0, 0, 0);
  }
}
// Of 16 x 16 outputs: the products of 128 k, 32 in each quarter.
template <bool EXACT>
__device__ __forceinline__ f32x4 mfma16_f8(const i32x8& n, const i32x8& m) {
  f32x4 c = {};
  if constexpr (EXACT) {
#pragma unroll
    for (int w = 0; w < 8; w += 2) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(f16_of(n[w], n[w + 1]), f16_of(m[w], m[w + 1]), c, 0, 0, 0);
    return c;
  } else {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(n, m, c, 0, 0, 0, 0, 0, 0);
  }
}

template <F8Act ACT>
__device__ __forceinline__ float act_f8(float g) {
  if constexpr (ACT == F8_SILU) return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
  else if constexpr (ACT == F8_GELU) return gelu_tanh(g);
  else return g;
}

// Slices of one block of 128 columns go global -> LDS directly into a ring of STAGES buffers (rows of eight
// 16-byte chunks, swizzled by dma_swz; the rows' scales behind them). A wavefront owns TM x TN blocks of
// 32 x 32; it holds its rows' codes of a slice, takes the weights' a block of 32 columns at a time, and
// meets the others once it has read the last of them, so that the stage can be filled again under the
// MFMAs of that last block. Gated: the first half of a wavefront's TN blocks are the gate's columns,
// the other half the same columns of up.
//
// Codes past K: whole chunks read as zeros (an offset past the resource); in a chunk that K ends in, the
// bytes past K of both operands are cleared in LDS before the last slice is read.
template <int BM, int BN, int WM, int WN, int STAGES, int MINW, F8Out OUT, F8Act ACT>
__global__ __launch_bounds__(WM * WN * 64, MINW) void gemm_f8_kernel(GemmF8Args a) {
  constexpr bool GATED = ACT != F8_NONE, EXACT = OUT != F8_BF16;
  constexpr int NT = WM * WN * 64, BK = 128, CPR = 8;
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  static_assert(TM * WM * 32 == BM && TN * WN * 32 == BN, "wave grid must tile the block");
  constexpr int ATOT = BM * CPR, BTOT = BN * CPR;
  static_assert(ATOT % NT == 0 && BTOT % NT == 0, "whole rounds of chunks per slice");
  constexpr int ACH = ATOT / NT, BCH = BTOT / NT, LPT = ACH + BCH + 1;
  static_assert(STAGES >= 2 && STAGES <= 4, "two to four stages");
  constexpr int SCALES = (ATOT + BTOT) * 16, SROWS = (BM + 63) / 64;
  constexpr int SLICE = SCALES + SROWS * 256;
  static_assert(SROWS <= WM * WN, "a wavefront per 64 scales");
  static_assert(STAGES * SLICE <= 160 * 1024, "stages do not fit in LDS");
  // output columns of the tile and of a wavefront; those of a wavefront lie in one block of weights' rows
  constexpr int ON = GATED ? BN / 2 : BN, WON = ON / WN;
  static_assert(WON <= kF8Block && kF8Block % WON == 0, "a wavefront's columns share a scale");
  __shared__ __attribute__((aligned(16))) char st0[SLICE];
  __shared__ __attribute__((aligned(16))) char st1[SLICE];
  __shared__ __attribute__((aligned(16))) char st2[STAGES > 2 ? SLICE : 16];
  __shared__ __attribute__((aligned(16))) char st3[STAGES > 3 ? SLICE : 16];
  auto stage = [&](auto s) -> char* {
    constexpr int S = decltype(s)::value % STAGES;
    if constexpr (S == 0) return st0;
    else if constexpr (S == 1) return st1;
    else if constexpr (S == 2) return st2;
    else return st3;
  };
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int l32 = lane & 31, g = lane >> 5;
  int mt, nt;
  const int nbm = (a.M + BM - 1) / BM, nbn = (a.N + ON - 1) / ON;
  f8_tile(nbm, nbn, mt, nt);
  const int m0 = mt * BM, n0 = nt * ON;
  const int nk = (a.K + BK - 1) / BK;

  // LDS row r of the weights' part holds, gated, column r / (2 WON) * WON + r % WON of the tile, of the gate where r / WON
  // is even, else of up: a wavefront's run of TN / 2 blocks of the gate is followed by the same run of up. A load of a
  // wavefront takes eight rows, R apart from round to round, so which of the two it reads goes by the
  // round, or by the wavefront where a round holds both.
  constexpr int R = NT / CPR;
  constexpr bool BY_WAVE = GATED && R % (2 * WON) == 0;
  static_assert(R % 16 == 0, "one swizzle for a lane's rows of every round");
  static_assert(!GATED || BY_WAVE || WON % R == 0, "a round holds rows of one, or whole runs of both");
  auto round_up = [](int i) constexpr { return GATED && !BY_WAVE && i * R / WON % 2 == 1; };
  auto round_column = [](int i) constexpr { return !GATED ? i * R : BY_WAVE ? i * R / 2 : i * R / (2 * WON) * WON + i * R % WON; };
  const bool wave_up = BY_WAVE && wave * 8 / WON % 2 == 1;
  const int wave_column = BY_WAVE ? wave * 8 / (2 * WON) * WON + wave * 8 % WON : wave * 8;
  const int kc = ((lane % CPR) ^ dma_swz<CPR>(wave * 8 + lane / CPR)) * 16;
  const int a_off = (wave * 8 + lane / CPR) * a.a.ld + kc;
  const int b_ld = wave_up ? a.up.ld : a.b.ld;
  const int b_off = (wave_column + lane / CPR) * b_ld + kc;
  const int u_off = GATED ? (wave_column + lane / CPR) * a.up.ld + kc : 0;
  // resources from the tile's first row to the end of the chunk that K ends in of its last: rows past it read as zeros
  const int kend = (a.K + 15) & ~15, o_rows = min(a.N - n0, ON) - 1;
  const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(a.a.q + (int64_t)m0 * a.a.ld, (uint32_t)((min(a.M - m0, BM) - 1) * a.a.ld + kend));
  const __amdgpu_buffer_rsrc_t rb = buffer_rsrc((wave_up ? a.up.q : a.b.q) + (int64_t)n0 * b_ld, (uint32_t)(o_rows * b_ld + kend));
  const __amdgpu_buffer_rsrc_t ru = GATED && !BY_WAVE ? buffer_rsrc(a.up.q + (int64_t)n0 * a.up.ld, (uint32_t)(o_rows * a.up.ld + kend)) : rb;
  const float* sa_at = a.a.scale + (int64_t)m0 * a.a.s_row;  // of the next slice to be fetched
  const uint32_t s_bytes = (uint32_t)(min(a.M - m0, BM) - 1) * (uint32_t)a.a.s_row * 4 + 4;
  const int s_wave = wave % SROWS;
  const int s_off = m0 + s_wave * 64 + lane < a.M && s_wave * 64 + lane < BM ? (s_wave * 64 + lane) * (int)a.a.s_row * 4 : kOffOOB;
  // Loads number n of slice kt; n runs from 0 to LPT. An offset past K stays past every resource
  // with the rounds' rows added (kOffOOB and those are below 2^31 each).
  int a_now, b_now, u_now;
  auto issue = [&](char* sb, int kt, int from, int to) __attribute__((always_inline)) {
    if (from == 0) {
      const bool in = kt * BK + kc < a.K;
      a_now = in ? a_off + kt * BK : kOffOOB;
      b_now = in ? b_off + kt * BK : kOffOOB;
      if constexpr (GATED && !BY_WAVE) u_now = in ? u_off + kt * BK : kOffOOB;
    }
#pragma unroll
    for (int n = from; n < to; ++n) {
      if (n < ACH) {
        buffer_load16_lds(ra, sb + (n * NT + wave * 64) * 16, (int)((uint32_t)a_now + (uint32_t)(n * R * a.a.ld)));
      } else if (n < ACH + BCH) {
        const int i = n - ACH;
        const bool up = round_up(i);
        buffer_load16_lds(up ? ru : rb, sb + (ATOT + i * NT + wave * 64) * 16,
                          (int)((uint32_t)(up ? u_now : b_now) + (uint32_t)(round_column(i) * (up ? a.up.ld : b_ld))));
      } else {
        buffer_load4_lds(buffer_rsrc(sa_at, kt < nk ? s_bytes : 0u), sb + SCALES + s_wave * 256, s_off);
        sa_at += kt + 1 < nk ? a.a.s_block : 0;
      }
    }
  };
  // clears the bytes past K in the last slice
  auto clear_tail = [&](char* sb) {
    const int c = (a.K % BK) / 16;
    for (int r = tid; r < BM + BN; r += NT) {
      char* p = sb + (r * CPR + (c ^ dma_swz<CPR>(r))) * 16;
      i32x4 v = *(i32x4*)p;
      const int left = a.K % 16;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int n = left - 4 * w;
        if (n < 4) v[w] = n > 0 ? (int)((uint32_t)v[w] & ((1u << (8 * n)) - 1u)) : 0;
      }
      *(i32x4*)p = v;
    }
    __syncthreads();
  };
  static_assert(BM % 16 == 0, "the weights' rows start at a multiple of 16, as their swizzle has it");

  // scales of the wavefront's block of weights, lane l those of slices l, 64 + l, ...
  const int sb_row = min(n0 + wn * WON, a.N - 1) / kF8Block;
  auto weights_scale = [&](const F8Codes& w, int kt) -> float {
    return w.scale[(int64_t)sb_row * w.s_row + (int64_t)min(kt + lane, nk - 1) * w.s_block];
  };
  float sb_v = weights_scale(a.b, 0), su_v = GATED ? weights_scale(a.up, 0) : 0.0f;

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  const int sw = dma_swz<CPR>(l32);  // row blocks are 32 apart: every row of a lane shares it
  // chunk g + c of a lane's first row (c even, so that g + c is g ^ c); the other chunks and blocks are
  // an exclusive or and a constant away, formed where they are used: kept, they cost 16 registers
  const int a_at = ((wm * TM * 32 + l32) * CPR + (g ^ sw)) * 16;
  const int b_at = (ATOT + (wn * TN * 32 + l32) * CPR + (g ^ sw)) * 16;
  // Blocks of a slice in the order p = j TM + i. The two MFMAs of block p + 1 are issued around the fmas of
  // block p, which are VALU work in the matrix core's shadow; block NP - 1's wait for the next slice.
  constexpr int NP = TM * TN;
  i32x8 af[TM][2], bf[2][2];
  float s_gate[TM], s_up[TM], pending = 0.0f;
  f32x16 d[2] = {};
  auto frag = [&](const char* cur, int at, int s) __attribute__((always_inline)) -> i32x8 {
    const i32x4 lo = *(const i32x4*)(cur + (at ^ (64 * s)));
    const i32x4 hi = *(const i32x4*)(cur + (at ^ (64 * s + 32)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto load_a = [&](const char* cur, int i) __attribute__((always_inline)) {
    int at = a_at;
    asm volatile("" : "+v"(at));
    af[i][0] = frag(cur + i * 32 * CPR * 16, at, 0);
    af[i][1] = frag(cur + i * 32 * CPR * 16, at, 1);
  };
  auto load_b = [&](const char* cur, int j) __attribute__((always_inline)) {
    int at = b_at;
    asm volatile("" : "+v"(at));
    bf[j & 1][0] = frag(cur + (j % TN) * 32 * CPR * 16, at, 0);
    bf[j & 1][1] = frag(cur + (j % TN) * 32 * CPR * 16, at, 1);
  };
  auto load_s = [&](const char* cur, float (&s)[TM]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) s[i] = *(const float*)(cur + SCALES + ((wm * TM + i) * 32 + l32) * 4);
  };
  auto fmas = [&](int p, int half, float s) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 8 * half; r < 8 * half + 8; ++r) acc[p % TM][p / TM][r] = __builtin_fmaf(d[p & 1][r], s, acc[p % TM][p / TM][r]);
    // computed here: moved behind later MFMAs they would keep those's results alive as well
    asm volatile("" : "+v"(acc[p % TM][p / TM]));
  };
  const f32x16 zero = {};
  static_assert(TN % 2 == 0 && NP % 2 == 0, "the next slice starts with the buffers that this one started with");
  float sa[TM], sa_next[TM];
  auto step = [&](auto st, int kt) __attribute__((always_inline)) {
    constexpr int S = decltype(st)::value;
    const char* const cur = stage(std::integral_constant<int, S>{});
    const char* const next = stage(std::integral_constant<int, S + 1>{});
    if ((kt & 63) == 0 && kt > 0) {
      sb_v = weights_scale(a.b, kt);
      if constexpr (GATED) su_v = weights_scale(a.up, kt);
      __builtin_amdgcn_s_waitcnt(0);
    }
    const float sb = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sb_v), kt & 63));
    const float su = GATED ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(su_v), kt & 63)) : 0.0f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      s_gate[i] = sa[i] * sb;
      s_up[i] = sa[i] * su;
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int i = p % TM, j = p / TM;
      if (p == NP - TM) {
        // every read of this stage has arrived: the MFMAs below take the last of them
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0<(STAGES - 2) * LPT>());
        bare_barrier();
        if (a.K % 16 != 0 && kt + 2 == nk) clear_tail(stage(std::integral_constant<int, S + 1>{}));
        load_s(next, sa_next);
      }
      // reads into registers that the MFMAs before have taken
      if (p == 0 && TM > 1) load_a(cur, TM - 1);
      if (i == 0) load_b(j + 1 < TN ? cur : next, j + 1);
      if (j == TN - 1 && i > 0) load_a(next, i - 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        d[p & 1] = mfma_f8<EXACT>(bf[j & 1][half], af[i][half], half ? d[p & 1] : zero);
        __builtin_amdgcn_sched_barrier(0);
        fmas((p + NP - 1) % NP, half, pending);
        // the stage's refill, spread over the last column's MFMAs
        if (j == TN - 1)
          issue(stage(std::integral_constant<int, S>{}), kt + STAGES, (2 * i + half) * LPT / (2 * TM), (2 * i + half + 1) * LPT / (2 * TM));
        __builtin_amdgcn_sched_barrier(0);
      }
      pending = GATED && j >= TN / 2 ? s_up[i] : s_gate[i];
    }
    if (TM == 1) load_a(next, 0);
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] = sa_next[i];
  };
  auto round = [&](int kt) __attribute__((always_inline)) {
    step(std::integral_constant<int, 0>{}, kt);
    step(std::integral_constant<int, 1>{}, kt + 1);
    if constexpr (STAGES > 2) step(std::integral_constant<int, 2>{}, kt + 2);
    if constexpr (STAGES > 3) step(std::integral_constant<int, 3>{}, kt + 3);
  };
  issue(stage(std::integral_constant<int, 0>{}), 0, 0, LPT);
  issue(stage(std::integral_constant<int, 1>{}), 1, 0, LPT);
  if constexpr (STAGES > 2) issue(stage(std::integral_constant<int, 2>{}), 2, 0, LPT);
  if constexpr (STAGES > 3) issue(stage(std::integral_constant<int, 3>{}), 3, 0, LPT);
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0<(STAGES - 1) * LPT>());
  bare_barrier();
  if (a.K % 16 != 0 && nk == 1) clear_tail(st0);
#pragma unroll
  for (int i = 0; i < TM - 1 || i == 0; ++i) load_a(st0, i);
  load_b(st0, 0);
  load_s(st0, sa);
  int kt = 0;
  for (; kt + STAGES <= nk; kt += STAGES) round(kt);
  if (kt < nk) step(std::integral_constant<int, 0>{}, kt);
  if constexpr (STAGES > 2)
    if (kt + 1 < nk) step(std::integral_constant<int, 1>{}, kt + 1);
  if constexpr (STAGES > 3)
    if (kt + 2 < nk) step(std::integral_constant<int, 2>{}, kt + 2);
  fmas(NP - 1, 0, pending);
  fmas(NP - 1, 1, pending);
  __builtin_amdgcn_s_waitcnt(0);  // the loads past K land before the LDS is used again or given up

  // Lane (l32, g) holds row l32 of each block and the columns 8 q + 4 g + 0..3. Values and bias first;
  // a gated wavefront has its outputs in the gate's blocks then.
  constexpr int TO = GATED ? TN / 2 : TN;
#pragma unroll
  for (int j = 0; j < TO; ++j) {
    const int nb = n0 + wn * WON + j * 32;
    const int n = min(nb + l32, a.N - 1);
    const float bias_v = a.bias ? a.bias[n] : 0.0f, up_v = GATED && a.up_bias ? a.up_bias[n] : 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int from = 8 * (r >> 2) + 4 * g + (r & 3);
      const float b = __shfl(bias_v, from);
      const float u = GATED ? __shfl(up_v, from) : 0.0f;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const float v = acc[i][j][r] + b;
        if constexpr (GATED)
          acc[i][j][r] = act_f8<ACT>(v) * (acc[i][j + TO][r] + u);
        else
          acc[i][j][r] = v;
      }
    }
  }
  // Every wavefront passes its part of the tile through LDS of its own, 32 rows at a time, so that
  // stores leave in whole rows of the part
  typedef uint32_t out16 __attribute__((ext_vector_type(4), aligned(1)));
  constexpr int ES = OUT == F8_F32 ? 4 : OUT == F8_BF16 ? 2 : 1;
  constexpr int E = 16 / ES, JG = OUT == F8_F32 ? 1 : TO;
  constexpr int PITCH = JG * 32 * ES + 16, CPW = JG * 32 / E, HALF = (WM * WN + 1) / 2;
  static_assert(HALF * 32 * PITCH <= SCALES, "the parts of half the wavefronts fit a stage");
  char* const part = (wave < HALF ? st0 + wave * 32 * PITCH : st1 + (wave - HALF) * 32 * PITCH);
  __syncthreads();
  BlockF8 bq[OUT == F8_CODES ? TM : 1];
  if constexpr (OUT == F8_CODES) {
    // the scale of a row's 128 columns: every wavefront's largest, joined in LDS
    static_assert(ON == kF8Block, "a tile holds whole blocks of outputs");
    constexpr int CP = WN + 1;
    static_assert(BM * CP * 4 <= SROWS * 256 * CP, "tops");
    uint32_t* const tops = (uint32_t*)(STAGES > 2 ? st2 : st1 + HALF * 32 * PITCH);
    static_assert(STAGES > 2 || HALF * 32 * PITCH + BM * CP * 4 <= SLICE, "tops fit behind the parts");
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      uint32_t t = 0;
#pragma unroll
      for (int j = 0; j < TO; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int n = n0 + wn * WON + j * 32 + 8 * (r >> 2) + 4 * g + (r & 3);
          if (n < a.N) t = max(t, abs_bits(acc[i][j][r]));
        }
      t = xor_max<32>(t);
      if (g == 0) tops[((wm * TM + i) * 32 + l32) * CP + wn] = t;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const uint32_t* const p = tops + ((wm * TM + i) * 32 + l32) * CP;
      uint32_t t = p[0];
#pragma unroll
      for (int w = 1; w < WN; ++w) t = max(t, p[w]);
      bq[i] = block_f8(t);
      const int m = m0 + (wm * TM + i) * 32 + l32;
      if (wn == 0 && g == 0 && m < a.M) a.out_scale[(int64_t)m * a.os_row + (int64_t)(n0 / kF8Block) * a.os_block] = bq[i].scale;
    }
  }
#pragma unroll
  for (int j0 = 0; j0 < TO; j0 += JG) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int j = 0; j < JG; ++j) {
        uint32_t c[4];
        if constexpr (OUT == F8_CODES) {
          float v[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) v[r] = acc[i][j0 + j][r];
          codes_f8(v, bq[i], c);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          char* const p = part + l32 * PITCH + (j * 32 + q * 8 + g * 4) * ES;
          const f32x16& v = acc[i][j0 + j];
          if constexpr (OUT == F8_F32)
            *(f32x4*)p = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
          else if constexpr (OUT == F8_BF16)
            *(uint2*)p = uint2{pack_bf16(v[4 * q], v[4 * q + 1]), pack_bf16(v[4 * q + 2], v[4 * q + 3])};
          else
            *(uint32_t*)p = c[q];
        }
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < (32 * CPW + 63) / 64; ++u) {
        const int c = u * 64 + lane, r = c / CPW, cc = c - r * CPW;
        if (32 * CPW % 64 != 0 && r >= 32) continue;
        const u32x4 o = *(const u32x4*)(part + r * PITCH + cc * 16);
        const int m = m0 + (wm * TM + i) * 32 + r, n = n0 + wn * WON + j0 * 32 + cc * E;
        char* const to = (char*)a.out + ((int64_t)m * a.ldo + n) * ES;
        if (m < a.M && n + E <= a.N) {
          __builtin_nontemporal_store(o, (out16*)to);
        } else if (m < a.M) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (n + e < a.N) {
              if constexpr (OUT == F8_F32)
                ((float*)to)[e] = __uint_as_float(o[e]);
              else if constexpr (OUT == F8_BF16)
                ((uint16_t*)to)[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
              else
                ((uint8_t*)to)[e] = (uint8_t)(o[e >> 2] >> (8 * (e & 3)));
            }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Few rows, up to 16 MT: the weights are read once and bound it, so a workgroup takes only sixteen columns (gated:
// of both projections), its W wavefronts share the blocks of K among them, each straight from memory to
// v_mfma_f32_16x16x128_f8f6f4, and the sums are joined in LDS in a fixed order.
template <int MT, int W, F8Out OUT, F8Act ACT>
__global__ __launch_bounds__(W * 64) void few_f8_kernel(GemmF8Args a) {
  constexpr bool GATED = ACT != F8_NONE;
  constexpr int P = GATED ? 2 : 1, AHEAD = MT == 1 ? 4 : 2;
  __shared__ __attribute__((aligned(16))) f32x4 sums[W][P][MT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const int nk = (a.K + kF8Block - 1) / kF8Block;
  // the resources hold the tile's rows to the end of the chunk that K ends in; rows past the last are it
  const int kend = (a.K + 15) & ~15;
  const int rows = min(a.N - n0, 16);
  const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(a.a.q, (uint32_t)((a.M - 1) * a.a.ld + kend));
  const __amdgpu_buffer_rsrc_t rb = buffer_rsrc(a.b.q + (int64_t)n0 * a.b.ld, (uint32_t)((rows - 1) * a.b.ld + kend));
  const __amdgpu_buffer_rsrc_t ru = GATED ? buffer_rsrc(a.up.q + (int64_t)n0 * a.up.ld, (uint32_t)((rows - 1) * a.up.ld + kend)) : rb;
  const int b_off = min(l16, rows - 1) * a.b.ld, u_off = GATED ? min(l16, rows - 1) * a.up.ld : 0;
  int a_off[MT];
  const float* sa[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = min(t * 16 + l16, a.M - 1);
    a_off[t] = m * a.a.ld;
    sa[t] = a.a.scale + (int64_t)m * a.a.s_row;
  }
  const float* const sb = a.b.scale + (int64_t)(n0 / kF8Block) * a.b.s_row;
  const float* const su = GATED ? a.up.scale + (int64_t)(n0 / kF8Block) * a.up.s_row : nullptr;
  // 32 bytes of a row from column k on; what lies past K is 0
  auto load = [&](__amdgpu_buffer_rsrc_t r, int off, int k) __attribute__((always_inline)) -> i32x8 {
    const i32x4 lo = __builtin_bit_cast(i32x4, buffer_load16(r, k < a.K ? off + k : kOffOOB));
    const i32x4 hi = __builtin_bit_cast(i32x4, buffer_load16(r, k + 16 < a.K ? off + k + 16 : kOffOOB));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto clear = [&](i32x8& v, int k) __attribute__((always_inline)) {
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const int n = a.K - k - 4 * w;
      if (n < 4) v[w] = n > 0 ? (int)((uint32_t)v[w] & ((1u << (8 * n)) - 1u)) : 0;
    }
  };
  f32x4 acc[P][MT] = {};
  for (int kb0 = wave; kb0 < nk; kb0 += AHEAD * W) {
    i32x8 b[AHEAD][P], x[AHEAD][MT];
    float s[AHEAD][MT], w[AHEAD][P];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int kb = kb0 + u * W, k = kb * kF8Block + 32 * g, sk = min(kb, nk - 1);
      b[u][0] = load(rb, b_off, k);
      if constexpr (GATED) b[u][P - 1] = load(ru, u_off, k);
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        x[u][t] = load(ra, a_off[t], k);
        s[u][t] = sa[t][(int64_t)sk * a.a.s_block];
      }
      w[u][0] = sb[(int64_t)sk * a.b.s_block];
      if constexpr (GATED) w[u][P - 1] = su[(int64_t)sk * a.up.s_block];
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int kb = kb0 + u * W, k = kb * kF8Block + 32 * g;
      if (kb >= nk) break;
      if (kb + 1 == nk && a.K % 16 != 0) {
#pragma unroll
        for (int p = 0; p < P; ++p) clear(b[u][p], k);
#pragma unroll
        for (int t = 0; t < MT; ++t) clear(x[u][t], k);
      }
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const f32x4 d = mfma16_f8<OUT != F8_BF16>(b[u][p], x[u][t]);
          const float f = s[u][t] * w[u][p];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[p][t][e] = __builtin_fmaf(d[e], f, acc[p][t][e]);
        }
    }
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[wave][p][t][lane] = acc[p][t];
  __syncthreads();
  for (int e = threadIdx.x; e < MT * 256; e += W * 64) {
    const int t = e >> 8, m = (e >> 4) & 15, c = e & 15, n = n0 + c;
    float v[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      v[p] = 0.0f;
#pragma unroll
      for (int k = 0; k < W; ++k) v[p] += ((const float*)&sums[k][p][t][(c >> 2) * 16 + m])[c & 3];
    }
    if (t * 16 + m >= a.M || n >= a.N) continue;
    v[0] += a.bias ? a.bias[n] : 0.0f;
    if constexpr (GATED) v[0] = act_f8<ACT>(v[0]) * (v[P - 1] + (a.up_bias ? a.up_bias[n] : 0.0f));
    const int64_t at = (int64_t)(t * 16 + m) * a.ldo + n;
    if constexpr (OUT == F8_F32)
      ((float*)a.out)[at] = v[0];
    else
      ((bf16*)a.out)[at] = (bf16)v[0];
  }
}

template <F8Out OUT, F8Act ACT>
static void launch_few(const GemmF8Args& a, hipStream_t s) {
  const dim3 grid((uint32_t)((a.N + 15) / 16));
  if (a.M <= 16)
    launch(few_f8_kernel<1, 8, OUT, ACT>, grid, dim3(512), 0, s, a);
  else if (a.M <= 32)
    launch(few_f8_kernel<2, 8, OUT, ACT>, grid, dim3(512), 0, s, a);
  else
    launch(few_f8_kernel<4, 8, OUT, ACT>, grid, dim3(512), 0, s, a);
}

// Tiles: BM x BN, wave grid, LDS stages, wavefronts per SIMD.
#define SF_F8_TILES(X)                    \
  X(kF8Deep64, 64, 64, 2, 1, 4, 2)        \
  X(kF8Tile128, 128, 128, 2, 2, 2, 2)     \
  X(kF8Tile128x256, 128, 256, 2, 4, 2, 2) \
  X(kF8Tile256x256, 256, 256, 4, 2, 2, 2)

template <F8Out OUT, F8Act ACT>
static hipError_t launch_f8(const GemmF8Args& a, hipStream_t s) {
  constexpr bool kGated = ACT != F8_NONE;
  F8Tile tile = choose_gemm_f8_tile(a.M, (long)a.N * (kGated ? 2 : 1), a.K, OUT == F8_CODES, OUT == F8_F32);
  switch (tile) {
    case kF8Few:
      if constexpr (OUT != F8_CODES) launch_few<OUT, ACT>(a, s);
      break;
#define SF_F8_CASE(id, bm, bn, wm, wn, st, mw)                                                                \
  case id: {                                                                                                  \
    constexpr int on = kGated ? bn / 2 : bn;                                                                  \
    const int64_t tiles = (((int64_t)a.M + bm - 1) / bm) * (((int64_t)a.N + on - 1) / on);                    \
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;                                                      \
    if constexpr ((OUT != F8_CODES || on == kF8Block) && (OUT == F8_BF16 || bm < 256)) /* never chosen otherwise */                             \
      launch(gemm_f8_kernel<bm, bn, wm, wn, st, mw, OUT, ACT>, dim3((uint32_t)tiles), dim3(wm * wn * 64), 0, s, a); \
    break;                                                                                                    \
  }
    SF_F8_TILES(SF_F8_CASE)
#undef SF_F8_CASE
  }
  return hipGetLastError();
}

hipError_t launch_gemm_f8(F8Out kind, F8Act act, const GemmF8Args& a, hipStream_t s) {
  switch (act) {
    case F8_NONE: return kind == F8_BF16 ? launch_f8<F8_BF16, F8_NONE>(a, s) : launch_f8<F8_F32, F8_NONE>(a, s);
    case F8_SILU:
      return kind == F8_BF16  ? launch_f8<F8_BF16, F8_SILU>(a, s)
             : kind == F8_F32 ? launch_f8<F8_F32, F8_SILU>(a, s)
                              : launch_f8<F8_CODES, F8_SILU>(a, s);
    case F8_GELU:
      return kind == F8_BF16  ? launch_f8<F8_BF16, F8_GELU>(a, s)
             : kind == F8_F32 ? launch_f8<F8_F32, F8_GELU>(a, s)
                              : launch_f8<F8_CODES, F8_GELU>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace sf
