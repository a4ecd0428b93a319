// Products of e4m3 codes with a scale per block of 128 on the matrix cores,
//   out[m][n] = sum_b (sum_{k in b} A[m][k] B[n][k]) sa[m][b] sb[n / 128][b] + bias[n],
// and of gated projections act(gate) up, both such products of the same rows.
//
// A block's products are summed by one v_mfma_f32_16x16x128_f8f6f4 from zero, then one fma per output
// multiplies by sa sb (rounded once) and adds to the sum over blocks, in fp32. The weights are the first
// operand, so a lane holds four adjacent columns of ONE row: one scale per lane and group of rows, and the
// scale of the weights' block is the same for the whole wavefront.
//
// That instruction adds eight products of adjacent k to each other first, and cuts each off, towards zero, below 2^-13 of
// the largest power of two that two operands of one have together (measured with pairs of products 2^-2 to 2^-17 apart: 2^-13 is
// kept, 2^-14 lost, 15/8 2^-11 becomes 7/4 2^-11; that rule gives the sums of 2048 columns of a bell's codes exactly up to
// K = 16 and to 3e-4 of what is cut off at 128; products eight apart are added in fp32): 1.5e-5 of the result on codes of
// a bell, a hundredth of what rounding it to bf16 costs. Outputs in fp32, and the fp32 scales of outputs that
// are codes, are for what comes after to see more than that: the operands' codes are converted to fp16, which holds
// every one, and multiplied by v_mfma_f32_16x16x32_f16 at half the rate (1e-8 on the same codes).
//
// What bounds it. Large products in bf16: the matrix cores at the clock that their power leaves, 8192^3 482 to 503 us by
// the codes' magnitudes, 2280 to 2190 TFLOP/s (a library's product with one scale per operand, without the fmas, 409). Outputs that are exact: the vector
// unit, which converts 128 pairs of codes and runs 64 fmas of a wavefront's 64 x 64 outputs a slice beside 1024 cycles of
// matrix work: gated 16384 x 2 x 4608 x 1152 to codes 333 to 359 us, to fp32 335, to bf16 176. Single rounds of tiles:
// the first slices and the outputs of all at once (gated 4096 x 2 x 2048 x 768 17 us). Few tiles: a turn's latencies and the
// L2's rate to one CU (517 x 1001 x 4321 fp32 15). Few rows: the weights' bytes and one chain of latencies (8 x 2 x 2048 x 768
// 4.7, the host's part of a call among them).
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
// Words 2 w and 2 w + 1 of 32 codes as fp16.
__device__ __forceinline__ f16x8 f16_of(const i32x8& v, int w) {
  const uint32_t lo = v[2 * w], hi = v[2 * w + 1];
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// 16 x 16 sums over 128 k (of which a quarter of the wavefront holds 32): at once, or over 32 k (eight a quarter) more.
__device__ __forceinline__ f32x4 mfma_f8(const i32x8& n, const i32x8& m) {
  const f32x4 zero = {};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(n, m, zero, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f16(const f16x8& n, const f16x8& m, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(n, m, c, 0, 0, 0);
}
template <bool EXACT>
__device__ __forceinline__ f32x4 sum_of_block(const i32x8& n, const i32x8& m) {
  if constexpr (EXACT) {
    f32x4 c = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) c = mfma_f16(f16_of(n, w), f16_of(m, w), c);
    return c;
  } else {
    return mfma_f8(n, m);
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
// 32 x 32 outputs; it holds its rows' codes of a slice, takes the weights' a block of 32 columns at a time, and
// meets the others once it has read the last of them, so that the stage can be filled again under the
// MFMAs of that last block. Gated: the first half of a wavefront's TN blocks are the gate's columns,
// the other half the same columns of up.
//
// Codes past K: whole chunks read as zeros (an offset past the resource); in a chunk that K ends in, the
// bytes past K of both operands are cleared in LDS before the last slice is read.
//
// WK > 1, for few tiles: as many groups of WM WN wavefronts share a tile, group g takes slices g, g + WK, ... (a stage holds one
// of each), and the first adds the others' sums to its own, in order, through LDS.
template <int BM, int BN, int WM, int WN, int WK, int STAGES, int MINW, F8Out OUT, F8Act ACT>
__global__ __launch_bounds__(WM * WN * WK * 64, MINW) void gemm_f8_kernel(GemmF8Args a) {
  constexpr bool GATED = ACT != F8_NONE, EXACT = OUT != F8_BF16;
  constexpr int NT = WM * WN * 64, BK = 128, CPR = 8;  // NT: of a group
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  static_assert(TM * WM * 32 == BM && TN * WN * 32 == BN, "wave grid must tile the block");
  constexpr int ATOT = BM * CPR, BTOT = BN * CPR;
  static_assert(ATOT % NT == 0 && BTOT % NT == 0, "whole rounds of chunks per slice");
  static_assert(STAGES >= 2 && STAGES <= 4, "two to four stages");
  // Two workgroups of 64 x 256 fill a CU's LDS with codes alone: each lane fetches its rows' scales itself then.
  constexpr bool OWN_SCALES = 2 * STAGES * WK * (ATOT + BTOT) * 16 == 160 * 1024;
  constexpr int SCALES = (ATOT + BTOT) * 16, SROWS = (BM + 63) / 64;
  constexpr int SLICE = SCALES + (OWN_SCALES ? 0 : SROWS * 256);
  constexpr int ACH = ATOT / NT, BCH = BTOT / NT, LPT = ACH + BCH + (OWN_SCALES ? 0 : 1);
  static_assert(SROWS <= WM * WN, "a wavefront per 64 scales");
  static_assert(STAGES * WK * SLICE <= 160 * 1024, "stages do not fit in LDS");
  static_assert(WK == 1 || OUT != F8_CODES, "the scales of codes are joined over a tile's only group");
  static_assert(WK == 1 || !OWN_SCALES, "a lane's own scales go from slice to slice");
  // output columns of the tile and of a wavefront; those of a wavefront lie in one block of weights' rows
  constexpr int ON = GATED ? BN / 2 : BN, WON = ON / WN;
  static_assert(WON <= kF8Block && kF8Block % WON == 0, "a wavefront's columns share a scale");
  __shared__ __attribute__((aligned(16))) char st0[WK * SLICE];
  __shared__ __attribute__((aligned(16))) char st1[WK * SLICE];
  __shared__ __attribute__((aligned(16))) char st2[STAGES > 2 ? WK * SLICE : 16];
  __shared__ __attribute__((aligned(16))) char st3[STAGES > 3 ? WK * SLICE : 16];
  auto stage = [&](auto s) -> char* {
    constexpr int S = decltype(s)::value % STAGES;
    if constexpr (S == 0) return st0;
    else if constexpr (S == 1) return st1;
    else if constexpr (S == 2) return st2;
    else return st3;
  };
  const int lane = threadIdx.x & 63, all_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = all_wave / (WM * WN), wave = all_wave % (WM * WN), tid = wave * 64 + lane;  // tid: in the group
  const int wm = wave / WN, wn = wave % WN;
  const int l16 = lane & 15, g = lane >> 4;
  int mt, nt;
  const int nbm = (a.M + BM - 1) / BM, nbn = (a.N + ON - 1) / ON;
  f8_tile(nbm, nbn, mt, nt);
  const int m0 = mt * BM, n0 = nt * ON;
  const int nk = (a.K + BK - 1) / BK, turns = (nk + WK - 1) / WK;
  const int mine = group * SLICE;  // of a stage

  // LDS row r of the weights' part holds, gated, column r / (2 WON) * WON + r % WON of the tile, of the gate where r / WON
  // is even, else of up: a wavefront's run of TN / 2 blocks of the gate is followed by the same run of up. A load of a
  // wavefront takes eight rows, R apart from round to round, so which of the two it reads goes by the
  // round, or by the wavefront where a round holds both.
  constexpr int R = NT / CPR;
  constexpr bool BY_WAVE = GATED && R % (2 * WON) == 0;
  constexpr int SWZ = R % 16 == 0 ? 1 : 2;  // rounds of eight rows alternate between two swizzles, a chunk apart
  static_assert(R % 8 == 0, "a lane's rows have one swizzle or two");
  static_assert(!GATED || BY_WAVE || WON % R == 0, "a round holds rows of one, or whole runs of both");
  auto round_up = [](int i) constexpr { return GATED && !BY_WAVE && i * R / WON % 2 == 1; };
  auto round_column = [](int i) constexpr { return !GATED ? i * R : BY_WAVE ? i * R / 2 : i * R / (2 * WON) * WON + i * R % WON; };
  const bool wave_up = BY_WAVE && wave * 8 / WON % 2 == 1;
  const int wave_column = BY_WAVE ? wave * 8 / (2 * WON) * WON + wave * 8 % WON : wave * 8;
  const int kc = ((lane % CPR) ^ dma_swz<CPR>(wave * 8 + lane / CPR)) * 16;
  const int a_off = (wave * 8 + lane / CPR) * a.a.ld;
  const int b_ld = wave_up ? a.up.ld : a.b.ld;
  const int b_off = (wave_column + lane / CPR) * b_ld;
  const int u_off = GATED ? (wave_column + lane / CPR) * a.up.ld : 0;
  // resources from the tile's first row to the end of the chunk that K ends in of its last: rows past it read as zeros
  const int kend = (a.K + 15) & ~15, o_rows = min(a.N - n0, ON) - 1;
  const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(a.a.q + (int64_t)m0 * a.a.ld, (uint32_t)((min(a.M - m0, BM) - 1) * a.a.ld + kend));
  const __amdgpu_buffer_rsrc_t rb = buffer_rsrc((wave_up ? a.up.q : a.b.q) + (int64_t)n0 * b_ld, (uint32_t)(o_rows * b_ld + kend));
  const __amdgpu_buffer_rsrc_t ru = GATED && !BY_WAVE ? buffer_rsrc(a.up.q + (int64_t)n0 * a.up.ld, (uint32_t)(o_rows * a.up.ld + kend)) : rb;
  int sa_left = nk;  // OWN_SCALES: slices whose scales are still to be fetched
  const float* sa_at = a.a.scale + (int64_t)m0 * a.a.s_row + min(group, nk - 1) * a.a.s_block;  // of the next slice to be fetched
  const uint32_t s_bytes = (uint32_t)(min(a.M - m0, BM) - 1) * (uint32_t)a.a.s_row * 4 + 4;
  const int s_wave = wave % SROWS;
  const int s_off = m0 + s_wave * 64 + lane < a.M && s_wave * 64 + lane < BM ? (s_wave * 64 + lane) * (int)a.a.s_row * 4 : kOffOOB;
  // Loads number `from` to `to` of the group's slice of a turn, LPT in all. An offset past K stays past every
  // resource with the rounds' rows added (kOffOOB and those are below 2^31 each).
  int a_now[SWZ], b_now[SWZ], u_now[SWZ];
  auto issue = [&](char* sb, int turn, int from, int to) __attribute__((always_inline)) {
    const int k0 = (turn * WK + group) * BK;
    if (from == 0) {
#pragma unroll
      for (int z = 0; z < SWZ; ++z) {
        const int k = k0 + (kc ^ (16 * z));
        a_now[z] = k < a.K ? a_off + k : kOffOOB;
        b_now[z] = k < a.K ? b_off + k : kOffOOB;
        if constexpr (GATED && !BY_WAVE) u_now[z] = k < a.K ? u_off + k : kOffOOB;
      }
    }
#pragma unroll
    for (int n = from; n < to; ++n) {
      if (n < ACH) {
        buffer_load16_lds(ra, sb + mine + (n * NT + wave * 64) * 16, (int)((uint32_t)a_now[n % SWZ] + (uint32_t)(n * R * a.a.ld)));
      } else if (n < ACH + BCH) {
        const int i = n - ACH;
        const bool up = round_up(i);
        buffer_load16_lds(up ? ru : rb, sb + mine + (ATOT + i * NT + wave * 64) * 16,
                          (int)((uint32_t)(up ? u_now : b_now)[i % SWZ] + (uint32_t)(round_column(i) * (up ? a.up.ld : b_ld))));
      } else {
        buffer_load4_lds(buffer_rsrc(sa_at, k0 < a.K ? s_bytes : 0u), sb + mine + SCALES + s_wave * 256, s_off);
        sa_at += k0 + WK * BK < a.K ? WK * a.a.s_block : 0;
      }
    }
  };
  // clears the bytes past K in the last slice
  auto clear_tail = [&](char* sb) {
    const int c = (a.K % BK) / 16;
    for (int r = tid; r < BM + BN && group == (nk - 1) % WK; r += NT) {
      char* p = sb + mine + (r * CPR + (c ^ dma_swz<CPR>(r))) * 16;
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

  // scales of the wavefront's block of weights, lane l those of turns l, 64 + l, ...
  const int sb_row = min(n0 + wn * WON, a.N - 1) / kF8Block;
  auto weights_scale = [&](const F8Codes& w, int turn) -> float {
    return w.scale[(int64_t)sb_row * w.s_row + (int64_t)min((turn + lane) * WK + group, nk - 1) * w.s_block];
  };
  float sb_v = weights_scale(a.b, 0), su_v = GATED ? weights_scale(a.up, 0) : 0.0f;

  // Units of 16 rows x 32 columns: unit u = j IB + i is rows i of column block j.
  constexpr int IB = TM * 2, NU = IB * TN, PARTS = EXACT ? 4 : 1;
  f32x4 acc[IB][TN][2];
#pragma unroll
  for (int i = 0; i < IB; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j][0] = acc[i][j][1] = f32x4{};
  const int sw = dma_swz<CPR>(l16);  // groups of rows are 16 apart: every row of a lane shares it
  // chunks 2 g and 2 g + 1 of a lane's first row: the quarter's 32 codes; other groups are a constant away
  const int a_at = mine + ((wm * TM * 32 + l16) * CPR + ((2 * g) ^ sw)) * 16;
  const int b_at = mine + (ATOT + (wn * TN * 32 + l16) * CPR + ((2 * g) ^ sw)) * 16;
  // The MFMAs of unit u + 1 are issued between the fmas of unit u, which are VALU work in the matrix core's shadow; the
  // last unit's wait for the next slice. EXACT: so are the conversions to fp16, each operand's once per slice.
  i32x8 af[IB], bf[EXACT ? 1 : 2][2];
  f16x8 a16[EXACT ? IB : 1][4], b16[2][4];
  f32x4 d[2][2] = {};
  float sa[IB], sa_next[IB], s_gate[IB], s_up[IB], pending = 0.0f;
  auto frag = [&](const char* cur, int at) __attribute__((always_inline)) -> i32x8 {
    const i32x4 lo = *(const i32x4*)(cur + at), hi = *(const i32x4*)(cur + (at ^ 16));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto load_a = [&](const char* cur, int i) __attribute__((always_inline)) { af[i] = frag(cur + i * 16 * CPR * 16, a_at); };
  auto load_b = [&](const char* cur, int j) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 2; ++c) bf[EXACT ? 0 : j & 1][c] = frag(cur + (j % TN * 2 + c) * 16 * CPR * 16, b_at);
  };
  auto load_s = [&](const char* cur, float (&s)[IB]) __attribute__((always_inline)) {
    if constexpr (OWN_SCALES) {
      const __amdgpu_buffer_rsrc_t r = buffer_rsrc(sa_at, s_bytes);
#pragma unroll
      for (int i = 0; i < IB; ++i)
        s[i] = __uint_as_float(
            __builtin_amdgcn_raw_buffer_load_b32(r, (wm * TM * 32 + i * 16 + l16) * (int)a.a.s_row * 4, 0, 0));
      sa_left -= 1;
      sa_at += sa_left > 0 ? a.a.s_block : 0;
      return;
    }
#pragma unroll
    for (int i = 0; i < IB; ++i) s[i] = *(const float*)(cur + mine + SCALES + (wm * TM * 32 + i * 16 + l16) * 4);
  };
  auto fmas = [&](int u, int c, int part, float s) __attribute__((always_inline)) {
    f32x4& to = acc[u % IB][u / IB][c];
#pragma unroll
    for (int r = 4 / PARTS * part; r < 4 / PARTS * (part + 1); ++r) to[r] = __builtin_fmaf(d[u & 1][c][r], s, to[r]);
    // computed here: moved behind later MFMAs they would keep those's results alive as well
    asm volatile("" : "+v"(to));
  };
  // EXACT: what part w of unit u is the first to multiply, one part ahead of it, so that no MFMA waits for a conversion:
  // the rows' codes in the first column block, the columns' in the first rows. c: the half of it.
  auto convert = [&](int u, int w, int c) __attribute__((always_inline)) {
    const int i = u % IB, j = u / IB;
    if (i == 0) b16[c][w] = f16_of(bf[0][c], w);
    if (j == 0 && c == 0) a16[i][w] = f16_of(af[i], w);
  };
  static_assert(TN % 2 == 0 && NU % 2 == 0, "the next slice starts with the buffers that this one started with");
  auto step = [&](auto st, int turn) __attribute__((always_inline)) {
    constexpr int S = decltype(st)::value;
    const char* const cur = stage(std::integral_constant<int, S>{});
    const char* const next = stage(std::integral_constant<int, S + 1>{});
    if ((turn & 63) == 0 && turn > 0) {
      sb_v = weights_scale(a.b, turn);
      if constexpr (GATED) su_v = weights_scale(a.up, turn);
      __builtin_amdgcn_s_waitcnt(0);
    }
    const bool live = WK == 1 || turn * WK + group < nk;  // past K, codes and the rows' scales are 0
    const float sb = live ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sb_v), turn & 63)) : 0.0f;
    const float su = GATED && live ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(su_v), turn & 63)) : 0.0f;
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      s_gate[i] = sa[i] * sb;
      s_up[i] = sa[i] * su;
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int i = u % IB, j = u / IB;
      if (u == NU - IB) {
        // every read of this stage has arrived: the MFMAs below take the last of them
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0<(STAGES - 2) * LPT>());
        bare_barrier();
        if (a.K % 16 != 0 && turn + 2 == turns) clear_tail(stage(std::integral_constant<int, S + 1>{}));
        load_s(next, sa_next);
      }
      // reads into registers that the MFMAs (EXACT: the conversions) before have taken
      if (i == (EXACT ? 1 : 0)) load_b(j + 1 < TN ? cur : next, j + 1);
      if constexpr (EXACT) {
        if (u == NU - IB) {
#pragma unroll
          for (int n = 0; n < IB; ++n) load_a(next, n);
        }
      } else {
        if (u == 0) load_a(cur, IB - 1);
        if (j == TN - 1 && i > 0) load_a(next, i - 1);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int w = 0; w < PARTS; ++w)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          if constexpr (EXACT) {
            d[u & 1][c] = mfma_f16(b16[c][w], a16[i][w], w ? d[u & 1][c] : f32x4{});
          } else {
            d[u & 1][c] = mfma_f8(bf[j & 1][c], af[i]);
          }
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (EXACT) convert((u + (w + 1) / PARTS) % NU, (w + 1) % PARTS, c);
          fmas((u + NU - 1) % NU, c, w, pending);
          // the stage's refill, spread over the last column's MFMAs
          constexpr int N = PARTS * 2 * IB;
          const int n = (i * PARTS + w) * 2 + c;
          if (j == TN - 1) issue(stage(std::integral_constant<int, S>{}), turn + STAGES, n * LPT / N, (n + 1) * LPT / N);
          __builtin_amdgcn_sched_barrier(0);
        }
      pending = GATED && j >= TN / 2 ? s_up[i] : s_gate[i];
    }
#pragma unroll
    for (int i = 0; i < IB; ++i) sa[i] = sa_next[i];
  };
  auto round = [&](int turn) __attribute__((always_inline)) {
    step(std::integral_constant<int, 0>{}, turn);
    step(std::integral_constant<int, 1>{}, turn + 1);
    if constexpr (STAGES > 2) step(std::integral_constant<int, 2>{}, turn + 2);
    if constexpr (STAGES > 3) step(std::integral_constant<int, 3>{}, turn + 3);
  };
  issue(stage(std::integral_constant<int, 0>{}), 0, 0, LPT);
  issue(stage(std::integral_constant<int, 1>{}), 1, 0, LPT);
  if constexpr (STAGES > 2) issue(stage(std::integral_constant<int, 2>{}), 2, 0, LPT);
  if constexpr (STAGES > 3) issue(stage(std::integral_constant<int, 3>{}), 3, 0, LPT);
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0<(STAGES - 1) * LPT>());
  bare_barrier();
  if (a.K % 16 != 0 && turns == 1) clear_tail(st0);
#pragma unroll
  for (int i = 0; i < (EXACT ? IB : IB - 1); ++i) load_a(st0, i);
  load_b(st0, 0);
  load_s(st0, sa);
  if constexpr (EXACT) {
    convert(0, 0, 0);
    convert(0, 0, 1);
  }
  int turn = 0;
  for (; turn + STAGES <= turns; turn += STAGES) round(turn);
  if (turn < turns) step(std::integral_constant<int, 0>{}, turn);
  if constexpr (STAGES > 2)
    if (turn + 1 < turns) step(std::integral_constant<int, 1>{}, turn + 1);
  if constexpr (STAGES > 3)
    if (turn + 2 < turns) step(std::integral_constant<int, 2>{}, turn + 2);
#pragma unroll
  for (int w = 0; w < PARTS; ++w) {
    fmas(NU - 1, 0, w, pending);
    fmas(NU - 1, 1, w, pending);
  }
  __builtin_amdgcn_s_waitcnt(0);  // the loads past K land before the LDS is used again or given up
  if constexpr (WK > 1) {
    static_assert((WK - 1) * BM * BN * 4 <= WK * SLICE, "the other groups' sums fit a stage");
    f32x4* const sums = (f32x4*)st0 + wave * NU * 2 * 64 + lane;
    constexpr int GROUP = BM * BN / 4;
    __syncthreads();
    if (group > 0) {
#pragma unroll
      for (int u = 0; u < 2 * NU; ++u) sums[(group - 1) * GROUP + u * 64] = acc[u / 2 % IB][u / 2 / IB][u & 1];
    }
    __syncthreads();
    if (group == 0) {
      for (int o = 0; o < WK - 1; ++o)
#pragma unroll
        for (int u = 0; u < 2 * NU; ++u) acc[u / 2 % IB][u / 2 / IB][u & 1] += sums[o * GROUP + u * 64];
    }
  }

  // Lane (l16, g) holds row l16 of each group of rows and the columns 16 c + 4 g + 0..3 of each block. Values and bias first;
  // a gated wavefront has its outputs in the gate's blocks then.
  constexpr int TO = GATED ? TN / 2 : TN;
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
  auto bias4 = [&](const float* p, int n) __attribute__((always_inline)) -> f32x4 {
    if (n + 4 <= a.N) return *(const f32x4_any*)(p + n);
    f32x4 v = {};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.N) v[e] = p[n + e];
    return v;
  };
#pragma unroll
  for (int j = 0; j < TO; ++j)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int n = n0 + wn * WON + j * 32 + 16 * c + 4 * g;
      f32x4 b = {}, u = {};
      if (a.bias) b = bias4(a.bias, n);
      if (GATED && a.up_bias) u = bias4(a.up_bias, n);
#pragma unroll
      for (int i = 0; i < IB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = acc[i][j][c][e] + b[e];
          if constexpr (GATED)
            acc[i][j][c][e] = act_f8<ACT>(v) * (acc[i][j + TO][c][e] + u[e]);
          else
            acc[i][j][c][e] = v;
        }
    }
  // Every wavefront passes its part of the tile through LDS of its own, 32 rows at a time, so that
  // stores leave in whole rows of the part
  typedef uint32_t out16 __attribute__((ext_vector_type(4), aligned(2)));
  constexpr int ES = OUT == F8_F32 ? 4 : 2;
  constexpr int E = 16 / ES, JG = OUT == F8_F32 ? 1 : TO;
  constexpr int PITCH = JG * 32 * ES + 16, CPW = JG * 32 / E, HALF = (WM * WN + 1) / 2;
  static_assert(HALF * 32 * PITCH <= WK * SLICE, "the parts of half the wavefronts fit a stage");
  char* const part = (wave < HALF ? st0 + wave * 32 * PITCH : st1 + (wave - HALF) * 32 * PITCH);
  __syncthreads();
  if (WK > 1 && group > 0) return;  // no barrier follows: codes have one group
  BlockF8 bq[OUT == F8_CODES ? IB : 1];
  if constexpr (OUT == F8_CODES) {
    // the scale of a row's 128 columns: every wavefront's largest, joined in LDS
    static_assert(ON == kF8Block, "a tile holds whole blocks of outputs");
    constexpr int CP = WN + 1;
    uint32_t* const tops = (uint32_t*)st1;
    static_assert(BM * CP * 4 <= SLICE, "the rows' largest fit a stage");
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      uint32_t t = 0;
#pragma unroll
      for (int j = 0; j < TO; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int n = n0 + wn * WON + j * 32 + 16 * (e >> 2) + 4 * g + (e & 3);
          if (n < a.N) t = max(t, abs_bits(acc[i][j][e >> 2][e & 3]));
        }
      t = xor_max<32>(xor_max<16>(t));
      if (g == 0) tops[(wm * TM * 32 + i * 16 + l16) * CP + wn] = t;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      const uint32_t* const p = tops + (wm * TM * 32 + i * 16 + l16) * CP;
      uint32_t t = p[0];
#pragma unroll
      for (int w = 1; w < WN; ++w) t = max(t, p[w]);
      bq[i] = block_f8(t);
      const int m = m0 + wm * TM * 32 + i * 16 + l16;
      if (wn == 0 && g == 0 && m < a.M) a.out_scale[(int64_t)m * a.os_row + (int64_t)(n0 / kF8Block) * a.os_block] = bq[i].scale;
    }
  }
  if constexpr (OUT == F8_CODES) {
    // the wavefronts' pieces of a row join in LDS, so that its 128 codes leave as one line (in pieces of
    // 32 bytes, 16384 x 4608 codes took 99 MB of writes instead of 78)
    constexpr int ROW = ON + 16;
    static_assert(BM * ROW <= SLICE, "the tile's codes fit a stage");
#pragma unroll
    for (int i = 0; i < IB; ++i) {
      float v[8 * TO];
#pragma unroll
      for (int e = 0; e < 8 * TO; ++e) v[e] = acc[i][e / 8][e / 4 % 2][e % 4];
      uint32_t q[2 * TO];
      codes_f8(v, bq[i], q);
      char* const p = st0 + (wm * TM * 32 + i * 16 + l16) * ROW + wn * WON + 4 * g;
#pragma unroll
      for (int c = 0; c < 2 * TO; ++c) *(uint32_t*)(p + c * 16) = q[c];
    }
    __syncthreads();
    for (int c = tid; c < BM * ON / 16; c += NT) {
      const int r = c / (ON / 16), m = m0 + r, n = n0 + c % (ON / 16) * 16;
      const u32x4 o = *(const u32x4*)(st0 + r * ROW + c % (ON / 16) * 16);
      uint8_t* const to = (uint8_t*)a.out + (int64_t)m * a.ldo + n;
      if (m < a.M && n + 16 <= a.N) {
        __builtin_nontemporal_store(o, (u32x4*)to);  // rows of codes start at multiples of 16
      } else if (m < a.M) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (n + e < a.N) to[e] = (uint8_t)(o[e >> 2] >> (8 * (e & 3)));
      }
    }
    return;
  }
#pragma unroll
  for (int j0 = 0; j0 < TO; j0 += JG) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const auto& rows = acc[2 * i + h];
        char* const p = part + (16 * h + l16) * PITCH + 4 * g * ES;
#pragma unroll
        for (int c = 0; c < 2 * JG; ++c) {
          const f32x4 v = rows[j0 + c / 2][c % 2];
          char* const to = p + c * 16 * ES;
          if constexpr (OUT == F8_F32)
            *(f32x4*)to = v;
          else
            *(uint2*)to = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
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
              else
                ((uint16_t*)to)[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
            }
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Few rows, up to 16 MT: the weights are read once and bound it, so a wavefront takes only sixteen columns (gated:
// of both projections) and a KS-th of the blocks of K, straight from memory to the matrix cores, and the sums
// are joined in LDS in a fixed order. Outputs that are codes have no such kernel: eight such runs of columns, the 128
// outputs that share a scale, in one workgroup took 20.7 us for 32 x 2 x 1152 x 1152, a tile of 32 x 256 9.6.
template <int MT, int KS, F8Out OUT, F8Act ACT>
__global__ __launch_bounds__(KS * 64) void few_f8_kernel(GemmF8Args a) {
  constexpr bool GATED = ACT != F8_NONE;
  constexpr int P = GATED ? 2 : 1, AHEAD = MT * P > 2 ? 2 : 4;
  __shared__ __attribute__((aligned(16))) f32x4 sums[KS][P][MT][64];
  const int lane = threadIdx.x & 63, ks = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int n0 = (int)blockIdx.x * 16;
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
  for (int kb0 = ks; kb0 < nk; kb0 += AHEAD * KS) {
    i32x8 b[AHEAD][P], x[AHEAD][MT];
    float s[AHEAD][MT], w[AHEAD][P];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int kb = kb0 + u * KS, k = kb * kF8Block + 32 * g, sk = min(kb, nk - 1);
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
      const int kb = kb0 + u * KS, k = kb * kF8Block + 32 * g;
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
          const f32x4 d = sum_of_block<OUT != F8_BF16>(b[u][p], x[u][t]);
          const float f = s[u][t] * w[u][p];
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[p][t][e] = __builtin_fmaf(d[e], f, acc[p][t][e]);
        }
    }
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[ks][p][t][lane] = acc[p][t];
  __syncthreads();
  // four adjacent columns of a row to a thread
  for (int e = threadIdx.x; e < MT * 64; e += KS * 64) {
    const int c = e % 4, m = e / 4 % 16, t = e / 64;
    const int row = t * 16 + m, n = n0 + c * 4, left = a.N - n;
    f32x4 v[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      v[p] = sums[0][p][t][c * 16 + m];
#pragma unroll
      for (int k = 1; k < KS; ++k) v[p] += sums[k][p][t][c * 16 + m];
    }
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = v[0][i];
      if (a.bias && i < left) x[i] += a.bias[n + i];
      if constexpr (GATED) {
        float u = v[P - 1][i];
        if (a.up_bias && i < left) u += a.up_bias[n + i];
        x[i] = act_f8<ACT>(x[i]) * u;
      }
    }
    if (row >= a.M) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) {
        if constexpr (OUT == F8_F32)
          ((float*)a.out)[(int64_t)row * a.ldo + n + i] = x[i];
        else
          ((bf16*)a.out)[(int64_t)row * a.ldo + n + i] = (bf16)x[i];
      }
  }
}

// K over four wavefronts, from 4096 on over eight (8 x 8192 x 4096 11.4 us and 9.3, 32 x 2 x 1152 x 4608 12.9 and 11.7, 8 x 1152
// x 4608 level; 16 x 1152 x 2048 4.0 and 4.2, 16 x 4608 x 1152 5.0 and 5.8).
template <F8Out OUT, F8Act ACT, int KS>
static void launch_few_of(const GemmF8Args& a, hipStream_t s) {
  const dim3 grid((uint32_t)((a.N + 15) / 16));
  if (a.M <= 16)
    launch(few_f8_kernel<1, KS, OUT, ACT>, grid, dim3(KS * 64), 0, s, a);
  else
    launch(few_f8_kernel<2, KS, OUT, ACT>, grid, dim3(KS * 64), 0, s, a);
}
template <F8Out OUT, F8Act ACT>
static void launch_few(const GemmF8Args& a, hipStream_t s) {
  if (a.K < 4096) launch_few_of<OUT, ACT, 4>(a, s);
  else launch_few_of<OUT, ACT, 8>(a, s);
}

// Tiles: BM x BN, wave grid, groups of it, LDS stages, wavefronts per SIMD.
#define SF_F8_TILES(X)                       \
  X(kF8Split32, 32, 64, 1, 1, 2, 3, 1)       \
  X(kF8Split32x4, 32, 64, 1, 1, 4, 3, 1)     \
  X(kF8Split64, 64, 64, 2, 1, 2, 4, 1)       \
  X(kF8Split64x4, 64, 64, 2, 1, 4, 2, 1)     \
  X(kF8Deep128, 128, 128, 4, 2, 1, 4, 2)     \
  X(kF8Tile128, 128, 128, 2, 2, 1, 2, 2)     \
  X(kF8Codes32, 32, 256, 1, 4, 1, 2, 2)      \
  X(kF8Codes64, 64, 256, 1, 4, 1, 2, 2)      \
  X(kF8Tile128x256, 128, 256, 2, 4, 1, 3, 2) \
  X(kF8Tile256x256, 256, 256, 4, 2, 1, 2, 2)

template <F8Out OUT, F8Act ACT>
static hipError_t launch_f8(const GemmF8Args& a, hipStream_t s) {
  constexpr bool kGated = ACT != F8_NONE;
  const F8Tile tile = choose_gemm_f8_tile(a.M, (long)a.N * (kGated ? 2 : 1), a.K, OUT == F8_CODES, OUT == F8_F32, kGated);
  switch (tile) {  // a tile without a kernel of this kind, which the rule does not give, is no answer
    case kF8Few:
      if constexpr (f8_has_tile(kF8Few, OUT == F8_CODES, OUT != F8_BF16)) {
        launch_few<OUT, ACT>(a, s);
        return hipGetLastError();
      }
      break;
#define SF_F8_CASE(id, bm, bn, wm, wn, wk, st, mw)                                                                               \
  case id:                                                                                                                       \
    if constexpr (f8_has_tile(id, OUT == F8_CODES, OUT != F8_BF16)) {                                                            \
      constexpr int on = kGated ? bn / 2 : bn;                                                                                   \
      const int64_t tiles = (((int64_t)a.M + bm - 1) / bm) * (((int64_t)a.N + on - 1) / on);                                     \
      if (tiles > 0x7fffffff) break;                                                                                             \
      launch(gemm_f8_kernel<bm, bn, wm, wn, wk, st, mw, OUT, ACT>, dim3((uint32_t)tiles), dim3(wm * wn * wk * 64), 0, s, a);     \
      return hipGetLastError();                                                                                                  \
    }                                                                                                                            \
    break;
    SF_F8_TILES(SF_F8_CASE)
#undef SF_F8_CASE
  }
  return hipErrorInvalidValue;
}

static hipError_t launch_part(F8Out kind, F8Act act, const GemmF8Args& a, hipStream_t s) {
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

// Events for a launch's own times (t_launch_events) go to the first part alone; nothing times these calls by them.
hipError_t launch_gemm_f8(F8Out kind, F8Act act, const GemmF8Args& a, hipStream_t s) {
  const int sides = act == F8_NONE ? 1 : 2;
  long rows, cols;
  choose_gemm_f8_parts(a.M, (long)a.N * sides, a.K, kind == F8_CODES, kind == F8_F32, rows, cols);
  cols /= sides;
  GemmF8Args first = a, rest = a;
  first.M = (int)rows;
  first.N = (int)cols;
  if (rows == a.M && cols == a.N) return launch_part(kind, act, first, s);
  const int es = kind == F8_CODES ? 1 : kind == F8_BF16 ? 2 : 4;
  if (rows < a.M) {
    rest.M = a.M - first.M;
    rest.a.q += rows * a.a.ld;
    rest.a.scale += rows * a.a.s_row;
    rest.out = (char*)a.out + rows * a.ldo * es;
    if (a.out_scale) rest.out_scale += rows * a.os_row;
  } else {  // a multiple of 128 columns
    rest.N = a.N - first.N;
    rest.b.q += cols * a.b.ld;
    rest.b.scale += cols / kF8Block * a.b.s_row;
    if (act != F8_NONE) {
      rest.up.q += cols * a.up.ld;
      rest.up.scale += cols / kF8Block * a.up.s_row;
    }
    if (a.bias) rest.bias += cols;
    if (a.up_bias) rest.up_bias += cols;
    rest.out = (char*)a.out + cols * es;
    if (a.out_scale) rest.out_scale += cols / kF8Block * a.os_block;
  }
  const hipError_t e = launch_part(kind, act, first, s);
  return e != hipSuccess ? e : launch_part(kind, act, rest, s);
}

}  // namespace sf
