// Products of 8-bit codes on the matrix cores, out[m][n] = (sum_k A[m][k] B[n][k]) sa[m] sb[n]
// + bias[n], or, in a network's blocks, that value's GELU, its place among the heads' queries,
// keys and transposed values, or h += gate times it: v_mfma_i32_32x32x32_i8, whose 32-bit sums
// are exact for every K the entry point allows, so no choice of tile changes a bit of a result.
// The weights are the first operand, so a lane ends up with four adjacent output columns of one
// row.
//
// What bounds it: the matrix cores at the clock that their power leaves, and what a tile costs
// besides its slices. 8192 x 8192 x 8192 takes 440 us (2500 TOP/s), 16384 x 4608 x 1152 102 us
// (1700), of which the 151 MB of outputs are 23 at the rate of a plain fill. Where a CU has one
// tile only, the L2 bounds it: 1023 x 777 x 4321 moves 64 x 64 tiles' slices at 75 bytes per ns and
// CU, 14 us (three sets of operands in turn, rows 4336 bytes apart; 10.4 with 4352, one set 11.2 and
// 10.0). Outputs that are written while the next tile is under way, by workgroups that stay and
// fetch across tiles, made a product of K = 128 a fifth faster, but the larger kernel's loop
// lost as much at 8192 x 8192 x 8192 (other sizes were not measured); slices of 64 and more stages lost,
// and K split over wavefronts took one row of 3456 x 1152 in 3.5 us instead of 4.3 and lost from 16
// rows on. K split over workgroups was not tried.
#include "sf_ops_device.h"
#include "sf_ops_rules.h"

namespace sf {

// Workgroup -> tile: each of the eight XCDs (workgroup b goes to XCD b % 8) takes a contiguous
// range of tiles, in groups of eight tile rows with M fastest, so that the rows and columns
// that a group touches are read from one L2 (groups of 2, 4 and 16 rows: level or up to 5 %
// slower).
__device__ __forceinline__ void i8_tile(int nbm, int nbn, int& mt, int& nt) {
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

// 128-wide slices of K go global -> LDS directly into a ring of STAGES buffers (rows of eight
// 16-byte chunks, swizzled by dma_swz); every wavefront owns a sub-tile of 32 x 32 blocks over
// the whole slice and reads its fragments one K step of 32 ahead, across the slice boundary
// too. The last K step of a slice has its operands in registers when the workgroup meets at
// the slice's one barrier, so that barrier frees the stage just read: its refill and the reads
// of the next slice's first fragments go out under that step's MFMAs.
//
// Codes past K: whole chunks read as zeros (an offset past the resource); in a chunk that K
// ends in, A's bytes past K are cleared in LDS before the last slice is read (a code times 0
// is 0, whatever B holds there).
template <int BM, int BN, int WM, int WN, int STAGES, int MINW, I8Kind KIND>
__global__ __launch_bounds__(WM * WN * 64, MINW) void gemm_i8_kernel(GemmI8Args a) {
  constexpr int NT = WM * WN * 64, BK = 128, CPR = 8, KS = 4;
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  static_assert(TM * WM * 32 == BM && TN * WN * 32 == BN, "wave grid must tile the block");
  constexpr int ATOT = BM * CPR, BTOT = BN * CPR;
  static_assert(ATOT % NT == 0 && BTOT % NT == 0, "whole rounds of chunks per slice");
  constexpr int ACH = ATOT / NT, BCH = BTOT / NT, LPT = ACH + BCH;
  static_assert(STAGES >= 2 && STAGES <= 4, "two to four stages");
  constexpr int SLICE = (ATOT + BTOT) * 16;
  static_assert(STAGES * SLICE <= 160 * 1024, "stages do not fit in LDS");
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
  const int nbm = (a.M + BM - 1) / BM, nbn = (a.N + BN - 1) / BN;
  i8_tile(nbm, nbn, mt, nt);
  const int m0 = mt * BM, n0 = nt * BN;
  // the epilogue's scales and bias are fetched now: lane l holds those of column l % 32 of each
  // block column and of row l % 32 of each block row
  float sa_v[TM], sb_v[TN], bias_v[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) sa_v[i] = a.sa[min(m0 + (wm * TM + i) * 32 + l32, a.M - 1)];
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int n = min(n0 + (wn * TN + j) * 32 + l32, a.N - 1);
    sb_v[j] = a.sb[n];
    bias_v[j] = a.bias ? a.bias[n] : 0.0f;
  }
  int a_off[ACH], b_off[BCH], a_kc[ACH], b_kc[BCH];
#pragma unroll
  for (int i = 0; i < ACH; ++i) {
    const int p = tid + i * NT, row = p / CPR;
    a_kc[i] = ((p % CPR) ^ dma_swz<CPR>(row)) * 16;
    a_off[i] = m0 + row < a.M ? row * a.lda + a_kc[i] : kOffOOB;
  }
#pragma unroll
  for (int i = 0; i < BCH; ++i) {
    const int p = tid + i * NT, row = p / CPR;
    b_kc[i] = ((p % CPR) ^ dma_swz<CPR>(row)) * 16;
    b_off[i] = n0 + row < a.N ? row * a.ldb + b_kc[i] : kOffOOB;
  }
  // resources based at the tile's first row and the slice's first column, as long as the
  // tile's rows (each to the end of the chunk that K ends in)
  const int8_t* const A0 = a.A + (int64_t)m0 * a.lda;
  const int8_t* const B0 = a.B + (int64_t)n0 * a.ldb;
  const int kend = (a.K + 15) & ~15;
  const uint32_t a_bytes = (uint32_t)(min(a.M - m0, BM) - 1) * a.lda + kend;
  const uint32_t b_bytes = (uint32_t)(min(a.N - n0, BN) - 1) * a.ldb + kend;
  auto issue = [&](auto fast, char* sb, int kt) __attribute__((always_inline)) {
    const int k0 = kt * BK;
    const bool live = k0 < a.K;
    const __amdgpu_buffer_rsrc_t ra = buffer_rsrc(A0 + k0, live ? a_bytes - k0 : 0u);
    const __amdgpu_buffer_rsrc_t rb = buffer_rsrc(B0 + k0, live ? b_bytes - k0 : 0u);
    constexpr bool F = decltype(fast)::value;
#pragma unroll
    for (int i = 0; i < ACH; ++i)
      buffer_load16_lds(ra, sb + (i * NT + wave * 64) * 16, F || k0 + a_kc[i] < a.K ? a_off[i] : kOffOOB);
#pragma unroll
    for (int i = 0; i < BCH; ++i)
      buffer_load16_lds(rb, sb + (ATOT + i * NT + wave * 64) * 16, F || k0 + b_kc[i] < a.K ? b_off[i] : kOffOOB);
  };
  // clears A's bytes past K in the last slice
  auto clear_tail = [&](char* sb) {
    const int c = (a.K % BK) / 16;
    for (int r = tid; r < BM; r += NT) {
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

  i32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
  const int sw = dma_swz<CPR>(l32);  // row blocks are 32 apart: every row of a lane shares it
  const int a_row = (wm * TM * 32 + l32) * CPR;
  const int b_row = ATOT + (wn * TN * 32 + l32) * CPR;
  i32x4 af[2][TM], bfr[2][TN];
  auto frags = [&](const char* cur, int buf, int kk) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) af[buf][i] = *(const i32x4*)(cur + (a_row + i * 32 * CPR + ((g + 2 * kk) ^ sw)) * 16);
#pragma unroll
    for (int j = 0; j < TN; ++j) bfr[buf][j] = *(const i32x4*)(cur + (b_row + j * 32 * CPR + ((g + 2 * kk) ^ sw)) * 16);
  };
  auto mfmas = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bfr[buf][j], af[buf][i], acc[i][j], 0, 0, 0);
  };
  constexpr int NM = TM * TN, ND = TM + TN;
  const int nk = (a.K + BK - 1) / BK;
  auto step = [&](auto fast, auto s, int kt) __attribute__((always_inline)) {
    constexpr int S = decltype(s)::value;
    const char* cur = stage(std::integral_constant<int, S>{});
#pragma unroll
    for (int kk = 0; kk + 1 < KS; ++kk) {
      frags(cur, (kk + 1) & 1, kk + 1);
      mfmas(kk & 1);
    }
    // reads spread ahead of the MFMAs of their step
#pragma unroll
    for (int i = 0; i < (KS - 1) * ND; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, NM >= ND ? NM / ND : 1, 0);
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0<(STAGES - 2) * LPT>());
    bare_barrier();
    if constexpr (!decltype(fast)::value)
      if (a.K % 16 != 0 && kt + 2 == nk) clear_tail(stage(std::integral_constant<int, S + 1>{}));
    issue(fast, stage(std::integral_constant<int, S>{}), kt + STAGES);
    frags(stage(std::integral_constant<int, S + 1>{}), 0, 0);
    mfmas((KS - 1) & 1);
#pragma unroll
    for (int i = 0; i < NM; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, (ND + NM - 1) / NM, 0);
      __builtin_amdgcn_sched_group_barrier(0x020, (LPT + NM - 1) / NM, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
  };
  auto round = [&](auto fast, int kt) __attribute__((always_inline)) {
    step(fast, std::integral_constant<int, 0>{}, kt);
    step(fast, std::integral_constant<int, 1>{}, kt + 1);
    if constexpr (STAGES > 2) step(fast, std::integral_constant<int, 2>{}, kt + 2);
    if constexpr (STAGES > 3) step(fast, std::integral_constant<int, 3>{}, kt + 3);
  };
  auto main_loop = [&](auto fast) __attribute__((always_inline)) {
    issue(fast, stage(std::integral_constant<int, 0>{}), 0);
    issue(fast, stage(std::integral_constant<int, 1>{}), 1);
    if constexpr (STAGES > 2) issue(fast, stage(std::integral_constant<int, 2>{}), 2);
    if constexpr (STAGES > 3) issue(fast, stage(std::integral_constant<int, 3>{}), 3);
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0<(STAGES - 1) * LPT>());
    bare_barrier();
    if constexpr (!decltype(fast)::value)
      if (a.K % 16 != 0 && nk == 1) clear_tail(st0);
    frags(st0, 0, 0);
    int kt = 0;
    if constexpr (!decltype(fast)::value)
      // steps that load whole slices (16384 x 1152 of 4500 columns: 82 us, 90 with every step's loads
      // checked against K; whole K take 1 % more for the larger kernel)
      for (; kt + 2 * STAGES < nk; kt += STAGES) round(std::true_type{}, kt);
    for (; kt + STAGES <= nk; kt += STAGES) round(fast, kt);
    if (kt < nk) step(fast, std::integral_constant<int, 0>{}, kt);
    if constexpr (STAGES > 2)
      if (kt + 1 < nk) step(fast, std::integral_constant<int, 1>{}, kt + 1);
    if constexpr (STAGES > 3)
      if (kt + 2 < nk) step(fast, std::integral_constant<int, 2>{}, kt + 2);
  };
  if (a.K % BK == 0)
    main_loop(std::true_type{});
  else
    main_loop(std::false_type{});
  __builtin_amdgcn_s_waitcnt(0);  // the loads past K land before the LDS is used again or given up

  // lane (l32, g) holds row l32 of each block and the columns 8 q + 4 g + 0..3
  typedef uint32_t out16 __attribute__((ext_vector_type(4), aligned(2)));
  if constexpr (KIND == I8_BF16 || KIND == I8_F32 || KIND == I8_GELU) {
    // Every wavefront passes its part of the tile through LDS of its own, 32 rows of JG blocks at
    // a time, so that stores leave in whole rows of the part, and past the L2: a launch ends
    // without a cache full of outputs, 16384 x 4608 x 1152 into memory that no cache holds after
    // 109 us, with ordinary stores 120, straight from the registers in pieces of 32 bytes 123
    // (128 x 192; 103, 123 and 163 for 256 x 256).
    typedef std::conditional_t<KIND == I8_F32, float, bf16> OT;
    constexpr int E = 16 / (int)sizeof(OT), JG = KIND == I8_F32 ? 1 : TN;
    constexpr int PITCH = JG * 32 * (int)sizeof(OT) + 16, CPW = JG * 32 / E, HALF = WM * WN / 2;
    static_assert(HALF * 32 * PITCH <= SLICE, "the parts of half the wavefronts fit a stage");
    char* const part = (wave < HALF ? st0 + wave * 32 * PITCH : st1 + (wave - HALF) * 32 * PITCH);
    __syncthreads();
#pragma unroll
    for (int j0 = 0; j0 < TN; j0 += JG) {
      float sb[JG][16], bias[JG][16];
#pragma unroll
      for (int j = 0; j < JG; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int from = 8 * (r >> 2) + 4 * g + (r & 3);
          sb[j][r] = __shfl(sb_v[j0 + j], from);
          bias[j][r] = __shfl(bias_v[j0 + j], from);
        }
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < JG; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = (float)acc[i][j0 + j][4 * q + e] * sa_v[i] * sb[j][4 * q + e] + bias[j][4 * q + e];
              if constexpr (KIND == I8_GELU) v[e] = gelu_tanh(v[e]);
            }
            char* const p = part + l32 * PITCH + (j * 32 + q * 8 + g * 4) * (int)sizeof(OT);
            if constexpr (KIND == I8_F32)
              *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
            else
              *(uint2*)p = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
          }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < 32 * CPW / 64; ++u) {
          const int c = u * 64 + lane, r = c / CPW, cc = c - r * CPW;
          const u32x4 o = *(const u32x4*)(part + r * PITCH + cc * 16);
          const int m = m0 + (wm * TM + i) * 32 + r, n = n0 + (wn * TN + j0) * 32 + cc * E;
          OT* const to = (OT*)a.out + (int64_t)m * a.ldo + n;
          if (m < a.M && n + E <= a.N) {
            __builtin_nontemporal_store(o, (out16*)to);
          } else if (m < a.M) {
#pragma unroll
            for (int e = 0; e < E; ++e)
              if (n + e < a.N) {
                if constexpr (KIND == I8_F32)
                  to[e] = __uint_as_float(o[e]);
                else
                  ((uint16_t*)to)[e] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
              }
          }
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
    return;
  }

  // The others store straight from the registers. q, k and v leave in eights: lanes l and l + 32
  // exchange halves, then the first has the eight columns of group q, the second those of q + 1.
  constexpr bool kEights = KIND == I8_QKV;
  constexpr int QS = kEights ? 2 : 1;  // groups of four columns to a store
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    // the residual and the gates of a block column are loaded before any is used (rows past M
    // and columns past N read others that exist; N is a multiple of four here)
    f32x4 h[KIND == I8_RES_GATE ? 4 : 1][TM], gate[KIND == I8_RES_GATE ? 4 : 1][TM];
    if constexpr (KIND == I8_RES_GATE) {
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int m = min(m0 + (wm * TM + i) * 32 + l32, a.M - 1);
        const int r = (int)fdiv((uint32_t)m, a.e.div_ntok);
        const float* const gates = a.e.table + (size_t)(r < a.e.n_slots ? r : r - a.e.n_slots) * a.e.ldt + a.e.gate_off;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int n = min(n0 + (wn * TN + j) * 32 + 8 * q + 4 * g, a.N - 4);
          h[q][i] = *(const f32x4*)(a.e.h + (size_t)m * a.e.ldh + n);
          gate[q][i] = *(const f32x4*)(gates + n);
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 4; q += QS) {
      float sb[4 * QS], bias[4 * QS];
#pragma unroll
      for (int r = 0; r < 4 * QS; ++r) {
        const int from = 8 * (q + (r >> 2)) + 4 * g + (r & 3);
        sb[r] = __shfl(sb_v[j], from);
        bias[r] = __shfl(bias_v[j], from);
      }
      const int n = n0 + (wn * TN + j) * 32 + 8 * q + (kEights ? 8 * g : 4 * g);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int m = m0 + (wm * TM + i) * 32 + l32;
        float v[4 * QS];
#pragma unroll
        for (int r = 0; r < 4 * QS; ++r) v[r] = (float)acc[i][j][4 * q + r] * sa_v[i] * sb[r] + bias[r];
        if constexpr (KIND == I8_RES_GATE) {
          f32x4 o = h[q][i];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += gate[q][i][e] * v[e];
          if (m < a.M && n < a.N) *(f32x4*)(a.e.h + (size_t)m * a.e.ldh + n) = o;
        } else if constexpr (KIND == I8_QKV) {
          const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16(v[0], v[1]), pack_bf16(v[4], v[5]), false, false);
          const auto y = __builtin_amdgcn_permlane32_swap(pack_bf16(v[2], v[3]), pack_bf16(v[6], v[7]), false, false);
          const u32x4 o = {x[0], y[0], x[1], y[1]};
          // the eight columns belong to one head (widths of heads are multiples of eight)
          if (m >= a.M || n >= a.N) continue;
          const int part = (int)fdiv((uint32_t)n, a.e.div_D), rem = n - part * a.e.D;
          const int head = (int)fdiv((uint32_t)rem, a.e.div_dh), d = rem - head * a.e.dh;
          const int r = (int)fdiv((uint32_t)m, a.e.div_ntok), tok = m - r * a.e.ntok;
          const size_t bh = (size_t)r * a.e.heads + head;
          if (part < 2) {
            *(u32x4*)((bf16*)(part == 0 ? a.e.q : a.e.k) + (bh * a.e.ntok + tok) * a.e.dh + d) = o;
          } else {
            // transposed, adjacent lanes adjacent tokens (in groups of four, vt_pos)
            uint16_t* const vt = (uint16_t*)a.e.vT + (bh * a.e.dh + d) * a.e.ldv + vt_pos(tok);
#pragma unroll
            for (int e = 0; e < 8; ++e) vt[(size_t)e * a.e.ldv] = (uint16_t)(o[e >> 1] >> (16 * (e & 1)));
          }
        }
      }
    }
  }
}

// Tiles: BM x BN, wave grid, LDS stages, wavefronts per SIMD.
#define SF_I8_TILES(X)                    \
  X(kI8Deep64, 64, 64, 2, 2, 4, 2)        \
  X(kI8Tile64, 64, 64, 2, 2, 2, 4)        \
  X(kI8Deep128, 128, 128, 2, 4, 4, 2)     \
  X(kI8Tile128, 128, 128, 2, 2, 2, 2)     \
  X(kI8Tile128x192, 128, 192, 2, 2, 2, 2) \
  X(kI8Tile192x256, 192, 256, 2, 4, 2, 2) \
  X(kI8Tile256x256, 256, 256, 2, 4, 2, 2)

template <I8Kind KIND>
static hipError_t launch_i8(const GemmI8Args& a, hipStream_t s) {
  constexpr bool kHeavy = KIND == I8_QKV || KIND == I8_GELU || KIND == I8_RES_GATE;
  switch (choose_gemm_i8_tile(a.M, a.N, a.K, kHeavy, KIND == I8_RES_GATE)) {
#define SF_I8_CASE(id, bm, bn, wm, wn, st, mw)                                                               \
  case id: {                                                                                                 \
    const int64_t tiles = (((int64_t)a.M + bm - 1) / bm) * (((int64_t)a.N + bn - 1) / bn);                   \
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;                                                     \
    if constexpr (!(kHeavy && id == kI8Tile256x256)) /* never chosen */                                     \
      launch(gemm_i8_kernel<bm, bn, wm, wn, st, mw, KIND>, dim3((uint32_t)tiles), dim3(wm * wn * 64), 0, s, a); \
    break;                                                                                                   \
  }
    SF_I8_TILES(SF_I8_CASE)
#undef SF_I8_CASE
  }
  return hipGetLastError();
}

hipError_t launch_gemm_i8(I8Kind kind, const GemmI8Args& a, hipStream_t s) {
  switch (kind) {
    case I8_BF16: return launch_i8<I8_BF16>(a, s);
    case I8_F32: return launch_i8<I8_F32>(a, s);
    case I8_QKV: return launch_i8<I8_QKV>(a, s);
    case I8_GELU: return launch_i8<I8_GELU>(a, s);
    case I8_RES_GATE: return launch_i8<I8_RES_GATE>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace sf
