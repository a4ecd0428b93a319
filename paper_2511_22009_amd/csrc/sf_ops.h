// Launches of the 8-bit codes and of the normalised and turned heads: on a caller's tensors and
// inside a model's blocks.
#pragma once

#include "sf_launch.h"

namespace sf {

// ---- rows to 8-bit codes -------------------------------------------------------------
struct QuantArgs {
  const void* x;        // [M][K], row length ldx, bf16 or fp32
  int64_t ldx;
  int M, K;
  int8_t* q;            // [M][K], row length ldq (a multiple of 16, 16-byte aligned)
  int64_t ldq;
  float* scale;         // [M]
};
hipError_t launch_quantize_rows(bool x_bf16, const QuantArgs& a, hipStream_t s);
// The rows of launch_ln as 8-bit codes, straight from their fp32 values: out int8, row length ldq (a
// multiple of 16, 16-byte aligned), and scale [M].
hipError_t launch_ln_codes(const LnArgs& a, int ldq, float* scale, hipStream_t s);

// ---- products of 8-bit codes: out = (A . B^T) sa[m] sb[n] + bias[n] ------------------
struct GemmI8Args {
  const int8_t* A;      // [M][K], row length lda (a multiple of 16, 16-byte aligned)
  const int8_t* B;      // [N][K], row length ldb
  int lda, ldb;
  int M, N, K;
  const float* sa;      // [M]
  const float* sb;      // [N]
  const float* bias;    // [N] or nullptr
  void* out;            // [M][N], row length ldo (I8_BF16, I8_F32, I8_GELU)
  int64_t ldo;
  GemmArgs e;           // the epilogue's fields (I8_QKV with which_base 0 and vperm, I8_RES_GATE);
                        // N, head width and h's rows as the bf16 projections need them
};
enum I8Kind {
  I8_BF16 = 0,   // out = value, bf16
  I8_F32,        // out = value, fp32
  I8_QKV,        // EPI_QKV
  I8_GELU,       // out = GELU_tanh(value), bf16
  I8_RES_GATE    // EPI_RES_GATE
};
hipError_t launch_gemm_i8(I8Kind kind, const GemmI8Args& a, hipStream_t s);

// ---- per-head norm and rotation of heads ---------------------------------------------
constexpr int kRopeAxes = 4;  // equals SF_ROPE_AXES
struct RopeHeads {
  const char* in;
  char* out;
  const float* gain;    // [dh] or nullptr
  int64_t in_row, in_tok, in_head;     // strides in elements
  int64_t out_row, out_tok, out_head;
};
struct RopeArgs {
  RopeHeads t[2];       // q and k (heads0 and heads - heads0 heads)
  int heads0, heads;
  int rows, tokens, dh;
  FastDiv div_tok;
  float eps;
  int pairs;            // rotated pairs
  int axes;
  int first[kRopeAxes + 1];  // first pair of each axis; past the last one, `pairs`
  int layout;           // SF_ROPE_*
  int spread;
  double log2_theta;
  int inverse;
  const float* pos;     // [rows][tokens][axes]
  int64_t pos_row;
  // filled in by launch_rope
  double rate[kRopeAxes];  // log2 of theta per pair of an axis
  FastDiv div_pairs;
  int chunks0;          // runs of heads of q (the others are of k)
  int step[2];          // heads of q and of k in a run
  int group_log2;       // lanes that share a head: 2^group_log2
};
// Fills in a plan's part of the arguments; false for a plan that does not fit heads of dh dims.
bool take_rope(int axes, const int* dims, int layout, int spread, double theta, int dh, RopeArgs* a);
// norm: divide by the root mean square and multiply by the gain; rotate: turn the pairs.
hipError_t launch_rope(bool is_bf16, bool norm, bool rotate, RopeArgs a, hipStream_t s);

}  // namespace sf
