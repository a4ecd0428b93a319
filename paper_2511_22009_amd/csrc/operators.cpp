// C ABI of the operators on the caller's own tensors: argument checks and launches.
#include "streamflow.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "sf_ops.h"

namespace sf {

bool take_rope(int axes, const int* dims, int layout, int spread, double theta, int dh, RopeArgs* a) {
  if (axes < 1 || axes > SF_ROPE_AXES || layout < SF_ROPE_ADJACENT || layout > SF_ROPE_AXIS_HALVES ||
      (spread != 0 && spread != 1) || !std::isfinite(theta) || !(theta > 1.0))
    return false;
  int pairs = 0;
  for (int i = 0; i < axes; ++i) {
    if (dims[i] < 0 || dims[i] % 2 || dims[i] > dh) return false;
    a->first[i] = pairs;
    pairs += dims[i] / 2;
  }
  if (2 * pairs > dh) return false;
  for (int i = axes; i <= SF_ROPE_AXES; ++i) a->first[i] = pairs;
  a->axes = axes;
  a->pairs = pairs;
  a->layout = layout;
  a->spread = spread;
  a->log2_theta = std::log2(theta);
  return true;
}

}  // namespace sf

namespace {

static_assert(sf::kRopeAxes == SF_ROPE_AXES, "axes of a rotation");

bool is_type(int t) { return t == SF_PREC_BF16 || t == SF_PREC_FP32; }
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Rows (columns, tokens) of one launch: a grid holds less than 2^32 threads, and a row takes at
// most 256. Longer calls are several launches.
constexpr int64_t kMostRows = 1 << 23;

// Whether every entry of the output has a place of its own as far as a stride of 0 tells.
bool own_places(const sf_heads& t, int rows, int tokens) {
  return !((rows > 1 && t.out_row == 0) || (tokens > 1 && t.out_token == 0) || (t.heads > 1 && t.out_head == 0));
}

// Whether results over their own inputs lie where these do, as far as the addresses tell.
bool apart_or_in_place(const sf_heads& t, int rows, int tokens) {
  return t.in != t.out || ((rows <= 1 || t.in_row == t.out_row) && (tokens <= 1 || t.in_token == t.out_token) &&
                           (t.heads <= 1 || t.in_head == t.out_head));
}

sf::RopeHeads take_heads(const sf_heads& t, const float* gain) {
  return sf::RopeHeads{(const char*)t.in, (char*)t.out, gain,       t.in_row,  t.in_token,
                       t.in_head,         t.out_row,    t.out_token, t.out_head};
}

int rope_call(const sf_heads* q, const sf_heads* k, const float* q_gain, const float* k_gain, bool norm, float eps, int type,
              int rows, int tokens, int dh, const sf_rope* rope, const float* pos, long long pos_row, int inverse,
              void* stream) {
  if (!q || !is_type(type) || rows < 0 || tokens < 0 || (int64_t)rows * tokens > 0x7fffffff || dh < 2 || dh > 256 || dh % 2 ||
      q->heads < 0 || (k && k->heads < 0) || (int64_t)q->heads + (k ? k->heads : 0) > 65535 || !(eps >= 0.0f) ||
      !std::isfinite(eps))
    return SF_E_INVAL;
  sf::RopeArgs a{};
  if (rope && !sf::take_rope(rope->axes, rope->dims, rope->layout, rope->spread, rope->theta, dh, &a)) return SF_E_INVAL;
  a.heads0 = q->heads;
  a.heads = q->heads + (k ? k->heads : 0);
  if (rows == 0 || tokens == 0 || a.heads == 0) return SF_OK;
  if (rope && !pos) return SF_E_INVAL;
  for (const sf_heads* t : {q, k})
    if (t && t->heads > 0 && (!t->in || !t->out || !own_places(*t, rows, tokens) || !apart_or_in_place(*t, rows, tokens)))
      return SF_E_INVAL;
  if (k && q->heads > 0 && k->heads > 0 && (q->out == k->out || q->out == k->in || k->out == q->in)) return SF_E_INVAL;
  a.t[0] = take_heads(*q, q_gain);
  if (k) a.t[1] = take_heads(*k, k_gain);
  a.dh = dh;
  a.eps = eps;
  a.inverse = inverse != 0;
  a.pos_row = pos_row;
  const int64_t most_tokens = std::min<int64_t>(tokens, kMostRows), most_rows = kMostRows / most_tokens;
  for (int64_t row = 0; row < rows; row += most_rows)
    for (int64_t token = 0; token < tokens; token += most_tokens) {
      sf::RopeArgs part = a;
      part.rows = (int)std::min(most_rows, rows - row);
      part.tokens = (int)std::min(most_tokens, tokens - token);
      part.div_tok = sf::make_fastdiv((uint32_t)part.tokens);
      for (sf::RopeHeads& t : part.t) {
        const int64_t size = type == SF_PREC_BF16 ? 2 : 4;
        if (t.in) t.in += size * (row * t.in_row + token * t.in_tok);
        if (t.out) t.out += size * (row * t.out_row + token * t.out_tok);
      }
      if (pos) part.pos = pos + row * pos_row + token * a.axes;
      const hipError_t e = sf::launch_rope(type == SF_PREC_BF16, norm, rope != nullptr, part, (hipStream_t)stream);
      if (e != hipSuccess) return SF_E_HIP;
    }
  return SF_OK;
}

}  // namespace

extern "C" {

int sf_quantize_rows(const void* x, int type, long long rows, int cols, long long ldx, signed char* codes, long long ldc,
                     float* scale, void* stream) {
  if (!is_type(type) || rows < 0 || rows > 0x7fffffff || cols < 1 || cols > (1 << 20)) return SF_E_INVAL;
  if (rows == 0) return SF_OK;
  if (!x || !codes || !scale || ldx < 0 || ldc % 16 || ldc < cols || !aligned16(codes)) return SF_E_INVAL;
  for (int64_t row = 0; row < rows; row += kMostRows) {
    const char* const from = (const char*)x + row * ldx * (type == SF_PREC_BF16 ? 2 : 4);
    const sf::QuantArgs a{from, ldx, (int)std::min<int64_t>(kMostRows, rows - row), cols, (int8_t*)codes + row * ldc, ldc, scale + row};
    if (sf::launch_quantize_rows(type == SF_PREC_BF16, a, (hipStream_t)stream) != hipSuccess) return SF_E_HIP;
  }
  return SF_OK;
}

int sf_matmul_i8(const signed char* a, long long lda, const float* a_scale, const signed char* b, long long ldb,
                 const float* b_scale, const float* bias, int M, int N, int K, void* out, long long ldo, int out_type,
                 void* stream) {
  if (!is_type(out_type) || M < 0 || N < 0 || K < 1 || K > 131071) return SF_E_INVAL;
  if (M == 0 || N == 0) return SF_OK;
  const long long need = ((long long)K + 15) / 16 * 16;
  constexpr long long kMostLd = 1ll << 23;  // a tile's rows stay within 32-bit offsets
  if (!a || !b || !a_scale || !b_scale || !out || !aligned16(a) || !aligned16(b) || lda % 16 || ldb % 16 || lda < need ||
      ldb < need || lda >= kMostLd || ldb >= kMostLd || ldo < N)
    return SF_E_INVAL;
  for (int64_t m = 0; m < M; m += kMostRows)
    for (int64_t n = 0; n < N; n += kMostRows) {
      char* const to = (char*)out + (m * ldo + n) * (out_type == SF_PREC_BF16 ? 2 : 4);
      const sf::GemmI8Args g{(const int8_t*)a + m * lda, (const int8_t*)b + n * ldb, (int)lda, (int)ldb,
                             (int)std::min<int64_t>(kMostRows, M - m), (int)std::min<int64_t>(kMostRows, N - n), K,
                             a_scale + m, b_scale + n, bias ? bias + n : nullptr, to, ldo, {}};
      const hipError_t e = sf::launch_gemm_i8(out_type == SF_PREC_BF16 ? sf::I8_BF16 : sf::I8_F32, g, (hipStream_t)stream);
      if (e != hipSuccess) return SF_E_HIP;
    }
  return SF_OK;
}

int sf_rotate(const sf_heads* x, int type, int rows, int tokens, int dh, const sf_rope* rope, const float* pos,
              long long pos_row, int inverse, void* stream) {
  if (!rope) return SF_E_INVAL;
  return rope_call(x, nullptr, nullptr, nullptr, false, 0.0f, type, rows, tokens, dh, rope, pos, pos_row, inverse, stream);
}

int sf_qk_norm_rotate(const sf_heads* q, const sf_heads* k, const float* q_gain, const float* k_gain, float eps, int type,
                      int rows, int tokens, int dh, const sf_rope* rope, const float* pos, long long pos_row,
                      void* stream) {
  return rope_call(q, k, q_gain, k_gain, true, eps, type, rows, tokens, dh, rope, pos, pos_row, 0, stream);
}

}  // extern "C"
