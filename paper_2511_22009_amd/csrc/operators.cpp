// C ABI of the operators on the caller's own tensors: argument checks and launches.
#include "streamflow.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "sf_ops.h"
#include "sf_ops_rules.h"

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
static_assert(sf::kF8Block == SF_F8_BLOCK, "columns of a block of codes");
static_assert((int)sf::NORM_NONE == SF_NORM_NONE && (int)sf::NORM_RMS == SF_NORM_RMS && (int)sf::NORM_LAYER == SF_NORM_LAYER, "norms");

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

constexpr long long kMostLd = 1ll << 23;  // a tile's rows of codes stay within 32-bit offsets

bool codes_fit(const sf_codes* c, int K) {
  const long long need = ((long long)K + 15) / 16 * 16;
  return c && c->codes && c->scale && aligned16(c->codes) && c->ld % 16 == 0 && c->ld >= need && c->ld < kMostLd && c->scale_row >= 0 &&
         c->scale_row < (1 << 20) && c->scale_block >= 0;
}

// The codes from a row on, which for weights starts a block.
sf::F8Codes take_codes(const sf_codes* c, int64_t row, int block_rows) {
  return sf::F8Codes{c->codes + row * c->ld, (int)c->ld, c->scale + row / block_rows * c->scale_row, c->scale_row, c->scale_block};
}

// Whether every scale of the output has a place of its own as far as a stride of 0 tells.
bool own_scales(long long rows, long long blocks, long long row, long long block) {
  return row >= 0 && block >= 0 && !(rows > 1 && row == 0) && !(blocks > 1 && block == 0);
}

int f8_call(const sf_codes* a, const sf_codes* b, const sf_codes* up, const float* bias, const float* up_bias, sf::F8Act act, int M,
            int N, int K, void* out, long long ldo, int out_type, float* out_scale, long long scale_row, long long scale_block,
            void* stream) {
  const bool codes = act != sf::F8_NONE && out_type == SF_TYPE_F8;
  if ((!is_type(out_type) && !codes) || M < 0 || N < 0 || K < 1 || K > (1 << 20)) return SF_E_INVAL;
  if (M == 0 || N == 0) return SF_OK;
  if (!codes_fit(a, K) || !codes_fit(b, K) || (act != sf::F8_NONE && !codes_fit(up, K)) || !out || ldo < N || out == a->codes ||
      out == b->codes || (up && out == up->codes))
    return SF_E_INVAL;
  if (codes && (!out_scale || !aligned16(out) || ldo % 16 || !own_scales(M, (N - 1) / SF_F8_BLOCK + 1, scale_row, scale_block)))
    return SF_E_INVAL;
  const int64_t size = codes ? 1 : out_type == SF_PREC_BF16 ? 2 : 4;
  const int64_t most = sf::f8_most_rows(N);
  for (int64_t m = 0; m < M; m += most)
    for (int64_t n = 0; n < N; n += sf::kF8MostColumns) {
      sf::GemmF8Args g{};
      g.a = take_codes(a, m, 1);
      g.b = take_codes(b, n, SF_F8_BLOCK);
      if (up) g.up = take_codes(up, n, SF_F8_BLOCK);
      g.M = (int)std::min<int64_t>(most, M - m);
      g.N = (int)std::min<int64_t>(sf::kF8MostColumns, N - n);
      g.K = K;
      g.bias = bias ? bias + n : nullptr;
      g.up_bias = up_bias ? up_bias + n : nullptr;
      g.out = (char*)out + (m * ldo + n) * size;
      g.ldo = ldo;
      if (codes) g.out_scale = out_scale + m * scale_row + n / SF_F8_BLOCK * scale_block;
      g.os_row = scale_row;
      g.os_block = scale_block;
      const sf::F8Out kind = codes ? sf::F8_CODES : out_type == SF_PREC_BF16 ? sf::F8_BF16 : sf::F8_F32;
      if (sf::launch_gemm_f8(kind, act, g, (hipStream_t)stream) != hipSuccess) return SF_E_HIP;
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

int sf_quantize_f8(const void* x, int type, long long rows, int cols, long long ldx, int block_rows, unsigned char* codes,
                   long long ldc, float* scale, long long scale_row, long long scale_block, void* stream) {
  if (!is_type(type) || rows < 0 || rows > 0x7fffffff || cols < 1 || cols > (1 << 20) || (block_rows != 1 && block_rows != SF_F8_BLOCK))
    return SF_E_INVAL;
  if (rows == 0) return SF_OK;
  const int blocks = (cols - 1) / SF_F8_BLOCK + 1;
  if (!x || !codes || !scale || ldx < 0 || ldc % 16 || ldc < cols || !aligned16(codes) || (const void*)codes == x || (const void*)scale == x ||
      !own_scales((rows - 1) / block_rows + 1, blocks, scale_row, scale_block))
    return SF_E_INVAL;
  const int64_t most = kMostRows / blocks / SF_F8_BLOCK * SF_F8_BLOCK;  // at least 1024
  for (int64_t row = 0; row < rows; row += most) {
    const sf::QuantF8Args a{(const char*)x + row * ldx * (type == SF_PREC_BF16 ? 2 : 4), ldx, (int)std::min<int64_t>(most, rows - row), cols,
                            codes + row * ldc, ldc, scale + row / block_rows * scale_row, scale_row, scale_block};
    if (sf::launch_quantize_f8(type == SF_PREC_BF16, block_rows != 1, a, (hipStream_t)stream) != hipSuccess) return SF_E_HIP;
  }
  return SF_OK;
}

int sf_matmul_f8(const sf_codes* a, const sf_codes* b, const float* bias, int M, int N, int K, void* out, long long ldo,
                 int out_type, void* stream) {
  return f8_call(a, b, nullptr, bias, nullptr, sf::F8_NONE, M, N, K, out, ldo, out_type, nullptr, 0, 0, stream);
}

int sf_gated_matmul_f8(const sf_codes* a, const sf_codes* gate, const sf_codes* up, const float* gate_bias, const float* up_bias,
                       int act, int M, int N, int K, void* out, long long ldo, int out_type, float* out_scale,
                       long long scale_row, long long scale_block, void* stream) {
  if (act != SF_ACT_SILU && act != SF_ACT_GELU_TANH) return SF_E_INVAL;
  return f8_call(a, gate, up, gate_bias, up_bias, act == SF_ACT_SILU ? sf::F8_SILU : sf::F8_GELU, M, N, K, out, ldo, out_type, out_scale,
                 scale_row, scale_block, stream);
}

int sf_residual_norm(const sf_block_rows* r, void* stream) {
  if (!r || r->samples < 0 || r->tokens < 0 || (int64_t)r->samples * r->tokens > 0x7fffffff || r->dims < 1 || r->dims > 16384 ||
      !is_type(r->h_type) || !is_type(r->y_type) || r->post < SF_NORM_NONE || r->post > SF_NORM_LAYER ||
      !std::isfinite(r->residual_scale) || !(r->eps >= 0.0f) || !std::isfinite(r->eps))
    return SF_E_INVAL;
  const bool out = r->out != nullptr, codes = out && r->out_type == SF_TYPE_F8;
  if (out && ((!is_type(r->out_type) && !codes) || r->pre < SF_NORM_NONE || r->pre > SF_NORM_LAYER)) return SF_E_INVAL;
  if (r->samples == 0 || r->tokens == 0) return SF_OK;
  const auto apart = [&](long long sample, long long token) { return !(r->samples > 1 && sample == 0) && !(r->tokens > 1 && token == 0); };
  if (!r->h || !r->y || !r->h_out || !apart(r->h_out_sample, r->h_out_token) || r->h_out == r->y) return SF_E_INVAL;
  if (r->h_out == r->h && ((r->samples > 1 && r->h_out_sample != r->h_sample) || (r->tokens > 1 && r->h_out_token != r->h_token)))
    return SF_E_INVAL;
  if (out && (!apart(r->out_sample, r->out_token) || r->out == r->h || r->out == r->y || r->out == r->h_out)) return SF_E_INVAL;
  if (codes && (!r->out_scale || !aligned16(r->out) || (r->samples > 1 && r->out_sample % 16) || (r->tokens > 1 && r->out_token % 16) ||
                !apart(r->out_scale_sample, r->out_scale_token) || (r->dims > SF_F8_BLOCK && r->out_scale_block == 0)))
    return SF_E_INVAL;
  sf::ResidualNormArgs a{};
  a.h = (const char*)r->h;
  a.y = (const char*)r->y;
  a.h_out = (char*)r->h_out;
  a.h_sample = r->h_sample;
  a.h_token = r->h_token;
  a.y_sample = r->y_sample;
  a.y_token = r->y_token;
  a.ho_sample = r->h_out_sample;
  a.ho_token = r->h_out_token;
  a.gate = r->gate;
  a.gate_sample = r->gate_sample;
  a.post = r->post;
  a.post_gain = r->post_gain;
  a.r = r->residual_scale;
  a.eps = r->eps;
  a.samples = r->samples;
  a.tokens = r->tokens;
  a.D = r->dims;
  sf::NormOut kind = sf::NORM_BF16;
  if (out) {
    kind = codes ? sf::NORM_CODES : r->out_type == SF_PREC_BF16 ? sf::NORM_BF16 : sf::NORM_F32;
    a.out = (char*)r->out;
    a.out_sample = r->out_sample;
    a.out_token = r->out_token;
    a.out_scale = r->out_scale;
    a.os_sample = r->out_scale_sample;
    a.os_token = r->out_scale_token;
    a.os_block = r->out_scale_block;
    a.pre = r->pre;
    a.pre_gain = r->pre_gain;
    a.scale = r->scale;
    a.scale_sample = r->scale_sample;
    a.shift = r->shift;
    a.shift_sample = r->shift_sample;
  }
  return sf::launch_residual_norm(r->h_type == SF_PREC_BF16, r->y_type == SF_PREC_BF16, kind, a, (hipStream_t)stream) == hipSuccess
             ? SF_OK
             : SF_E_HIP;
}

}  // extern "C"
