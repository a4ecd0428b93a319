// The operators on torch tensors, as operators.py offers them: shapes, types and devices are
// checked, outputs that are not given allocated, and the library's entry points called on the
// current stream of the tensors' device. In C++, since the smallest calls take 3 us on the GPU and
// their checks in Python took longer: norm and rotation of one token 5.7 us of host time instead of
// 11.0, rows to codes 4.9 instead of 7.8, products 4.4 instead of 8.8; 3.1 of each are the launch and
// 1 to 2 the allocations.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <sstream>
#include <string>

#include "streamflow.h"

namespace {

// What bind() was given: raises the exception of a status code, and gives a device's raw stream.
PyObject* g_check = nullptr;
PyObject* g_raw_stream = nullptr;
decltype(&sf_quantize_rows) g_quantize_rows = nullptr;
decltype(&sf_matmul_i8) g_matmul_i8 = nullptr;
decltype(&sf_rotate) g_rotate = nullptr;
decltype(&sf_qk_norm_rotate) g_qk_norm_rotate = nullptr;
decltype(&sf_quantize_f8) g_quantize_f8 = nullptr;
decltype(&sf_matmul_f8) g_matmul_f8 = nullptr;
decltype(&sf_gated_matmul_f8) g_gated_matmul_f8 = nullptr;
decltype(&sf_residual_norm) g_residual_norm = nullptr;

struct Refused {
  PyObject* type;
  std::string what;
};
struct Raised {};  // a Python exception is set

template <typename... T>
std::string text(const T&... parts) {
  std::ostringstream s;
  (s << ... << parts);
  return s.str();
}
template <typename... T>
[[noreturn]] void bad_type(const T&... parts) {
  throw Refused{PyExc_TypeError, text(parts...)};
}
template <typename... T>
[[noreturn]] void bad_value(const T&... parts) {
  throw Refused{PyExc_ValueError, text(parts...)};
}

const auto kReals = {at::kBFloat16, at::kFloat};
const auto kFloats = {at::kFloat};
const auto kCodes = {at::kChar};
const auto kF8Codes = {at::kFloat8_e4m3fn};

// A tensor of the call under way whose class dispatches to Python: a fake of torch's tracing, whose address is no memory, or
// one that keeps its values elsewhere. stream_of() refuses it, after every other check, which CPU tests run on fakes.
thread_local const char* t_elsewhere = nullptr;

const at::Tensor& tensor(PyObject* o, const char* what, std::initializer_list<at::ScalarType> types) {
  if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) bad_type(what, ": expected a CUDA tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && c10::GradMode::is_enabled())
    bad_type(what, ": requires grad, and nothing here is differentiated; call under torch.no_grad() or detach it");
  if (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined())
    bad_type(what, ": carries a forward-mode tangent, and nothing here is differentiated; call with the primal that unpack_dual() gives");
  if (t.is_neg()) bad_type(what, ": a lazily negated view, whose memory holds the opposite values; call resolve_neg()");
  if (t._is_zerotensor()) bad_type(what, ": zeros without memory; clone it");
  if (!t_elsewhere && t.unsafeGetTensorImpl()->is_python_dispatch()) t_elsewhere = what;
  for (const at::ScalarType s : types)
    if (t.scalar_type() == s) return t;
  bad_type(what, ": expected ", types.size() > 1 ? "BFloat16 or Float" : c10::toString(*types.begin()), ", got ",
           c10::toString(t.scalar_type()));
}

int type_of(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? SF_PREC_BF16 : SF_PREC_FP32; }

// Address of n adjacent fp32 values; None (where allowed) is a null pointer.
const float* vector(PyObject* o, const char* what, int64_t n, int device, bool none = false) {
  if (none && o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what, kFloats);
  if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
    bad_value(what, ": expected ", n, " adjacent values, got shape ", t.sizes(), ", strides ", t.strides());
  if (t.get_device() != device) bad_value(what, ": on ", t.device(), ", the call is on cuda:", device);
  return (const float*)t.data_ptr();
}

// The stream of a call whose tensors have passed their checks.
void* stream_of(int device) {
  if (t_elsewhere) bad_type(t_elsewhere, ": a fake tensor, or one of a class with a dispatch of its own, has no values at its address");
  PyObject* const index = PyLong_FromLong(device);
  PyObject* const raw = index ? PyObject_CallOneArg(g_raw_stream, index) : nullptr;
  Py_XDECREF(index);
  if (!raw) throw Raised{};
  void* const s = PyLong_AsVoidPtr(raw);
  Py_DECREF(raw);
  if (!s && PyErr_Occurred()) throw Raised{};
  return s;
}

void check(int rc, const char* name) {
  if (rc == SF_OK) return;
  PyObject* const r = PyObject_CallFunction(g_check, "is", rc, name);
  Py_XDECREF(r);
  if (!r) throw Raised{};
}

int as_int(int64_t v, const char* what) {
  if (v > 0x7fffffff) bad_value(what, ": ", v, " is more than a call takes");
  return (int)v;
}

// Other Python threads run while this one allocates or calls the library, either of which may wait for
// the GPU; an exception takes the lock again on its way.
class Unlocked {
 public:
  Unlocked() : state_(PyEval_SaveThread()) {}
  ~Unlocked() { PyEval_RestoreThread(state_); }
  Unlocked(const Unlocked&) = delete;

 private:
  PyThreadState* state_;
};
template <typename F>
auto unlocked(F f) {
  const Unlocked u;
  return f();
}

PyObject* pair(PyObject* a, PyObject* b) {
  PyObject* const r = a && b ? PyTuple_Pack(2, a, b) : nullptr;
  Py_XDECREF(a);
  Py_XDECREF(b);
  return r;
}
// A call's result: the tensor that was given for it, which has new values now (a backward pass that had kept the
// old ones has to see that, as after torch's own calls), or the one made here.
PyObject* given_or(PyObject* given, const at::Tensor& made) {
  if (given != Py_None) {
    const at::Tensor& t = THPVariable_Unpack(given);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    return Py_NewRef(given);
  }
  return THPVariable_Wrap(made);
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// Row length of codes whose rows start at multiples of 16 bytes.
int64_t pitch_of(const at::Tensor& t, const char* what, int64_t need) {
  if (t.size(1) > 1 && t.stride(1) != 1) bad_value(what, ": expected rows of adjacent codes, got strides ", t.strides());
  const int64_t ld = t.size(0) > 1 ? t.stride(0) : need;
  if (ld % 16 || ld < need || (uintptr_t)t.data_ptr() % 16)
    bad_value(what, ": rows have to start at multiples of 16 bytes, at least ", need, " apart (strides ", t.strides(),
              "), as quantize_rows and quantize_f8 leave them");
  return ld;
}

// x, out | None, scale | None -> (codes, scale)
PyObject* quantize_rows(PyObject* const* args) {
  const at::Tensor& x = tensor(args[0], "x", kReals);
  if (x.dim() != 2 || x.size(1) < 1 || (x.size(1) > 1 && x.stride(1) != 1))
    bad_value("x: expected rows of adjacent values, got shape ", x.sizes(), ", strides ", x.strides());
  const int64_t rows = x.size(0), cols = x.size(1), need = up16(cols);
  const int device = x.get_device();
  const int width = as_int(cols, "x");
  at::Tensor codes, scale;
  int64_t ldc = cols < 1024 ? need : (cols + 127) / 128 * 128;  // whole cache lines
  if (args[1] != Py_None) {
    codes = tensor(args[1], "out", kCodes);
    if (codes.sizes() != x.sizes() || codes.get_device() != device)
      bad_value("out: expected ", x.sizes(), " on ", x.device(), ", got ", codes.sizes(), " on ", codes.device());
    ldc = pitch_of(codes, "out", need);
  }
  float* to = const_cast<float*>(vector(args[2], "scale", rows, device, true));
  void* const stream = stream_of(device);
  const c10::DeviceGuard guard(x.device());
  const int rc = unlocked([&] {
    if (!codes.defined()) {
      codes = at::empty_strided({rows, ldc}, {ldc, 1}, x.options().dtype(at::kChar));
      if (ldc != cols) codes = codes.narrow(1, 0, cols);
    }
    if (args[2] == Py_None) {
      scale = at::empty_strided({rows}, {1}, x.options().dtype(at::kFloat));
      to = (float*)scale.data_ptr();
    }
    return g_quantize_rows(x.data_ptr(), type_of(x), rows, width, x.stride(0), (signed char*)codes.data_ptr(), ldc, to, stream);
  });
  check(rc, "sf_quantize_rows");
  return pair(given_or(args[1], codes), given_or(args[2], scale));
}

int64_t codes_of(const at::Tensor& t, const char* what) {
  if (t.dim() != 2 || t.size(1) < 1) bad_value(what, ": expected codes [rows, cols], got shape ", t.sizes());
  const int64_t rows = t.size(0), cols = t.size(1), need = up16(cols), ld = pitch_of(t, what, need);
  // rows are read in pieces of 16 bytes: the last one's has to lie in the storage too
  if (cols != need && rows && t.storage_offset() + (rows - 1) * ld + need > (int64_t)t.storage().nbytes())
    bad_value(what, ": the last row ends its storage inside a piece of 16 bytes");
  return ld;
}

// a, a_scale, b, b_scale, bias | None, type, out | None -> out
PyObject* matmul_i8(PyObject* const* args) {
  const at::Tensor& a = tensor(args[0], "a", kCodes);
  const at::Tensor& b = tensor(args[2], "b", kCodes);
  const int64_t lda = codes_of(a, "a"), ldb = codes_of(b, "b");
  const int64_t M = a.size(0), K = a.size(1), N = b.size(0);
  const int device = a.get_device();
  if (b.size(1) != K || b.get_device() != device)
    bad_value("b: expected [N, ", K, "] on ", a.device(), ", got ", b.sizes(), " on ", b.device());
  const float* const sa = vector(args[1], "a_scale", M, device);
  const float* const sb = vector(args[3], "b_scale", N, device);
  const float* const bias = vector(args[4], "bias", N, device, true);
  const int m = as_int(M, "a"), n = as_int(N, "b"), k = as_int(K, "a");
  at::Tensor out;
  int64_t ldo = N;
  long type = 0;
  if (args[6] == Py_None) {
    type = PyLong_AsLong(args[5]);
    if (type == -1 && PyErr_Occurred()) throw Raised{};
  } else {
    out = tensor(args[6], "out", kReals);
    if (out.dim() != 2 || out.size(0) != M || out.size(1) != N || out.get_device() != device || (N > 1 && out.stride(1) != 1) ||
        (M > 1 && out.stride(0) < N))
      bad_value("out: expected [", M, ", ", N, "] with adjacent columns on ", a.device(), ", got ", out.sizes(), ", strides ",
                out.strides(), " on ", out.device());
    if (M > 1) ldo = out.stride(0);
  }
  void* const stream = stream_of(device);
  const c10::DeviceGuard guard(a.device());
  const int rc = unlocked([&] {
    if (!out.defined()) out = at::empty_strided({M, N}, {N, 1}, a.options().dtype(type == SF_PREC_BF16 ? at::kBFloat16 : at::kFloat));
    return g_matmul_i8((const signed char*)a.data_ptr(), lda, sa, (const signed char*)b.data_ptr(), ldb, sb, bias, m, n, k,
                       out.data_ptr(), ldo, type_of(out), stream);
  });
  check(rc, "sf_matmul_i8");
  return given_or(args[6], out);
}

const at::Tensor& heads_in(PyObject* o, const char* what) {
  const at::Tensor& t = tensor(o, what, kReals);
  if (t.dim() != 4 || (t.size(3) > 1 && t.stride(3) != 1))
    bad_value(what, ": expected [rows, tokens, heads, dims] with adjacent dims, got shape ", t.sizes(), ", strides ", t.strides());
  return t;
}

// The output that is given for x, or an undefined tensor.
at::Tensor heads_out(const at::Tensor& x, const char* what, PyObject* given) {
  if (given == Py_None) return {};
  const at::Tensor& out = tensor(given, what, {x.scalar_type()});
  if (out.sizes() != x.sizes() || out.get_device() != x.get_device() || (x.size(3) > 1 && out.stride(3) != 1))
    bad_value(what, " out: expected ", x.sizes(), " with adjacent dims on ", x.device(), ", got ", out.sizes(), ", strides ",
              out.strides(), " on ", out.device());
  return out;
}

// x and its output, allocated where none is given, as the library takes them.
sf_heads heads_of(const at::Tensor& x, int heads, at::Tensor& out) {
  if (!out.defined()) {
    out = at::empty_like(x);
    // an x whose entries overlap (windows): its strides' order is not the output's
    if (out.stride(3) != 1) out = at::empty_like(x, at::MemoryFormat::Contiguous);
  }
  return sf_heads{x.data_ptr(), out.data_ptr(), heads,         x.stride(0),  x.stride(1),
                  x.stride(2),  out.stride(0),  out.stride(1), out.stride(2)};
}

struct Positions {
  const float* at;
  int64_t row;
};
Positions positions(PyObject* o, const sf_rope& rope, const at::Tensor& x) {
  const at::Tensor& p = tensor(o, "positions", kFloats);
  const int64_t rows = x.size(0), tokens = x.size(1), d = p.dim();
  const bool shared = d == 2 || (d == 3 && p.size(0) == 1);
  if ((!shared && (d != 3 || p.size(0) != rows)) || p.size(d - 2) != tokens || p.size(d - 1) != rope.axes ||
      p.get_device() != x.get_device())
    bad_value("positions: expected [tokens, axes] or [rows, tokens, axes] = [", rows, ", ", tokens, ", ", rope.axes, "] on ", x.device(),
              ", got ", p.sizes(), " on ", p.device());
  if ((rope.axes > 1 && p.stride(d - 1) != 1) || (tokens > 1 && p.stride(d - 2) != rope.axes))
    bad_value("positions: expected [tokens, axes] without gaps, got strides ", p.strides());
  return {(const float*)p.data_ptr(), shared ? 0 : p.stride(0)};
}

const sf_rope* rope_of(PyObject* address) {
  const sf_rope* const r = (const sf_rope*)PyLong_AsVoidPtr(address);
  if (!r && PyErr_Occurred()) throw Raised{};
  return r;
}

// x, positions, address of the sf_rope, inverse, out | None -> out
PyObject* rotate(PyObject* const* args) {
  const at::Tensor& x = heads_in(args[0], "x");
  const sf_rope* const rope = rope_of(args[2]);
  const Positions pos = positions(args[1], *rope, x);
  const int inverse = PyObject_IsTrue(args[3]);
  if (inverse < 0) throw Raised{};
  at::Tensor out = heads_out(x, "x", args[4]);
  const int rows = as_int(x.size(0), "x"), tokens = as_int(x.size(1), "x"), heads = as_int(x.size(2), "x"), dims = as_int(x.size(3), "x");
  void* const stream = stream_of(x.get_device());
  const c10::DeviceGuard guard(x.device());
  const int rc = unlocked([&] {
    const sf_heads h = heads_of(x, heads, out);
    return g_rotate(&h, type_of(x), rows, tokens, dims, rope, pos.at, pos.row, inverse, stream);
  });
  check(rc, "sf_rotate");
  return given_or(args[4], out);
}

// q, k | None, q_gain | None, k_gain | None, positions, address of the sf_rope (0: the norm alone),
// eps, q out | None, k out | None -> (q, k)
PyObject* qk_norm_rotate(PyObject* const* args) {
  const at::Tensor& q = heads_in(args[0], "q");
  const bool has_k = args[1] != Py_None;
  const int device = q.get_device();
  const int64_t dims = q.size(3);
  if (has_k) {
    const at::Tensor& k = heads_in(args[1], "k");
    if (k.size(0) != q.size(0) || k.size(1) != q.size(1) || k.size(3) != dims || k.scalar_type() != q.scalar_type() ||
        k.get_device() != device)
      bad_value("k: ", k.sizes(), " of ", c10::toString(k.scalar_type()), " on ", k.device(), " does not go with q: ", q.sizes(),
                " of ", c10::toString(q.scalar_type()), " on ", q.device());
  }
  const float* const q_gain = vector(args[2], "q_gain", dims, device, true);
  const float* const k_gain = vector(args[3], "k_gain", dims, device, true);
  const sf_rope* const rope = rope_of(args[5]);
  Positions pos{nullptr, 0};
  if (rope) {
    if (args[4] == Py_None) bad_value("positions: needed with rotary");
    pos = positions(args[4], *rope, q);
  }
  const double eps = PyFloat_AsDouble(args[6]);
  if (eps == -1.0 && PyErr_Occurred()) throw Raised{};
  at::Tensor q_out = heads_out(q, "q", args[7]), k_out;
  const at::Tensor* const k = has_k ? &THPVariable_Unpack(args[1]) : nullptr;
  if (k) k_out = heads_out(*k, "k", args[8]);
  const int rows = as_int(q.size(0), "q"), tokens = as_int(q.size(1), "q"), dh = as_int(dims, "q");
  const int q_heads = as_int(q.size(2), "q"), k_heads = k ? as_int(k->size(2), "k") : 0;
  void* const stream = stream_of(device);
  const c10::DeviceGuard guard(q.device());
  const int rc = unlocked([&] {
    const sf_heads hq = heads_of(q, q_heads, q_out), hk = k ? heads_of(*k, k_heads, k_out) : sf_heads{};
    return g_qk_norm_rotate(&hq, k ? &hk : nullptr, q_gain, k_gain, (float)eps, type_of(q), rows, tokens, dh, rope, pos.at,
                            pos.row, stream);
  });
  check(rc, "sf_qk_norm_rotate");
  return pair(given_or(args[7], q_out), has_k ? given_or(args[8], k_out) : Py_NewRef(Py_None));
}

// ---- e4m3 codes -------------------------------------------------------------------------

int64_t blocks_of(int64_t n) { return (n + SF_F8_BLOCK - 1) / SF_F8_BLOCK; }
int64_t codes_pitch(int64_t cols) { return cols < 1024 ? up16(cols) : (cols + 127) / 128 * 128; }  // whole cache lines
bool is_codes(const at::Tensor& t) { return t.scalar_type() == at::kFloat8_e4m3fn; }
int out_type_of(const at::Tensor& t) { return is_codes(t) ? (int)SF_TYPE_F8 : type_of(t); }
at::ScalarType scalar_of(long type) {
  return type == SF_TYPE_F8 ? at::kFloat8_e4m3fn : type == SF_PREC_BF16 ? at::kBFloat16 : at::kFloat;
}
long long_of(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
float float_of(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return (float)v;
}

// Scales [rows][blocks] that are given for codes, to be read or written.
at::Tensor scales_given(PyObject* o, const char* what, int64_t rows, int64_t blocks, const at::Tensor& codes) {
  const at::Tensor& t = tensor(o, what, kFloats);
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != blocks || t.get_device() != codes.get_device())
    bad_value(what, ": expected [", rows, ", ", blocks, "] on ", codes.device(), ", got ", t.sizes(), " on ", t.device());
  return t;
}
// New ones, those of adjacent rows adjacent, as the products read them fastest.
at::Tensor new_scales(int64_t rows, int64_t blocks, const at::Tensor& like) {
  return at::empty_strided({rows, blocks}, {1, rows}, like.options().dtype(at::kFloat));
}

// x, block_rows, out | None, scale | None -> (codes, scale)
PyObject* quantize_f8(PyObject* const* args) {
  const at::Tensor& x = tensor(args[0], "x", kReals);
  if (x.dim() != 2 || x.size(1) < 1 || (x.size(1) > 1 && x.stride(1) != 1))
    bad_value("x: expected rows of adjacent values, got shape ", x.sizes(), ", strides ", x.strides());
  const long block_rows = long_of(args[1]);
  if (block_rows != 1 && block_rows != SF_F8_BLOCK) bad_value("block_rows: expected 1 or ", SF_F8_BLOCK, ", got ", block_rows);
  const int64_t rows = x.size(0), cols = x.size(1), need = up16(cols), blocks = blocks_of(cols);
  const int64_t scale_rows = block_rows == 1 ? rows : blocks_of(rows);
  const int width = as_int(cols, "x");
  at::Tensor codes, scale;
  int64_t ldc = codes_pitch(cols);
  if (args[2] != Py_None) {
    codes = tensor(args[2], "out", kF8Codes);
    if (codes.sizes() != x.sizes() || codes.get_device() != x.get_device())
      bad_value("out: expected ", x.sizes(), " on ", x.device(), ", got ", codes.sizes(), " on ", codes.device());
    ldc = pitch_of(codes, "out", need);
  }
  if (args[3] != Py_None) scale = scales_given(args[3], "scale", scale_rows, blocks, x);
  void* const stream = stream_of(x.get_device());
  const c10::DeviceGuard guard(x.device());
  const int rc = unlocked([&] {
    if (!codes.defined()) {
      codes = at::empty_strided({rows, ldc}, {ldc, 1}, x.options().dtype(at::kFloat8_e4m3fn));
      if (ldc != cols) codes = codes.narrow(1, 0, cols);
    }
    if (!scale.defined()) scale = new_scales(scale_rows, blocks, x);
    return g_quantize_f8(x.data_ptr(), type_of(x), rows, width, x.stride(0), (int)block_rows, (unsigned char*)codes.data_ptr(), ldc,
                         (float*)scale.data_ptr(), scale.stride(0), scale.stride(1), stream);
  });
  check(rc, "sf_quantize_f8");
  return pair(given_or(args[2], codes), given_or(args[3], scale));
}

// Codes [rows][K] and their scales, of `block_rows` rows each, as a product reads them.
sf_codes f8_codes(PyObject* codes, PyObject* scale, const char* what, const char* scale_what, int64_t block_rows, const at::Tensor* first) {
  const at::Tensor& t = tensor(codes, what, kF8Codes);
  const int64_t ld = codes_of(t, what);
  if (first && (t.size(1) != first->size(1) || t.get_device() != first->get_device()))
    bad_value(what, ": expected [rows, ", first->size(1), "] on ", first->device(), ", got ", t.sizes(), " on ", t.device());
  const at::Tensor s = scales_given(scale, scale_what, block_rows == 1 ? t.size(0) : blocks_of(t.size(0)), blocks_of(t.size(1)), t);
  return sf_codes{(const unsigned char*)t.data_ptr(), ld, (const float*)s.data_ptr(), s.size(0) > 1 ? s.stride(0) : 0, s.stride(1)};
}

// The output [M][N] of a product that is given, or an undefined tensor; its row length.
at::Tensor product_out(PyObject* o, int64_t M, int64_t N, const at::Tensor& a, bool codes_too, int64_t* ldo) {
  if (o == Py_None) return {};
  const bool codes = codes_too && THPVariable_Check(o) && is_codes(THPVariable_Unpack(o));
  const at::Tensor out = codes ? tensor(o, "out", kF8Codes) : tensor(o, "out", kReals);
  if (out.dim() != 2 || out.size(0) != M || out.size(1) != N || out.get_device() != a.get_device() || (N > 1 && out.stride(1) != 1) ||
      (M > 1 && out.stride(0) < N))
    bad_value("out: expected [", M, ", ", N, "] with adjacent columns on ", a.device(), ", got ", out.sizes(), ", strides ", out.strides(),
              " on ", out.device());
  if (codes)
    *ldo = pitch_of(out, "out", up16(N));
  else if (M > 1)
    *ldo = out.stride(0);
  return out;
}

// a, a_scale, b, b_scale, bias | None, type, out | None -> out
PyObject* matmul_f8(PyObject* const* args) {
  const sf_codes ca = f8_codes(args[0], args[1], "a", "a_scale", 1, nullptr);
  const at::Tensor& a = THPVariable_Unpack(args[0]);
  const sf_codes cb = f8_codes(args[2], args[3], "b", "b_scale", SF_F8_BLOCK, &a);
  const int64_t M = a.size(0), K = a.size(1), N = THPVariable_Unpack(args[2]).size(0);
  const float* const bias = vector(args[4], "bias", N, a.get_device(), true);
  const int m = as_int(M, "a"), n = as_int(N, "b"), k = as_int(K, "a");
  const long type = long_of(args[5]);
  int64_t ldo = N;
  at::Tensor out = product_out(args[6], M, N, a, false, &ldo);
  void* const stream = stream_of(a.get_device());
  const c10::DeviceGuard guard(a.device());
  const int rc = unlocked([&] {
    if (!out.defined()) out = at::empty_strided({M, N}, {N, 1}, a.options().dtype(scalar_of(type)));
    return g_matmul_f8(&ca, &cb, bias, m, n, k, out.data_ptr(), ldo, type_of(out), stream);
  });
  check(rc, "sf_matmul_f8");
  return given_or(args[6], out);
}

// a, a_scale, gate, gate_scale, up, up_scale, gate_bias | None, up_bias | None, act, type, out | None,
// out_scale | None -> out, or (out, out_scale) where out is codes
PyObject* gated_matmul_f8(PyObject* const* args) {
  const sf_codes ca = f8_codes(args[0], args[1], "a", "a_scale", 1, nullptr);
  const at::Tensor& a = THPVariable_Unpack(args[0]);
  const sf_codes cg = f8_codes(args[2], args[3], "gate", "gate_scale", SF_F8_BLOCK, &a);
  const sf_codes cu = f8_codes(args[4], args[5], "up", "up_scale", SF_F8_BLOCK, &a);
  const int64_t M = a.size(0), K = a.size(1), N = THPVariable_Unpack(args[2]).size(0);
  if (THPVariable_Unpack(args[4]).size(0) != N) bad_value("up: expected ", N, " rows as gate has, got ", THPVariable_Unpack(args[4]).size(0));
  const float* const gate_bias = vector(args[6], "gate_bias", N, a.get_device(), true);
  const float* const up_bias = vector(args[7], "up_bias", N, a.get_device(), true);
  const int m = as_int(M, "a"), n = as_int(N, "gate"), k = as_int(K, "a");
  const long act = long_of(args[8]), type = long_of(args[9]);
  int64_t ldo = N;
  at::Tensor out = product_out(args[10], M, N, a, true, &ldo), scale;
  const bool codes = out.defined() ? is_codes(out) : type == SF_TYPE_F8;
  if (args[11] != Py_None) {
    if (!codes) bad_value("out_scale: only with outputs that are codes");
    scale = scales_given(args[11], "out_scale", M, blocks_of(N), a);
  }
  void* const stream = stream_of(a.get_device());
  const c10::DeviceGuard guard(a.device());
  const int rc = unlocked([&] {
    if (!out.defined()) {
      if (codes) ldo = codes_pitch(N);
      out = at::empty_strided({M, ldo}, {ldo, 1}, a.options().dtype(scalar_of(type)));
      if (ldo != N) out = out.narrow(1, 0, N);
    }
    if (codes && !scale.defined()) scale = new_scales(M, blocks_of(N), a);
    return g_gated_matmul_f8(&ca, &cg, &cu, gate_bias, up_bias, (int)act, m, n, k, out.data_ptr(), ldo, out_type_of(out),
                             codes ? (float*)scale.data_ptr() : nullptr, codes ? scale.stride(0) : 0, codes ? scale.stride(1) : 0, stream);
  });
  check(rc, "sf_gated_matmul_f8");
  return codes ? pair(given_or(args[10], out), given_or(args[11], scale)) : given_or(args[10], out);
}

// ---- residual rows --------------------------------------------------------------------

// Rows [samples][tokens][dims], or [tokens][dims] for one sample.
struct Rows {
  void* at;
  int64_t sample, token;
};
Rows rows_of(const at::Tensor& t, const char* what) {
  const int64_t d = t.dim();
  if ((d != 2 && d != 3) || t.size(d - 1) < 1 || (t.size(d - 1) > 1 && t.stride(d - 1) != 1))
    bad_value(what, ": expected [samples, tokens, dims] or [tokens, dims] with adjacent dims, got shape ", t.sizes(), ", strides ",
              t.strides());
  return Rows{t.data_ptr(), d == 3 ? t.stride(0) : 0, t.stride(d - 2)};
}
void same_rows(const at::Tensor& t, const char* what, const at::Tensor& h) {
  if (t.sizes() != h.sizes() || t.get_device() != h.get_device())
    bad_value(what, ": expected ", h.sizes(), " on ", h.device(), ", got ", t.sizes(), " on ", t.device());
}
// A vector of every sample, or one for all.
const float* per_sample(PyObject* o, const char* what, const at::Tensor& h, int64_t samples, int64_t dims, long long* stride) {
  *stride = 0;
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what, kFloats);
  const int64_t d = t.dim();
  if ((d != 1 && d != 2) || t.size(d - 1) != dims || (d == 2 && t.size(0) != samples && t.size(0) != 1) || t.get_device() != h.get_device() ||
      (dims > 1 && t.stride(d - 1) != 1))
    bad_value(what, ": expected [", samples, ", ", dims, "] or [", dims, "] with adjacent dims on ", h.device(), ", got ", t.sizes(),
              ", strides ", t.strides(), " on ", t.device());
  if (d == 2 && t.size(0) > 1) *stride = t.stride(0);
  return (const float*)t.data_ptr();
}

// h, y, gate | None, post, post_gain | None, residual_scale, pre (-1: no second output), pre_gain | None,
// scale | None, shift | None, eps, type, h_out | None, out | None, out_scale | None -> (h_out, out | (out, out_scale) | None)
PyObject* residual_norm(PyObject* const* args) {
  const at::Tensor& h = tensor(args[0], "h", kReals);
  const at::Tensor& y = tensor(args[1], "y", kReals);
  const Rows hr = rows_of(h, "h"), yr = rows_of(y, "y");
  same_rows(y, "y", h);
  const int64_t dim = h.dim(), samples = dim == 3 ? h.size(0) : 1, tokens = h.size(dim - 2), dims = h.size(dim - 1);
  const int device = h.get_device();
  sf_block_rows r{};
  r.samples = as_int(samples, "h");
  r.tokens = as_int(tokens, "h");
  r.dims = as_int(dims, "h");
  r.h = hr.at;
  r.h_type = type_of(h);
  r.h_sample = hr.sample;
  r.h_token = hr.token;
  r.y = yr.at;
  r.y_type = type_of(y);
  r.y_sample = yr.sample;
  r.y_token = yr.token;
  r.gate = per_sample(args[2], "gate", h, samples, dims, &r.gate_sample);
  r.post = (int)long_of(args[3]);
  r.post_gain = vector(args[4], "post_gain", dims, device, true);
  r.residual_scale = float_of(args[5]);
  const long pre = long_of(args[6]);
  const bool two = pre >= 0;
  r.pre = (int)pre;
  r.pre_gain = vector(args[7], "pre_gain", dims, device, true);
  r.scale = per_sample(args[8], "scale", h, samples, dims, &r.scale_sample);
  r.shift = per_sample(args[9], "shift", h, samples, dims, &r.shift_sample);
  r.eps = float_of(args[10]);
  const long type = long_of(args[11]);
  at::Tensor h_out, out, scale;
  if (args[12] != Py_None) {
    h_out = tensor(args[12], "h_out", {h.scalar_type()});
    same_rows(h_out, "h_out", h);
    rows_of(h_out, "h_out");
  }
  if (!two)
    for (const int i : {7, 8, 9, 13, 14})
      if (args[i] != Py_None) bad_value("pre_gain, scale, shift, out and out_scale: only with pre");
  if (args[13] != Py_None) {
    const bool is = THPVariable_Check(args[13]) && is_codes(THPVariable_Unpack(args[13]));
    out = is ? tensor(args[13], "out", kF8Codes) : tensor(args[13], "out", kReals);
    same_rows(out, "out", h);
    const Rows o = rows_of(out, "out");
    if (is && ((tokens > 1 && o.token % 16) || (samples > 1 && o.sample % 16) || (uintptr_t)o.at % 16))
      bad_value("out: rows of codes have to start at multiples of 16 bytes (strides ", out.strides(), ")");
  }
  const bool codes = two && (out.defined() ? is_codes(out) : type == SF_TYPE_F8);
  if (args[14] != Py_None) {
    if (!codes) bad_value("out_scale: only with outputs that are codes");
    scale = tensor(args[14], "out_scale", kFloats);
    if (scale.dim() != dim || scale.get_device() != device || (dim == 3 && scale.size(0) != samples) || scale.size(dim - 2) != tokens ||
        scale.size(dim - 1) != blocks_of(dims))
      bad_value("out_scale: expected one value per row and ", SF_F8_BLOCK, " dims on ", h.device(), ", got ", scale.sizes(), " on ", scale.device());
  }
  void* const stream = stream_of(device);
  const c10::DeviceGuard guard(h.device());
  const int rc = unlocked([&] {
    if (!h_out.defined()) h_out = at::empty(h.sizes(), h.options());
    const Rows ho = rows_of(h_out, "h_out");
    r.h_out = ho.at;
    r.h_out_sample = ho.sample;
    r.h_out_token = ho.token;
    if (two) {
      if (!out.defined()) {
        if (codes) {
          const int64_t ld = codes_pitch(dims);
          out = dim == 3 ? at::empty({samples, tokens, ld}, h.options().dtype(at::kFloat8_e4m3fn))
                         : at::empty({tokens, ld}, h.options().dtype(at::kFloat8_e4m3fn));
          if (ld != dims) out = out.narrow(dim - 1, 0, dims);
        } else {
          out = at::empty(h.sizes(), h.options().dtype(scalar_of(type)));
        }
      }
      if (codes && !scale.defined()) {
        const int64_t blocks = blocks_of(dims);
        scale = dim == 3 ? at::empty_strided({samples, tokens, blocks}, {tokens, 1, samples * tokens}, h.options().dtype(at::kFloat))
                         : new_scales(tokens, blocks, h);
      }
      const Rows o = rows_of(out, "out");
      r.out = o.at;
      r.out_type = out_type_of(out);
      r.out_sample = o.sample;
      r.out_token = o.token;
      if (codes) {
        r.out_scale = (float*)scale.data_ptr();
        r.out_scale_sample = dim == 3 ? scale.stride(0) : 0;
        r.out_scale_token = scale.stride(dim - 2);
        r.out_scale_block = scale.stride(dim - 1);
      }
    }
    return g_residual_norm(&r, stream);
  });
  check(rc, "sf_residual_norm");
  PyObject* const second = !two ? Py_NewRef(Py_None)
                           : codes ? pair(given_or(args[13], out), given_or(args[14], scale))
                                   : given_or(args[13], out);
  return pair(given_or(args[12], h_out), second);
}

template <int N>
void addresses(PyObject* const* args, void* (&at)[N]) {
  for (int i = 0; i < N; ++i) {
    at[i] = PyLong_AsVoidPtr(args[i]);
    if (!at[i] && PyErr_Occurred()) throw Raised{};
  }
}

// check, raw_stream and the addresses of the first four entry points
PyObject* bind(PyObject* const* args) {
  void* at[4];
  addresses(args + 2, at);
  g_quantize_rows = (decltype(g_quantize_rows))at[0];
  g_matmul_i8 = (decltype(g_matmul_i8))at[1];
  g_rotate = (decltype(g_rotate))at[2];
  g_qk_norm_rotate = (decltype(g_qk_norm_rotate))at[3];
  g_check = Py_NewRef(args[0]);
  g_raw_stream = Py_NewRef(args[1]);
  return Py_NewRef(Py_None);
}

// The addresses of those in 8-bit floating point, after bind().
PyObject* bind_f8(PyObject* const* args) {
  void* at[4];
  addresses(args, at);
  g_quantize_f8 = (decltype(g_quantize_f8))at[0];
  g_matmul_f8 = (decltype(g_matmul_f8))at[1];
  g_gated_matmul_f8 = (decltype(g_gated_matmul_f8))at[2];
  g_residual_norm = (decltype(g_residual_norm))at[3];
  return Py_NewRef(Py_None);
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N || (F != bind && !g_check)) {
    PyErr_Format(PyExc_TypeError, n != N ? "expected %d arguments" : "not bound", N);
    return nullptr;
  }
  t_elsewhere = nullptr;
  try {
    return F(args);
  } catch (const Refused& e) {
    PyErr_SetString(e.type, e.what.c_str());
  } catch (const Raised&) {
  }
  return nullptr;
  END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {{"bind", (PyCFunction)(void (*)(void))call<bind, 6>, METH_FASTCALL, nullptr},
                          {"bind_f8", (PyCFunction)(void (*)(void))call<bind_f8, 4>, METH_FASTCALL, nullptr},
                          {"quantize_rows", (PyCFunction)(void (*)(void))call<quantize_rows, 3>, METH_FASTCALL, nullptr},
                          {"matmul_i8", (PyCFunction)(void (*)(void))call<matmul_i8, 7>, METH_FASTCALL, nullptr},
                          {"rotate", (PyCFunction)(void (*)(void))call<rotate, 5>, METH_FASTCALL, nullptr},
                          {"qk_norm_rotate", (PyCFunction)(void (*)(void))call<qk_norm_rotate, 9>, METH_FASTCALL, nullptr},
                          {"quantize_f8", (PyCFunction)(void (*)(void))call<quantize_f8, 4>, METH_FASTCALL, nullptr},
                          {"matmul_f8", (PyCFunction)(void (*)(void))call<matmul_f8, 7>, METH_FASTCALL, nullptr},
                          {"gated_matmul_f8", (PyCFunction)(void (*)(void))call<gated_matmul_f8, 12>, METH_FASTCALL, nullptr},
                          {"residual_norm", (PyCFunction)(void (*)(void))call<residual_norm, 15>, METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&kModule); }
