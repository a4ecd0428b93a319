// The operators on torch tensors, as operators.py offers them: shapes, types and devices are
// checked, outputs that are not given allocated, and the library's entry points called on the
// current stream of the tensors' device. In C++, since the smallest calls take 3 us on the GPU and
// their checks in Python took longer: norm and rotation of one token 5.7 us of host time instead of
// 11.0, rows to codes 4.9 instead of 7.8, products 4.4 instead of 8.8; 3.1 of each are the launch and
// 1 to 2 the allocations.
#include <Python.h>

#include <ATen/ATen.h>
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

const at::Tensor& tensor(PyObject* o, const char* what, std::initializer_list<at::ScalarType> types) {
  if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) bad_type(what, ": expected a CUDA tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && c10::GradMode::is_enabled())
    bad_type(what, ": requires grad, and nothing here is differentiated; call under torch.no_grad() or detach it");
  if (t.is_neg()) bad_type(what, ": a lazily negated view, whose memory holds the opposite values; call resolve_neg()");
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

void* stream_of(int device) {
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
PyObject* given_or(PyObject* given, const at::Tensor& made) {
  if (given != Py_None) return Py_NewRef(given);
  return THPVariable_Wrap(made);
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// Row length of codes whose rows start at multiples of 16 bytes.
int64_t pitch_of(const at::Tensor& t, const char* what, int64_t need) {
  if (t.size(1) > 1 && t.stride(1) != 1) bad_value(what, ": expected rows of adjacent codes, got strides ", t.strides());
  const int64_t ld = t.size(0) > 1 ? t.stride(0) : need;
  if (ld % 16 || ld < need || (uintptr_t)t.data_ptr() % 16)
    bad_value(what, ": rows have to start at multiples of 16 bytes, at least ", need, " apart (strides ", t.strides(),
              "); quantize_rows leaves them so");
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
  const c10::DeviceGuard guard(x.device());
  void* const stream = stream_of(device);
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
  const c10::DeviceGuard guard(a.device());
  void* const stream = stream_of(device);
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
  const c10::DeviceGuard guard(x.device());
  void* const stream = stream_of(x.get_device());
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
  const c10::DeviceGuard guard(q.device());
  void* const stream = stream_of(device);
  const int rc = unlocked([&] {
    const sf_heads hq = heads_of(q, q_heads, q_out), hk = k ? heads_of(*k, k_heads, k_out) : sf_heads{};
    return g_qk_norm_rotate(&hq, k ? &hk : nullptr, q_gain, k_gain, (float)eps, type_of(q), rows, tokens, dh, rope, pos.at,
                            pos.row, stream);
  });
  check(rc, "sf_qk_norm_rotate");
  return pair(given_or(args[7], q_out), has_k ? given_or(args[8], k_out) : Py_NewRef(Py_None));
}

// check, raw_stream and the addresses of the four entry points
PyObject* bind(PyObject* const* args) {
  void* at[4];
  for (int i = 0; i < 4; ++i) {
    at[i] = PyLong_AsVoidPtr(args[2 + i]);
    if (!at[i] && PyErr_Occurred()) throw Raised{};
  }
  g_quantize_rows = (decltype(g_quantize_rows))at[0];
  g_matmul_i8 = (decltype(g_matmul_i8))at[1];
  g_rotate = (decltype(g_rotate))at[2];
  g_qk_norm_rotate = (decltype(g_qk_norm_rotate))at[3];
  g_check = Py_NewRef(args[0]);
  g_raw_stream = Py_NewRef(args[1]);
  return Py_NewRef(Py_None);
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N || (F != bind && !g_check)) {
    PyErr_Format(PyExc_TypeError, n != N ? "expected %d arguments" : "not bound", N);
    return nullptr;
  }
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
                          {"quantize_rows", (PyCFunction)(void (*)(void))call<quantize_rows, 3>, METH_FASTCALL, nullptr},
                          {"matmul_i8", (PyCFunction)(void (*)(void))call<matmul_i8, 7>, METH_FASTCALL, nullptr},
                          {"rotate", (PyCFunction)(void (*)(void))call<rotate, 5>, METH_FASTCALL, nullptr},
                          {"qk_norm_rotate", (PyCFunction)(void (*)(void))call<qk_norm_rotate, 9>, METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() { return PyModule_Create(&kModule); }
