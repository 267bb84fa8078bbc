// Python binding of the serving operators (include/wavezip_serve.h): checks of
// torch tensors, outputs, and the calls, for paper_2607_23265_amd/serve.py.
//
// The smallest calls take less time on the GPU (6 us) than a binding in
// Python needed to look at a dozen tensors (12.5 us a call), so that looking is
// done here.  Structs go to and fro as bytes, with the device they lie on.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>

#include <cmath>
#include <cstring>
#include <stdexcept>
#include <string>

#include "wavezip_serve.h"

namespace {

PyObject* wz_error = nullptr;  // the exception that carries a wz_status

struct Refused : std::runtime_error {  // becomes a ValueError
  using std::runtime_error::runtime_error;
};
struct Raised {};  // a Python exception is set already

[[noreturn]] void refuse(const std::string& what) { throw Refused(what); }

// Arguments ------------------------------------------------------------------

const at::Tensor& tensor(const char* name, PyObject* x) {
  if (!THPVariable_Check(x)) refuse(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(x);
}
int64_t integer(const char* name, PyObject* x) {
  const int64_t v = PyLong_AsLongLong(x);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v != int32_t(v)) refuse(std::string(name) + " must fit in 32 bits");
  return v;
}
int32_t count(const char* name, int64_t v) {  // a size, for a field of 32 bits
  if (v > 0x7fffffff) refuse(std::string(name) + " must fit in 32 bits");
  return int32_t(v);
}
int32_t truth(PyObject* x) {
  const int v = PyObject_IsTrue(x);
  if (v < 0) throw Raised{};
  return v;
}
const char* type_name(at::ScalarType t) {
  return t == at::kFloat ? "float32" : t == at::kBFloat16 ? "bfloat16" : t == at::kInt ? "int32"
       : t == at::kChar ? "int8" : t == at::kByte ? "uint8" : "float8_e4m3fn";
}
bool numbers(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }
int32_t code(at::ScalarType t) { return t == at::kFloat ? WZ_F32 : WZ_BF16; }

// A contiguous tensor, on `device` unless that is -1.
const at::Tensor& dense(const char* name, PyObject* x, at::ScalarType type, int device = -1) {
  const at::Tensor& t = tensor(name, x);
  if (!t.is_cuda() || !t.is_contiguous() || t.scalar_type() != type || (device >= 0 && t.get_device() != device))
    refuse(std::string(name) + " must be a contiguous " + type_name(type) + " tensor on " +
           (device < 0 ? "a GPU" : "cuda:" + std::to_string(device)));
  return t;
}
// Row stride of t [tokens, heads, dim], whose heads must lie together (-1: any).
int64_t rows_of(const char* name, const at::Tensor& t, int64_t tokens, int64_t heads, int64_t dim, int device,
                at::ScalarType type) {
  if (t.dim() != 3 || t.size(2) != dim || (heads >= 0 && t.size(1) != heads) || (tokens >= 0 && t.size(0) != tokens) ||
      t.scalar_type() != type || !t.is_cuda() || t.get_device() != device)
    refuse(std::string(name) + " must be [" + (tokens < 0 ? "tokens" : std::to_string(tokens)) + ", " +
           (heads < 0 ? "heads" : std::to_string(heads)) + ", " + std::to_string(dim) + "] on cuda:" +
           std::to_string(device) + ", of type " + type_name(type));
  if (t.stride(2) != 1 || (t.stride(1) != dim && t.size(1) > 1))
    refuse(std::string(name) + ": the heads of a row must lie together");
  return t.size(0) > 1 ? t.stride(0) : t.size(1) * dim;  // (a single row has no stride)
}
// Row stride of a matrix whose rows' elements lie together.
int64_t matrix(const char* name, const at::Tensor& t, bool floats, int device = -1) {
  if (t.dim() != 2 || !(floats ? numbers(t.scalar_type()) : t.scalar_type() == at::kChar) || !t.is_cuda() ||
      (device >= 0 && t.get_device() != device))
    refuse(std::string(name) + " must be a matrix on the GPU of type " + (floats ? "float32 or bfloat16" : "int8"));
  if (t.stride(1) != 1 && t.size(1) > 1) refuse(std::string(name) + ": the elements of a row must lie together");
  return t.size(0) > 1 ? t.stride(0) : t.size(1);
}
bool is(const at::Tensor& t, std::initializer_list<int64_t> shape) { return t.sizes() == at::IntArrayRef(shape); }

at::Tensor empty_on(const at::Tensor& like, at::IntArrayRef shape, at::ScalarType type) {
  return at::empty(shape, like.options().dtype(type).requires_grad(false));
}

// A struct with its kind (several have the same size) and its device, as bytes.
template <typename T>
struct Kind;
template <>
struct Kind<wz_cache> {
  static constexpr const char* name = "PagedCache";
  static constexpr int32_t mark = 0x635a5701;
};
template <>
struct Kind<wz_ragged> {
  static constexpr const char* name = "Ragged";
  static constexpr int32_t mark = 0x725a5702;
};
template <>
struct Kind<wz_rotation> {
  static constexpr const char* name = "Rotation";
  static constexpr int32_t mark = 0x745a5703;
};
template <typename T>
struct On {
  T x;
  int32_t mark, device;
};
template <typename T>
PyObject* pack(const T& x, int device) {
  const On<T> y{x, Kind<T>::mark, device};
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&y), sizeof y);
}
template <typename T>
On<T> unpack(PyObject* x) {
  On<T> y;
  const bool fits = PyBytes_Check(x) && PyBytes_GET_SIZE(x) == Py_ssize_t(sizeof y);
  if (fits) std::memcpy(&y, PyBytes_AS_STRING(x), sizeof y);
  if (!fits || y.mark != Kind<T>::mark) refuse(std::string("a ") + Kind<T>::name + " is expected");
  return y;
}

// Calls f(stream) with `device` current, on its current stream.
template <typename F>
void call(const char* where, int device, F f) {
  const auto index = static_cast<c10::DeviceIndex>(device);
  const c10::DeviceGuard guard(at::Device(at::kCUDA, index));
  const wz_status st = f(static_cast<void*>(c10::hip::getCurrentHIPStream(index).stream()));
  if (st == WZ_OK) return;
  if (PyObject* e = PyObject_CallFunction(wz_error, "is", int(st), where)) {
    PyErr_SetObject(wz_error, e);
    Py_DECREF(e);
  }
  throw Raised{};
}

// No C++ exception passes into the interpreter.
template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F f) {
  if (given != wanted) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", wanted, given);
    return nullptr;
  }
  try {
    return f();
  } catch (const Raised&) {
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// Structs --------------------------------------------------------------------

PyObject* cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 4, [&] {
    const at::Tensor& k = tensor("k", a[0]);
    if (k.dim() != 4) refuse("k must be [pages, kv_heads, page_size, head_dim]");
    const int64_t pages = k.size(0), heads = k.size(1), page = k.size(2), dim = k.size(3);
    dense("k", a[0], at::kFloat8_e4m3fn);
    const int device = k.get_device();
    const at::Tensor& v = dense("v", a[1], at::kFloat8_e4m3fn, device);
    const at::Tensor& ks = dense("k_scale", a[2], at::kFloat, device);
    const at::Tensor& vs = dense("v_scale", a[3], at::kFloat, device);
    if (!is(v, {pages, heads, dim, page})) refuse("v must be [pages, kv_heads, head_dim, page_size]");
    if (!is(ks, {pages, heads}) || !is(vs, {pages, heads})) refuse("k_scale and v_scale must be [pages, kv_heads]");
    return pack(wz_cache{k.data_ptr(), v.data_ptr(), static_cast<float*>(ks.data_ptr()),
                         static_cast<float*>(vs.data_ptr()), count("pages", pages), count("kv_heads", heads),
                         count("page_size", page), count("head_dim", dim)}, device);
  });
}

PyObject* ragged(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const at::Tensor& start = dense("start", a[0], at::kInt);
    const int device = start.get_device();
    const at::Tensor& kv_len = dense("kv_len", a[1], at::kInt, device);
    const at::Tensor& table = dense("table", a[2], at::kInt, device);
    const int64_t batch = kv_len.numel();
    if (kv_len.dim() != 1 || !is(start, {batch + 1}) || table.dim() != 2 || table.size(0) != batch)
      refuse("start must be [batch + 1], kv_len [batch] and table [batch, pages]");
    return pack(wz_ragged{static_cast<const int32_t*>(start.data_ptr()), static_cast<const int32_t*>(kv_len.data_ptr()),
                          static_cast<const int32_t*>(table.data_ptr()), count("batch", batch), 0,
                          int32_t(integer("max_tokens", a[3])), int32_t(integer("max_kv", a[4])),
                          count("table", table.size(1))}, device);
  });
}

// (positions and tokens come with the call)
PyObject* rotation(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 3, [&] {
    const at::Tensor& table = dense("table", a[0], at::kFloat);
    if (!PyTuple_Check(a[1])) refuse("sections must be a tuple");
    const Py_ssize_t sections = PyTuple_GET_SIZE(a[1]);
    if (table.dim() != 2 || sections > 3) refuse("table must be [max_pos, rot_dim], with at most three sections");
    wz_rotation r{static_cast<const float*>(table.data_ptr()), nullptr, count("max_pos", table.size(0)),
                  count("rot_dim", table.size(1)), sections ? int32_t(sections) : 1, truth(a[2]), {0, 0, 0}};
    for (Py_ssize_t i = 0; i < sections; ++i)
      r.sections[i] = int32_t(integer("a section", PyTuple_GET_ITEM(a[1], i)));
    if (sections == 1 && 2 * int64_t(r.sections[0]) != table.size(1)) refuse("the sections must sum to rot_dim / 2");
    return pack(r, table.get_device());
  });
}

// Calls ----------------------------------------------------------------------

// (cache, batch, k, v, rotation, positions, q, q_out) -> q_out or None
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const auto c = unpack<wz_cache>(a[0]);
    auto r = unpack<wz_ragged>(a[1]);
    const int device = c.device;
    const at::Tensor &k = tensor("k", a[2]), &v = tensor("v", a[3]);
    const at::ScalarType type = k.scalar_type();
    if (!numbers(type) || r.device != device)
      refuse("k must be float32 or bfloat16, and the batch on the cache's device");
    const int64_t ks = rows_of("k", k, -1, c.x.kv_heads, c.x.head_dim, device, type), tokens = k.size(0);
    const int64_t vs = rows_of("v", v, tokens, c.x.kv_heads, c.x.head_dim, device, type);
    r.x.tokens = count("tokens", tokens);
    const void* q_at = nullptr;
    int64_t qs = 0, heads = 0, os = 0;
    at::Tensor out;
    if (a[6] != Py_None) {
      const at::Tensor& q = tensor("q", a[6]);
      qs = rows_of("q", q, tokens, -1, c.x.head_dim, device, type), heads = q.size(1), q_at = q.data_ptr();
      out = a[7] == Py_None ? empty_on(q, {tokens, heads, c.x.head_dim}, at::kBFloat16) : tensor("q_out", a[7]);
      os = rows_of("q_out", out, tokens, heads, c.x.head_dim, device, at::kBFloat16);
    }
    On<wz_rotation> turn{};
    const bool turned = a[4] != Py_None;
    if (turned) {
      turn = unpack<wz_rotation>(a[4]);
      if (a[5] == Py_None) refuse("a rotation needs positions");
      const at::Tensor& at_ = dense("positions", a[5], at::kInt, device);
      // (the count alone would take [tokens, axes] and turn by other tokens' positions)
      const int64_t axes = turn.x.axes;
      if (at_.numel() != axes * tokens || !(axes == 1 || at_.dim() == 1 || at_.size(0) == axes) || turn.device != device)
        refuse("positions must be [axes, tokens], on the device of the table");
      turn.x.positions = static_cast<const int32_t*>(at_.data_ptr());
    }
    call("wz_cache_append", device, [&](void* s) {
      return wz_cache_append(&c.x, &r.x, turned ? &turn.x : nullptr, k.data_ptr(), ks, v.data_ptr(), vs, q_at, qs,
                             count("q_heads", heads), out.defined() ? out.data_ptr() : nullptr, os, code(type), s);
    });
    if (!out.defined()) Py_RETURN_NONE;
    return a[7] == Py_None ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[7]);
  });
}

// (cache, batch, q_heads, tokens, window) -> bytes of workspace
PyObject* workspace(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const auto c = unpack<wz_cache>(a[0]);
    auto r = unpack<wz_ragged>(a[1]);
    const int32_t window = int32_t(integer("window", a[4]));
    const wz_attention cfg{int32_t(integer("q_heads", a[2])), window > 0, window, 1.f};
    r.x.tokens = int32_t(integer("tokens", a[3]));
    return PyLong_FromSize_t(wz_attention_workspace_bytes(&c.x, &r.x, &cfg));
  });
}

// (cache, batch, q, scale, causal, window, out, lse, ws) -> out
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const auto c = unpack<wz_cache>(a[0]);
    auto r = unpack<wz_ragged>(a[1]);
    const int device = c.device;
    if (r.device != device) refuse("the batch must be on the cache's device");
    const at::Tensor& q = tensor("q", a[2]);
    const int64_t dim = c.x.head_dim, qs = rows_of("q", q, -1, -1, dim, device, at::kBFloat16);
    const int64_t tokens = q.size(0), heads = q.size(1);
    r.x.tokens = count("tokens", tokens);
    const double scale = a[3] == Py_None ? 1 / std::sqrt(double(dim)) : PyFloat_AsDouble(a[3]);
    if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
    const wz_attention cfg{count("q_heads", heads), truth(a[4]), int32_t(integer("window", a[5])), float(scale)};
    const at::Tensor out = a[6] == Py_None ? empty_on(q, {tokens, heads, dim}, at::kBFloat16) : tensor("out", a[6]);
    const int64_t os = rows_of("out", out, tokens, heads, dim, device, at::kBFloat16);
    float* lse = nullptr;
    if (a[7] != Py_None) {
      const at::Tensor& t = dense("lse", a[7], at::kFloat, device);
      if (!is(t, {tokens, heads})) refuse("lse must be [tokens, q_heads]");
      lse = static_cast<float*>(t.data_ptr());
    }
    at::Tensor ws;
    if (a[8] == Py_None) {
      const size_t need = wz_attention_workspace_bytes(&c.x, &r.x, &cfg);
      if (need) ws = empty_on(q, {int64_t(need)}, at::kByte);
    } else {
      ws = dense("ws", a[8], at::kByte, device);
    }
    call("wz_cache_attention", device, [&](void* s) {
      return wz_cache_attention(&c.x, &r.x, &cfg, q.data_ptr(), qs, out.data_ptr(), os, lse,
                                ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? size_t(ws.numel()) : 0, s);
    });
    return a[6] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(a[6]);
  });
}

// (x, out, scale) -> (out, scale)
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 3, [&]() -> PyObject* {
    const at::Tensor& x = tensor("x", a[0]);
    const int64_t xs = matrix("x", x, true), rows = x.size(0), cols = x.size(1);
    const int device = x.get_device();
    const at::Tensor out = a[1] == Py_None ? empty_on(x, {rows, cols}, at::kChar) : tensor("out", a[1]);
    const at::Tensor scale =
        a[2] == Py_None ? empty_on(x, {rows}, at::kFloat) : dense("scale", a[2], at::kFloat, device);
    const int64_t qs = matrix("out", out, false, device);
    if (!is(out, {rows, cols}) || !is(scale, {rows})) refuse("out must have the shape of x, and scale [rows]");
    call("wz_quantize_rows", device, [&](void* s) {
      return wz_quantize_rows(x.data_ptr(), xs, count("rows", rows), count("cols", cols), code(x.scalar_type()),
                              static_cast<int8_t*>(out.data_ptr()), qs, static_cast<float*>(scale.data_ptr()), s);
    });
    PyObject* const both = PyTuple_New(2);
    if (!both) throw Raised{};
    PyTuple_SET_ITEM(both, 0, a[1] == Py_None ? THPVariable_Wrap(out) : Py_NewRef(a[1]));
    PyTuple_SET_ITEM(both, 1, a[2] == Py_None ? THPVariable_Wrap(scale) : Py_NewRef(a[2]));
    return both;
  });
}

// (a, a_scale, w, w_scale, bias, out, out_dtype) -> out
PyObject* matmul_int(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 7, [&]() -> PyObject* {
    const at::Tensor &x = tensor("a", a[0]), &w = tensor("w", a[2]);
    const int64_t as = matrix("a", x, false);
    const int device = x.get_device();
    const int64_t ws = matrix("w", w, false, device);
    const int64_t M = x.size(0), K = x.size(1), N = w.size(0);
    if (w.size(1) != K) refuse("a and w must have the same columns");
    const at::Tensor &a_scale = dense("a_scale", a[1], at::kFloat, device),
                     &w_scale = dense("w_scale", a[3], at::kFloat, device);
    const float* bias = nullptr;
    bool fits = a_scale.numel() == M && w_scale.numel() == N;
    if (a[4] != Py_None) {
      const at::Tensor& b = dense("bias", a[4], at::kFloat, device);
      fits = fits && b.numel() == N, bias = static_cast<const float*>(b.data_ptr());
    }
    if (!fits) refuse("a_scale must be [M], w_scale and bias [N]");
    at::Tensor out;
    if (a[5] == Py_None) {
      if (!THPDtype_Check(a[6])) refuse("out_dtype must be a dtype");
      const at::ScalarType type = reinterpret_cast<THPDtype*>(a[6])->scalar_type;
      if (!numbers(type)) refuse("out must be [M, N] float32 or bfloat16");
      out = empty_on(x, {M, N}, type);
    } else {
      out = tensor("out", a[5]);
    }
    const int64_t os = matrix("out", out, true, device);
    if (!is(out, {M, N})) refuse("out must be [M, N] float32 or bfloat16");
    call("wz_matmul_int", device, [&](void* s) {
      return wz_matmul_int(static_cast<const int8_t*>(x.data_ptr()), as, static_cast<const float*>(a_scale.data_ptr()),
                           static_cast<const int8_t*>(w.data_ptr()), ws, static_cast<const float*>(w_scale.data_ptr()),
                           bias, count("M", M), count("N", N), count("K", K), out.data_ptr(), os,
                           code(out.scalar_type()), s);
    });
    return a[5] == Py_None ? THPVariable_Wrap(std::move(out)) : Py_NewRef(a[5]);
  });
}

PyObject* raise_as(PyObject*, PyObject* error) {
  Py_XSETREF(wz_error, Py_NewRef(error));
  Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(cache), FAST(ragged), FAST(rotation), FAST(append), FAST(workspace), FAST(attention),
                         FAST(quantize_rows), FAST(matmul_int), {"raise_as", raise_as, METH_O, nullptr}, {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serve", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serve() { return PyModule_Create(&module); }
