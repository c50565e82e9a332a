// CPython module of the binding's per-call work: argument checks, output tensors, descriptors and the call into libla2.so.
//
// A small call costs what the host takes for it: batch 1, 16 heads, a decode step's kernel runs 3 us and a short prefill's 8 to 14, a
// launch takes the host 3.6, and checks, allocations and marshalling in Python and ctypes took 4 to 9 more (decode 7.8 us a call,
// la2_fwd_state 13.1, la2_fwd with la2_bwd 25.6; from here 5.2, 6.8, 14.2).  Every entry point of the library is
// wrapped by its own type: a pointer takes a tensor (its data), None or a handle, a size also a tensor (its bytes), a descriptor a
// [batch, heads, seqlen, head_dim] tensor or a la2_desc in a buffer.  The interpreter lock is released for the call.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>

#include <cstring>
#include <exception>
#include <tuple>
#include <utility>
#include <vector>

#include "../../include/la2.h"

namespace {

struct Raised {};   // a Python exception has been set

[[noreturn]] void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Raised{};
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "la2: expected a tensor, got %s", Py_TYPE(o)->tp_name);
    throw Raised{};
  }
  return THPVariable_Unpack(o);
}

int32_t dtype_code(const at::Tensor& t) {
  const auto s = t.scalar_type();
  if (s == at::kBFloat16) return LA2_BF16;
  if (s == at::kHalf) return LA2_F16;
  if (s == at::kFloat) return LA2_F32;
  PyErr_Format(PyExc_TypeError, "la2: dtype must be torch.bfloat16, torch.float16 or torch.float32, got %s", c10::toString(s));
  throw Raised{};
}

int32_t extent(int64_t n) {
  if (n > INT32_MAX) raise(PyExc_OverflowError, "la2: an extent of 2^31 or more");
  return (int32_t)n;
}

la2_desc desc_of(const at::Tensor& t) {
  if (t.dim() != 4) raise(PyExc_ValueError, "la2: expected a [batch, heads, seqlen, head_dim] tensor");
  if (t.size(3) > 1 && t.stride(3) != 1) raise(PyExc_ValueError, "la2: the feature dimension must be contiguous");
  la2_desc d{};
  d.batch = extent(t.size(0));
  d.heads = extent(t.size(1));
  d.seqlen = extent(t.size(2));
  d.head_dim = extent(t.size(3));
  d.dtype = dtype_code(t);
  d.stride_b = t.stride(0);
  d.stride_h = t.stride(1);
  d.stride_n = t.stride(2);
  return d;
}

// ---- one argument of an entry point, by its type
template <typename T>
struct Arg;

template <typename T>
struct Arg<T*> {
  T* value;
  explicit Arg(PyObject* o) {
    if (o == Py_None) {
      value = nullptr;
    } else if (PyLong_Check(o)) {
      value = static_cast<T*>(PyLong_AsVoidPtr(o));
      if (PyErr_Occurred()) throw Raised{};
    } else {
      value = static_cast<T*>(tensor(o).data_ptr());
    }
  }
  T* get() const { return value; }
};
template <>
struct Arg<const la2_desc*> {
  la2_desc desc;
  explicit Arg(PyObject* o) {
    if (THPVariable_Check(o)) {
      desc = desc_of(THPVariable_Unpack(o));
      return;
    }
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw Raised{};
    const bool fits = b.len == (Py_ssize_t)sizeof(desc);
    if (fits) std::memcpy(&desc, b.buf, sizeof(desc));
    PyBuffer_Release(&b);
    if (!fits) raise(PyExc_ValueError, "la2: not a la2_desc");
  }
  const la2_desc* get() const { return &desc; }
};
template <typename T>
struct Integer {
  T value;
  explicit Integer(PyObject* o) {
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw Raised{};
    value = (T)x;
    if ((long long)value != x) raise(PyExc_OverflowError, "la2: an integer argument out of range");
  }
  T get() const { return value; }
};
template <>
struct Arg<int32_t> : Integer<int32_t> { using Integer::Integer; };
template <>
struct Arg<int64_t> : Integer<int64_t> { using Integer::Integer; };
template <>
struct Arg<size_t> {
  size_t value;
  explicit Arg(PyObject* o) {
    if (o == Py_None) {
      value = 0;
    } else if (THPVariable_Check(o)) {
      const at::Tensor& t = THPVariable_Unpack(o);
      value = (size_t)t.numel() * t.element_size();
    } else {
      value = PyLong_AsSize_t(o);
      if (PyErr_Occurred()) throw Raised{};
    }
  }
  size_t get() const { return value; }
};
template <>
struct Arg<float> {
  float value;
  explicit Arg(PyObject* o) {   // what float(o) takes
    PyObject* const f = PyNumber_Float(o);
    if (f == nullptr) throw Raised{};
    value = (float)PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
  }
  float get() const { return value; }
};

template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "la2: unknown C++ exception");
  }
  return nullptr;
}

template <auto F>
struct Entry;
template <typename... A, la2_status (*F)(A...)>
struct Entry<F> {
  template <size_t... I>
  static PyObject* run(PyObject* const* args, std::index_sequence<I...>) {
    const std::tuple<Arg<A>...> a{Arg<A>(args[I])...};
    la2_status st;
    Py_BEGIN_ALLOW_THREADS
    st = F(std::get<I>(a).get()...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
  }
  static PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
      if (n != (Py_ssize_t)sizeof...(A)) {
        PyErr_Format(PyExc_TypeError, "la2: %zd arguments, not %zd", (Py_ssize_t)sizeof...(A), n);
        throw Raised{};
      }
      return run(args, std::index_sequence_for<A...>{});
    });
  }
};

// ---- checks and tensors
// same_layout(ref, ...): ValueError unless all have ref's shape, strides, dtype and device
PyObject* same_layout(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n < 1) raise(PyExc_TypeError, "la2: no tensor");
    const at::Tensor& ref = tensor(args[0]);
    for (Py_ssize_t i = 1; i < n; i++) {
      const at::Tensor& o = tensor(args[i]);
      if (o.sizes() != ref.sizes() || o.strides() != ref.strides() || o.scalar_type() != ref.scalar_type() || o.device() != ref.device())
        raise(PyExc_ValueError, "la2: all sequence tensors must share shape, strides, dtype and device");
    }
    Py_RETURN_NONE;
  });
}

// The Python functions hand these arguments on as they are, and an entry point also takes a number for a pointer: the caller's own
// number is refused here, before it can become an address on the device.
void tensor_or_none(PyObject* o) {
  if (o != Py_None) tensor(o);
}

// given(lam, ...): TypeError unless lam is a tensor and every other one a tensor or None
PyObject* given(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n < 1) raise(PyExc_TypeError, "la2: no decay");
    tensor(args[0]);
    for (Py_ssize_t i = 1; i < n; i++) tensor_or_none(args[i]);
    Py_RETURN_NONE;
  });
}

// like(t): an uninitialised tensor of t's shape, strides, dtype and device
PyObject* like(PyObject*, PyObject* arg) {
  return guarded([&] {
    const at::Tensor& t = tensor(arg);
    return THPVariable_Wrap(at::empty_strided(t.sizes(), t.strides(), at::TensorOptions().dtype(t.dtype()).device(t.device())));
  });
}

// f32(t, extent, ...): an uninitialised fp32 tensor of these extents on t's device
PyObject* f32(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&] {
    int64_t size[8];
    if (n < 1 || n > 9) raise(PyExc_TypeError, "la2: one to eight extents");
    for (Py_ssize_t i = 1; i < n; i++) size[i - 1] = Integer<int64_t>(args[i]).get();
    return THPVariable_Wrap(at::empty(at::IntArrayRef(size, n - 1), at::TensorOptions().dtype(at::kFloat).device(tensor(args[0]).device())));
  });
}

// workspace(t, op): the workspace that la2_workspace_bytes asks for, or None
PyObject* workspace(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 2) raise(PyExc_TypeError, "la2: a tensor and an operation");
    const at::Tensor& t = tensor(args[0]);
    const la2_desc d = desc_of(t);
    const size_t need = la2_workspace_bytes(&d, Integer<int32_t>(args[1]).get());
    if (need == 0) Py_RETURN_NONE;
    return THPVariable_Wrap(at::empty({(int64_t)need}, at::TensorOptions().dtype(at::kByte).device(t.device())));
  });
}

// state(s, t, name[, sequences]): s where it is a dense fp32 [batch, heads, d, d] state of t [batch, heads, n, d] (or
// [sequences, heads, d, d] of a packed t [positions, heads, d]) on t's device; None for None and for a state of no elements
PyObject* state(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 3 && n != 4) raise(PyExc_TypeError, "la2: a state, a tensor, a name and a number of sequences");
    if (args[0] == Py_None) Py_RETURN_NONE;
    const at::Tensor &s = tensor(args[0]), &t = tensor(args[1]);
    const int64_t d = t.size(-1), rows = n == 4 ? Integer<int64_t>(args[3]).get() : t.size(0), heads = t.size(1);
    if (s.scalar_type() != at::kFloat || s.dim() != 4 || s.size(0) != rows || s.size(1) != heads || s.size(2) != d || s.size(3) != d ||
        !s.is_contiguous() || s.device() != t.device()) {
      PyErr_Format(PyExc_ValueError, "%U must be dense fp32 %s on the tensors' device", args[2],
                   n == 4 ? "[sequences, H, d, d]" : "[b, H, d, d]");
      throw Raised{};
    }
    if (s.numel() == 0) Py_RETURN_NONE;
    Py_INCREF(args[0]);
    return args[0];
  });
}

// decode_shape(name, dims, q, k, v, kv[, lam, ...]): checks a decoding call's tensors (dims 3: [b, H, d], 4: [b, H, T, d]; lam and what
// follows as given() does); q's extents and the dtype's code
PyObject* decode_shape(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n < 6) raise(PyExc_TypeError, "la2: name, dims, q, k, v, kv");
    if (n > 6) tensor(args[6]);
    for (Py_ssize_t i = 7; i < n; i++) tensor_or_none(args[i]);
    const int64_t dims = Integer<int64_t>(args[1]).get();
    const at::Tensor& q = tensor(args[2]);
    if (q.dim() != dims) {
      PyErr_Format(PyExc_ValueError, "%U: q must have %d dimensions", args[0], (int)dims);
      throw Raised{};
    }
    for (int i = 2; i < 5; i++) {
      const at::Tensor& x = tensor(args[i]);
      if (x.sizes() != q.sizes() || x.scalar_type() != q.scalar_type() || !x.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%U: q, k, v must be dense %s of one dtype", args[0], dims == 3 ? "[b, H, d]" : "[b, H, T, d]");
        throw Raised{};
      }
    }
    const at::Tensor& kv = tensor(args[5]);
    const int64_t d = q.size(dims - 1);
    if (kv.scalar_type() != at::kFloat || kv.dim() != 4 || kv.size(0) != q.size(0) || kv.size(1) != q.size(1) || kv.size(2) != d ||
        kv.size(3) != d || !kv.is_contiguous()) {
      PyErr_Format(PyExc_ValueError, "%U: kv_state must be dense fp32 [b, H, d, d]", args[0]);
      throw Raised{};
    }
    const int code = dtype_code(q);
    if (dims == 3) return Py_BuildValue("LLLi", (long long)q.size(0), (long long)q.size(1), (long long)d, code);
    return Py_BuildValue("LLLLi", (long long)q.size(0), (long long)q.size(1), (long long)q.size(2), (long long)d, code);
  });
}

// ---- the operators around the recurrence: checks, output tensors and the call.  Each answers with a tuple of outputs, or with the
// status (a number) of a refused call.
struct Rows {   // a tensor as rows of features
  int64_t rows = 1, width = 1, stride = 1;
};
Rows rows_of(const at::Tensor& t, const char* what) {
  Rows r;
  const int64_t dims = t.dim();
  if (dims < 1 || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1)) {
    PyErr_Format(PyExc_ValueError, "la2: %s must have contiguous features", what);
    throw Raised{};
  }
  r.width = t.size(dims - 1);
  r.stride = r.width;
  for (int64_t d = 0; d < dims - 1; d++) r.rows *= t.size(d);
  if (t.numel() == 0) return r;   // no element, no distance
  bool seen = false;   // a dimension of more than one entry, and with it the rows' distance
  int64_t next = 0;    // stride that the dimension in front of those seen has to have
  for (int64_t d = dims - 2; d >= 0; d--) {
    const int64_t n = t.size(d);
    if (n == 1) continue;
    if (!seen) r.stride = t.stride(d);
    else if (t.stride(d) != next) {
      PyErr_Format(PyExc_ValueError, "la2: %s must be rows at one distance", what);
      throw Raised{};
    }
    seen = true;
    next = t.stride(d) * n;
  }
  return r;
}
// The strides that elements lie at: those of dimensions of one entry count for nothing
bool same_strides(const at::Tensor& t, const at::Tensor& ref) {
  if (t.numel() == 0) return true;
  for (int64_t d = 0; d < t.dim(); d++)
    if (t.size(d) > 1 && t.stride(d) != ref.stride(d)) return false;
  return true;
}
void same_rows(const at::Tensor& t, const at::Tensor& ref, const char* what) {
  if (t.sizes() != ref.sizes() || !same_strides(t, ref) || t.scalar_type() != ref.scalar_type() || t.device() != ref.device()) {
    PyErr_Format(PyExc_ValueError, "la2: %s: another shape, layout, dtype or device than expected", what);
    throw Raised{};
  }
}
// o, where it is a contiguous tensor of this type and these sizes on ref's device
const at::Tensor& dense(PyObject* o, const at::Tensor& ref, at::ScalarType type, at::IntArrayRef sizes, const char* what) {
  const at::Tensor& t = tensor(o);
  if (t.sizes() != sizes || t.scalar_type() != type || t.device() != ref.device() || !t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "la2: %s: another shape, dtype or device than expected, or not contiguous", what);
    throw Raised{};
  }
  return t;
}
at::Tensor fresh(at::IntArrayRef sizes, const at::Tensor& ref, at::ScalarType type) {
  return at::empty(sizes, at::TensorOptions().dtype(type).device(ref.device()));
}
at::Tensor as(const at::Tensor& t) { return at::empty_strided(t.sizes(), t.strides(), at::TensorOptions().dtype(t.dtype()).device(t.device())); }
// The caller's tensor (dense() of it), or a new one
at::Tensor dense_or_new(PyObject* o, const at::Tensor& ref, at::ScalarType type, at::IntArrayRef sizes, const char* what) {
  return o == Py_None ? fresh(sizes, ref, type) : dense(o, ref, type, sizes, what);
}
at::Tensor same_or_new(PyObject* o, const at::Tensor& ref, const char* what) {
  if (o == Py_None) return as(ref);
  same_rows(tensor(o), ref, what);
  return tensor(o);
}
// Data of an optional dense vector
template <typename T>
const T* dense_or_null(PyObject* o, const at::Tensor& ref, at::ScalarType type, at::IntArrayRef sizes, const char* what) {
  return o == Py_None ? nullptr : static_cast<const T*>(dense(o, ref, type, sizes, what).data_ptr());
}
// The caller's workspace or a new one of `need` bytes (undefined for none)
at::Tensor workspace_of(PyObject* o, const at::Tensor& ref, size_t need) {
  if (o != Py_None) {
    const at::Tensor& t = tensor(o);
    if (t.device() != ref.device()) raise(PyExc_ValueError, "la2: the workspace is on another device");
    if (!t.is_contiguous()) raise(PyExc_ValueError, "la2: the workspace must be contiguous");   // its bytes are counted from its elements
    return t;
  }
  return need == 0 ? at::Tensor() : fresh({(int64_t)need}, ref, at::kByte);
}
void* data(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
size_t bytes(const at::Tensor& t) { return t.defined() ? (size_t)t.numel() * t.element_size() : 0; }
PyObject* wrap(const at::Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(t);
}
template <typename... T>
PyObject* answer(la2_status st, const T&... t) {
  if (st != LA2_OK) return PyLong_FromLong((long)st);
  PyObject* const out = PyTuple_New(sizeof...(T));
  if (out == nullptr) return nullptr;
  Py_ssize_t i = 0;
  const bool fine = ([&] {
    PyObject* const o = wrap(t);
    if (o == nullptr) return false;
    PyTuple_SET_ITEM(out, i++, o);
    return true;
  }() && ...);
  if (fine) return out;
  Py_DECREF(out);
  return nullptr;
}
// The call without the interpreter lock.  Its arguments are evaluated before the lock is released: what can raise (a pointer of a
// tensor without storage, an extent) raises with the lock held.
template <typename... P, typename... A>
la2_status unlocked(la2_status (*entry)(P...), A... args) {
  static_assert(sizeof...(P) == sizeof...(A), "the entry point's arguments");
  la2_status st;
  Py_BEGIN_ALLOW_THREADS
  st = entry(args...);
  Py_END_ALLOW_THREADS
  return st;
}
bool truth(PyObject* o) {
  const int t = PyObject_IsTrue(o);
  if (t < 0) throw Raised{};
  return t != 0;
}
void expects(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return;
  PyErr_Format(PyExc_TypeError, "la2: %zd arguments, not %zd", want, n);
  throw Raised{};
}

// layer_norm_fwd(x, weight, bias, eps, out, mean, rstd, stream): (y, mean, rstd)
PyObject* layer_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expects(n, 8);
    const at::Tensor& x = tensor(a[0]);
    const Rows r = rows_of(x, "x");
    const int dtype = dtype_code(x);
    const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
    const float* const weight = dense_or_null<float>(a[1], x, at::kFloat, {r.width}, "weight");
    const float* const bias = dense_or_null<float>(a[2], x, at::kFloat, {r.width}, "bias");
    const float eps = Arg<float>(a[3]).get();
    const at::Tensor y = same_or_new(a[4], x, "out"), mean = dense_or_new(a[5], x, at::kFloat, lead, "mean"),
                     rstd = dense_or_new(a[6], x, at::kFloat, lead, "rstd");
    void* const stream = Arg<void*>(a[7]).get();
    return answer(unlocked(la2_layer_norm_fwd, r.rows, extent(r.width), dtype, r.stride, x.data_ptr(), weight, bias, eps, y.data_ptr(),
                           static_cast<float*>(mean.data_ptr()), static_cast<float*>(rstd.data_ptr()), stream),
                  y, mean, rstd);
  });
}

// layer_norm_bwd(dy, x, mean, rstd, weight, want_d_weight, want_d_bias, out, workspace, stream): (dx, d_weight, d_bias)
PyObject* layer_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expects(n, 10);
    const at::Tensor &dy = tensor(a[0]), &x = tensor(a[1]);
    const Rows r = rows_of(x, "x");
    const int dtype = dtype_code(x);
    same_rows(dy, x, "dy");
    const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
    const float* const mean = static_cast<const float*>(dense(a[2], x, at::kFloat, lead, "mean").data_ptr());
    const float* const rstd = static_cast<const float*>(dense(a[3], x, at::kFloat, lead, "rstd").data_ptr());
    const float* const weight = dense_or_null<float>(a[4], x, at::kFloat, {r.width}, "weight");
    at::Tensor dw, db;
    if (truth(a[5])) dw = fresh({r.width}, x, at::kFloat);
    if (truth(a[6])) db = fresh({r.width}, x, at::kFloat);
    const at::Tensor dx = same_or_new(a[7], x, "out");
    const int32_t width = extent(r.width);
    const at::Tensor ws = workspace_of(a[8], x, dw.defined() || db.defined() ? la2_layer_norm_workspace_bytes(r.rows, width, dtype) : 0);
    void* const stream = Arg<void*>(a[9]).get();
    return answer(unlocked(la2_layer_norm_bwd, r.rows, width, dtype, r.stride, x.data_ptr(), dy.data_ptr(), weight, mean, rstd,
                           dx.data_ptr(), static_cast<float*>(data(dw)), static_cast<float*>(data(db)), data(ws), bytes(ws), stream),
                  dx, dw, db);
  });
}

la2_linear_desc linear_desc(const at::Tensor& x, const at::Tensor& w, PyObject* act) {
  la2_linear_desc d{};
  const Rows rx = rows_of(x, "x"), rw = rows_of(w, "w");
  if (w.dim() != 2 || rw.width != rx.width) raise(PyExc_ValueError, "la2: w must be [out_features, in_features] of x's features");
  if (w.scalar_type() != x.scalar_type() || w.device() != x.device()) raise(PyExc_ValueError, "la2: x and w must share dtype and device");
  d.rows = rx.rows;
  d.in_features = extent(rx.width);
  d.out_features = extent(rw.rows);
  d.dtype = dtype_code(x);
  d.act = Integer<int32_t>(act).get();
  d.stride_x = rx.stride;
  d.stride_w = rw.stride;
  return d;
}
void of_output(const at::Tensor& t, const at::Tensor& x, const la2_linear_desc& d, const char* what) {
  if (t.dim() != x.dim() || t.sizes().slice(0, x.dim() - 1) != x.sizes().slice(0, x.dim() - 1) || t.size(x.dim() - 1) != d.out_features ||
      t.scalar_type() != x.scalar_type() || t.device() != x.device()) {
    PyErr_Format(PyExc_ValueError, "la2: %s must be x's rows of out_features, x's dtype and device", what);
    throw Raised{};
  }
}

// linear_fwd(x, w, bias, residual, act, want_pre, out, pre, workspace, stream): (y, pre or None)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expects(n, 10);
    const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
    la2_linear_desc d = linear_desc(x, w, a[4]);
    const float* const bias = dense_or_null<float>(a[2], x, at::kFloat, {d.out_features}, "bias");
    at::Tensor y, pre;
    const void* residual = nullptr;
    if (a[3] != Py_None) {
      of_output(tensor(a[3]), x, d, "residual");
      residual = tensor(a[3]).data_ptr();
      y = same_or_new(a[6], tensor(a[3]), "out");
    } else if (a[6] != Py_None) {
      of_output(tensor(a[6]), x, d, "out");
      y = tensor(a[6]);
    } else {
      at::DimVector sizes(x.sizes().begin(), x.sizes().end());
      sizes[sizes.size() - 1] = d.out_features;
      y = fresh(sizes, x, x.scalar_type());
    }
    d.stride_y = rows_of(y, "out").stride;
    if (a[7] != Py_None || truth(a[5])) pre = same_or_new(a[7], y, "pre");
    const at::Tensor ws = workspace_of(a[8], x, la2_linear_workspace_bytes(&d, LA2_OP_FWD));
    void* const stream = Arg<void*>(a[9]).get();
    return answer(unlocked(la2_linear_fwd, &d, x.data_ptr(), w.data_ptr(), bias, residual, y.data_ptr(), data(pre), data(ws), bytes(ws),
                           stream),
                  y, pre);
  });
}

// linear_bwd(dy, x, w, pre, act, want_dx, want_dw, want_d_bias, workspace, stream): (dx, dw, d_bias), None for what is not wanted
PyObject* linear_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expects(n, 10);
    const at::Tensor &dy = tensor(a[0]), &x = tensor(a[1]), &w = tensor(a[2]);
    la2_linear_desc d = linear_desc(x, w, a[4]);
    of_output(dy, x, d, "dy");
    d.stride_y = rows_of(dy, "dy").stride;
    const void* pre = nullptr;
    if (a[3] != Py_None) {
      same_rows(tensor(a[3]), dy, "pre");
      pre = tensor(a[3]).data_ptr();
    }
    at::Tensor dx, dw, db;
    if (truth(a[5])) dx = as(x);
    if (truth(a[6])) dw = as(w);
    if (truth(a[7])) db = fresh({d.out_features}, x, at::kFloat);
    const at::Tensor ws = workspace_of(a[8], x, la2_linear_workspace_bytes(&d, LA2_OP_BWD));
    void* const stream = Arg<void*>(a[9]).get();
    return answer(unlocked(la2_linear_bwd, &d, x.data_ptr(), w.data_ptr(), pre, dy.data_ptr(), data(dx), data(dw), static_cast<float*>(data(db)),
                           data(ws), bytes(ws), stream),
                  dx, dw, db);
  });
}

// beam_select(logits, scores, finished, eos, workspace, stream): (scores, parent, token, finished)
PyObject* beam_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expects(n, 6);
    const at::Tensor& logits = tensor(a[0]);
    if (logits.dim() != 3) raise(PyExc_ValueError, "la2: logits must be [batch, beams, vocab]");
    const Rows r = rows_of(logits, "logits");
    const int dtype = dtype_code(logits);
    const int32_t batch = extent(logits.size(0)), beams = extent(logits.size(1)), vocab = extent(r.width);
    const at::IntArrayRef lead = logits.sizes().slice(0, 2);
    const float* const scores = static_cast<const float*>(dense(a[1], logits, at::kFloat, lead, "scores").data_ptr());
    const uint8_t* const finished = dense_or_null<uint8_t>(a[2], logits, at::kBool, lead, "finished");
    const int32_t eos = Integer<int32_t>(a[3]).get();
    const at::Tensor ws = workspace_of(a[4], logits, la2_beam_select_workspace_bytes(batch, beams, vocab, dtype));
    const at::Tensor out = fresh(lead, logits, at::kFloat), parent = fresh(lead, logits, at::kInt), token = fresh(lead, logits, at::kInt),
                     done = fresh(lead, logits, at::kBool);
    void* const stream = Arg<void*>(a[5]).get();
    return answer(unlocked(la2_beam_select, batch, beams, vocab, dtype, r.stride, logits.data_ptr(), scores, finished, eos,
                           static_cast<float*>(out.data_ptr()), static_cast<int32_t*>(parent.data_ptr()),
                           static_cast<int32_t*>(token.data_ptr()), static_cast<uint8_t*>(done.data_ptr()), data(ws), bytes(ws), stream),
                  out, parent, token, done);
  });
}

// beam_reorder(states (a sequence of tensors), parent, stream): the status
PyObject* beam_reorder(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    expects(n, 3);
    const at::Tensor& parent = tensor(a[1]);
    if (parent.dim() != 2 || parent.scalar_type() != at::kInt || !parent.is_contiguous())
      raise(PyExc_ValueError, "la2: parent must be contiguous int32 [batch, beams]");
    const int32_t batch = extent(parent.size(0)), beams = extent(parent.size(1));
    PyObject* const seq = PySequence_Fast(a[0], "la2: states must be tensors");
    if (seq == nullptr) throw Raised{};
    struct Release {
      PyObject* o;
      ~Release() { Py_DECREF(o); }
    } release{seq};
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(seq);
    std::vector<void*> at((size_t)count);
    int64_t row = 0;
    for (Py_ssize_t i = 0; i < count; i++) {
      const at::Tensor& s = tensor(PySequence_Fast_GET_ITEM(seq, i));
      if (s.dim() < 1 || s.size(0) != (int64_t)batch * beams || !s.is_contiguous() || s.device() != parent.device())
        raise(PyExc_ValueError, "la2: states must be contiguous, one for each of batch * beams, on parent's device");
      const int64_t size = s.size(0) == 0 ? 0 : s.numel() / s.size(0) * (int64_t)s.element_size();
      if (i > 0 && size != row) raise(PyExc_ValueError, "la2: states must be of one size");
      row = size;
      at[(size_t)i] = s.data_ptr();
    }
    void* const stream = Arg<void*>(a[2]).get();
    const int32_t states = extent(count);
    const int32_t* const from = static_cast<const int32_t*>(parent.data_ptr());
    return PyLong_FromLong((long)unlocked(la2_beam_reorder, states, at.data(), batch, beams, row, from, stream));
  });
}

#define FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
#define ENTRY(f) FAST(#f, (&Entry<f>::call))
PyMethodDef methods[] = {
    ENTRY(la2_fwd), ENTRY(la2_fwd_noalloc), ENTRY(la2_bwd), ENTRY(la2_fwd_state), ENTRY(la2_bwd_saved), ENTRY(la2_fwd_norm),
    ENTRY(la2_bwd_norm), ENTRY(la2_fwd_state_norm), ENTRY(la2_bwd_state_norm), ENTRY(la2_fwd_varlen), ENTRY(la2_bwd_varlen),
    ENTRY(la2_fwd_varlen_state), ENTRY(la2_bwd_varlen_state), ENTRY(la2_fwd_varlen_norm), ENTRY(la2_bwd_varlen_norm),
    ENTRY(la2_decode_step), ENTRY(la2_decode_step_norm), ENTRY(la2_decode_multi), ENTRY(la2_decode_multi_norm),
    ENTRY(la2_left_product_fwd), ENTRY(la2_left_product_bwd),
    FAST("same_layout", same_layout), FAST("given", given), FAST("f32", f32), FAST("workspace", workspace), FAST("state", state),
    FAST("decode_shape", decode_shape), FAST("layer_norm_fwd", layer_norm_fwd), FAST("layer_norm_bwd", layer_norm_bwd),
    FAST("linear_fwd", linear_fwd), FAST("linear_bwd", linear_bwd), FAST("beam_select", beam_select), FAST("beam_reorder", beam_reorder),
    {"like", like, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
#undef ENTRY
#undef FAST

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_la2_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the Python and the torch whose headers this was compiled with; the binding refuses any other (a tensor's layout in memory
// is what the checks above read)
PyMODINIT_FUNC PyInit__la2_native() {
  PyObject* const m = PyModule_Create(&module);
  if (m == nullptr) return nullptr;
  PyObject* const built = Py_BuildValue("(iis)", PY_MAJOR_VERSION, PY_MINOR_VERSION, LA2_TORCH_VERSION);
  if (built == nullptr || PyModule_AddObject(m, "built_for", built) != 0) {
    Py_XDECREF(built);
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
