// What the Python bindings share: checks of torch tensors, outputs, errors.

#ifndef ASYMSPEC_STEP_BINDING_H_
#define ASYMSPEC_STEP_BINDING_H_

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <hip/hip_runtime_api.h>

#include <initializer_list>
#include <string>

#include "asymspec.h"

namespace asym_bind {

using at::Tensor;

inline PyObject* g_error = nullptr;      // AsymSpecError

// What a call refuses: a Python exception of `type`.
struct Refused {
  PyObject* type;
  std::string what;
};
struct Raised {};                 // a Python exception is set

[[noreturn]] inline void refuse(std::string what, PyObject* type = PyExc_ValueError) { throw Refused{type, std::move(what)}; }

inline void check(int status) {
  if (status == ASYMSPEC_OK) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", status, asymspec_status_string(status));
  if (e != nullptr) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Raised{};
}

inline std::string text(at::ScalarType t) {
  switch (t) {
    case at::kInt: return "int32";
    case at::kLong: return "int64";
    case at::kFloat: return "float32";
    case at::kBFloat16: return "bfloat16";
    default: return c10::toString(t);
  }
}
inline std::string text(at::IntArrayRef s) {
  std::string r = "[";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + "]";
}

// The tensor behind a Python argument; null for None.
inline const Tensor* tensor(const char* name, PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor", PyExc_TypeError);
  const Tensor& t = THPVariable_Unpack(o);
  // (torch keeps a sign, or that all is zero, beside the memory of such tensors)
  if (t.is_neg() || t._is_zerotensor()) refuse(std::string(name) + " is lazily negated or zero: pass its clone()");
  return &t;
}
inline const Tensor& given(const char* name, PyObject* o) {
  const Tensor* t = tensor(name, o);
  if (t == nullptr) refuse(std::string(name) + " must be a tensor", PyExc_TypeError);
  return *t;
}

// Address of a tensor that has to be as said; null for none.
inline void* need(const char* name, const Tensor* t, at::ScalarType type, at::IntArrayRef shape, const at::Device& dev,
           bool contiguous = true) {
  if (t == nullptr) return nullptr;
  if (t->scalar_type() != type || t->sizes() != shape || t->device() != dev || !t->has_storage())
    refuse(std::string(name) + " must be " + text(type) + " " + text(shape) + " on " + dev.str() + ", got " +
           text(t->scalar_type()) + " " + text(t->sizes()) + " on " + t->device().str());
  if (contiguous && !t->is_contiguous()) refuse(std::string(name) + " must be contiguous");
  return t->data_ptr();
}
template <class T>
T* need_as(const char* name, const Tensor* t, at::IntArrayRef shape, const at::Device& dev, bool contiguous = true) {
  return (T*)need(name, t, c10::CppTypeToScalarType<T>::value, shape, dev, contiguous);
}

// Ahead of a call that writes a tensor (null: none): nothing of it is recorded, so one
// that requires a gradient would get a wrong one.
inline void writable(const char* name, const Tensor* t) {
  if (t != nullptr && t->requires_grad() && c10::GradMode::is_enabled())
    refuse(std::string(name) + " requires a gradient and would be written to: detach it, or call under torch.no_grad()");
}
// Behind it: a new version, as behind every in-place operation, so that a backward pass
// that saved the tensor says so.  (Inference tensors have no versions.)
inline void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

inline int logit_type(const Tensor& t, const char* name = "logits") {
  if (t.scalar_type() == at::kBFloat16) return ASYMSPEC_BF16;
  if (t.scalar_type() == at::kFloat) return ASYMSPEC_FP32;
  refuse(std::string(name) + " must be bfloat16 or float32, got " + text(t.scalar_type()), PyExc_TypeError);
}

inline int64_t number(const char* name, PyObject* o, int64_t lo, int64_t hi) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v < lo || v > hi)
    refuse(std::string(name) + " must be in [" + std::to_string(lo) + ", " + std::to_string(hi) + "]");
  return v;
}
constexpr int64_t kMostInt = 0x7FFFFFFF;

// The tensors' device current while a call is enqueued.
struct OnDevice {
  int before = -1;
  explicit OnDevice(const at::Device& dev) {
    if (!dev.is_cuda()) refuse("tensors must be on the GPU, got " + dev.str());
    int now = 0;
    if (hipGetDevice(&now) == hipSuccess && now != dev.index()) {
      before = now;
      if (hipSetDevice(dev.index()) != hipSuccess) check(ASYMSPEC_E_DEVICE);
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

inline void* stream_of(PyObject* o) {
  void* s = PyLong_AsVoidPtr(o);
  if (s == nullptr && PyErr_Occurred()) throw Raised{};
  return s;
}

// The outputs of a call: the caller's tensors, or new ones, which share one
// allocation (each costs about as much as the launch's own share).
struct Outs {
  PyObject* tuple;
  Tensor own[5];
  const Tensor* at[5] = {};
  size_t offset[5];
  at::ScalarType type[5];
  int64_t shape[5][4];
  int dims[5];
  int n, said = 0;
  size_t bytes = 0;
  Outs(PyObject* o, int n_) : tuple(o), n(n_) {
    if (o == Py_None) return;
    if (!PyTuple_Check(o) && !PyList_Check(o)) refuse("out must be a tuple of tensors", PyExc_TypeError);
    if (PySequence_Fast_GET_SIZE(o) != n) refuse("out must have " + std::to_string(n) + " tensors");
    for (int i = 0; i < n; ++i) {
      at[i] = &given("out", PySequence_Fast_GET_ITEM(o, i));
      writable("out", at[i]);
    }
  }
  bool made() const { return tuple == Py_None; }
  at::IntArrayRef sizes(int i) const { return at::IntArrayRef(shape[i], dims[i]); }
  // Says the next output: its type and shape.
  void is(at::ScalarType t, std::initializer_list<int64_t> dim) {
    const int i = said++;
    type[i] = t;
    dims[i] = 0;
    offset[i] = bytes;
    size_t size = c10::elementSize(t);
    for (int64_t d : dim) {
      shape[i][dims[i]++] = d;
      size *= (size_t)d;
    }
    bytes += (size + 15) / 16 * 16;
  }
  void is(at::ScalarType t, int64_t d0) { is(t, {d0}); }
  void is(at::ScalarType t, int64_t d0, int64_t d1) { is(t, {d0, d1}); }
  // Makes the new ones, and `extra` bytes behind them, whose address it returns.
  void* make(const at::Device& dev, size_t extra = 0) {
    const size_t all = (made() ? bytes : 0) + extra;
    if (all == 0) return nullptr;
    base = at::empty({(int64_t)all}, at::TensorOptions().dtype(at::kByte).device(dev));
    if (!made()) return base.data_ptr();
    for (int i = 0; i < n; ++i) {
      auto t = c10::make_intrusive<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(),
                                                    c10::scalarTypeToTypeMeta(type[i]));
      t->set_storage_offset((int64_t)(offset[i] / c10::elementSize(type[i])));
      t->set_sizes_contiguous(sizes(i));
      own[i] = Tensor(std::move(t));
      at[i] = &own[i];
    }
    return (char*)base.data_ptr() + bytes;
  }
  // Address of output i, which has to be as said.
  template <class T>
  T* ptr(const char* name, int i, const at::Device& dev, bool contiguous = true) const {
    return (T*)need(name, at[i], type[i], sizes(i), dev, contiguous);
  }
  // (behind the call)
  PyObject* result() {
    if (!made())
      for (int i = 0; i < n; ++i) written(*at[i]);
    PyObject* r = PyTuple_New(n);
    if (r == nullptr) throw Raised{};
    for (int i = 0; i < n; ++i) {
      PyObject* t = made() ? THPVariable_Wrap(std::move(own[i])) : PySequence_Fast_GET_ITEM(tuple, i);
      if (!made()) Py_INCREF(t);
      if (t == nullptr) {
        Py_DECREF(r);
        throw Raised{};
      }
      PyTuple_SET_ITEM(r, i, t);
    }
    return r;
  }

 private:
  Tensor base;
};

// No C++ exception leaves a call.
template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F&& f) {
  try {
    if (n != want) refuse("wrong number of arguments", PyExc_TypeError);
    return f();
  } catch (const Refused& e) {
    PyErr_SetString(e.type, e.what.c_str());
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}

}  // namespace asym_bind

#endif  // ASYMSPEC_STEP_BINDING_H_
