// Python binding of the operators around the decision step: torch tensors in,
// the C ABI of asymspec_step.h on the caller's stream, torch tensors out.
//
// These calls take 3 to 10 us on the device, and a serving loop issues a handful
// of them a step, so what the host does around a launch is what they cost.  A
// dozen tensors checked one attribute at a time from Python take longer than the
// kernel (16 to 18 us a call); here a call is bound by its launch and its outputs'
// allocation.  step.py holds the Python signatures and their documentation.

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <hip/hip_runtime_api.h>

#include <string>

#include "asymspec_step.h"
#include "span.h"

namespace {

using at::Tensor;

PyObject* g_error = nullptr;      // AsymSpecError

// What a call refuses: a Python exception of `type`.
struct Refused {
  PyObject* type;
  std::string what;
};
struct Raised {};                 // a Python exception is set

[[noreturn]] void refuse(std::string what, PyObject* type = PyExc_ValueError) { throw Refused{type, std::move(what)}; }

void check(int status) {
  if (status == ASYMSPEC_OK) return;
  PyObject* e = PyObject_CallFunction(g_error, "is", status, asymspec_status_string(status));
  if (e != nullptr) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Raised{};
}

std::string text(at::ScalarType t) {
  switch (t) {
    case at::kInt: return "int32";
    case at::kLong: return "int64";
    case at::kFloat: return "float32";
    case at::kBFloat16: return "bfloat16";
    default: return c10::toString(t);
  }
}
std::string text(at::IntArrayRef s) {
  std::string r = "[";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + "]";
}

// The tensor behind a Python argument; null for None.
const Tensor* tensor(const char* name, PyObject* o) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor", PyExc_TypeError);
  const Tensor& t = THPVariable_Unpack(o);
  // (torch keeps a sign, or that all is zero, beside the memory of such tensors)
  if (t.is_neg() || t._is_zerotensor()) refuse(std::string(name) + " is lazily negated or zero: pass its clone()");
  return &t;
}
const Tensor& given(const char* name, PyObject* o) {
  const Tensor* t = tensor(name, o);
  if (t == nullptr) refuse(std::string(name) + " must be a tensor", PyExc_TypeError);
  return *t;
}

// Address of a tensor that has to be as said; null for none.
void* need(const char* name, const Tensor* t, at::ScalarType type, at::IntArrayRef shape, const at::Device& dev,
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
void writable(const char* name, const Tensor* t) {
  if (t != nullptr && t->requires_grad() && c10::GradMode::is_enabled())
    refuse(std::string(name) + " requires a gradient and would be written to: detach it, or call under torch.no_grad()");
}
// Behind it: a new version, as behind every in-place operation, so that a backward pass
// that saved the tensor says so.  (Inference tensors have no versions.)
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

int logit_type(const Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return ASYMSPEC_BF16;
  if (t.scalar_type() == at::kFloat) return ASYMSPEC_FP32;
  refuse("logits must be bfloat16 or float32, got " + text(t.scalar_type()), PyExc_TypeError);
}

int64_t number(const char* name, PyObject* o, int64_t lo, int64_t hi) {
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

void* stream_of(PyObject* o) {
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
  int64_t shape[5][2];
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
  void is(at::ScalarType t, int64_t d0, int64_t d1 = -1) {
    const int i = said++;
    type[i] = t;
    shape[i][0] = d0;
    shape[i][1] = d1;
    dims[i] = d1 < 0 ? 1 : 2;
    offset[i] = bytes;
    const size_t size = (size_t)d0 * (d1 < 0 ? 1 : (size_t)d1) * c10::elementSize(t);
    bytes += (size + 15) / 16 * 16;
  }
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

// logits, history, lengths, prompt_lengths, draft_tokens, repetition, frequency,
// presence, bias_ids, bias_values, mask, mask_index, id_map, out, stream
PyObject* shape_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 15, [&]() -> PyObject* {
    const Tensor& x = given("logits", a[0]);
    asymspec_shape s{};
    s.dtype = logit_type(x);
    if (x.dim() != 3) refuse("logits must be [B, R, V]");
    const int64_t B = x.size(0), R = x.size(1), V = x.size(2);
    if (B > kMostInt || R > kMostInt || V > kMostInt) check(ASYMSPEC_E_ARG);
    const at::Device dev = x.device();
    const Tensor* given_out = tensor("out", a[13]);
    const Tensor& out = given_out != nullptr ? *given_out : x;
    if (out.scalar_type() != x.scalar_type() || out.sizes() != x.sizes() || out.device() != dev)
      refuse("out must have the logits' shape, dtype and device");
    if (V > 1 && (x.stride(2) != 1 || out.stride(2) != 1)) refuse("rows of logits must be contiguous");
    writable(given_out != nullptr ? "out" : "logits", &out);
    const Tensor *history = tensor("history", a[1]), *lengths = tensor("lengths", a[2]),
                 *prompt = tensor("prompt_lengths", a[3]), *drafts = tensor("draft_tokens", a[4]),
                 *bias_ids = tensor("bias_ids", a[8]), *bias_values = tensor("bias_values", a[9]),
                 *mask = tensor("mask", a[10]), *mask_index = tensor("mask_index", a[11]),
                 *id_map = tensor("id_map", a[12]);
    int64_t L = 0, D = 0, n_bias = 0, n_masks = 0, n_ids = 0;
    if (history != nullptr) {
      if (history->dim() != 2 || lengths == nullptr) refuse("history must be [B, L] with lengths [B]");
      L = history->size(1);
    } else if (lengths != nullptr || prompt != nullptr) {
      refuse("lengths belong to a history");
    }
    if (drafts != nullptr) {
      if (drafts->dim() != 2 || (drafts->size(1) > 1 && drafts->stride(1) != 1))
        refuse("draft_tokens must be [B, D], its rows contiguous");
      D = drafts->size(1);
      s.draft_stride = drafts->stride(0);
      if (D < R - 1) refuse("rows behind R - 1 drafts need as many draft_tokens");
    }
    if ((bias_ids == nullptr) != (bias_values == nullptr)) refuse("bias_ids and bias_values belong together");
    if (bias_ids != nullptr) {
      if (bias_ids->dim() != 2) refuse("bias_ids must be [B, n]");
      n_bias = bias_ids->size(1);
    }
    if ((mask == nullptr) != (mask_index == nullptr)) refuse("mask and mask_index belong together");
    if (mask != nullptr) {
      if (mask->dim() != 2) refuse("mask must be [M, ceil(V / 32)]");
      n_masks = mask->size(0);
    }
    if (id_map != nullptr) n_ids = id_map->numel();
    if (L > kMostInt || D > kMostInt || n_bias > kMostInt || n_masks > kMostInt || n_ids > kMostInt)
      check(ASYMSPEC_E_ARG);
    s.request_stride = x.stride(0);
    s.row_stride = x.stride(1);
    s.out_request_stride = out.stride(0);
    s.out_row_stride = out.stride(1);
    s.history = need_as<int>("history", history, {B, L}, dev);
    s.lengths = need_as<int>("lengths", lengths, {B}, dev);
    s.prompt_lengths = need_as<int>("prompt_lengths", prompt, {B}, dev);
    s.draft_tokens = need_as<int>("draft_tokens", drafts, {B, D}, dev, false);
    s.id_map = need_as<int>("id_map", id_map, {n_ids}, dev);
    s.repetition = need_as<float>("repetition", tensor("repetition", a[5]), {B}, dev);
    s.frequency = need_as<float>("frequency", tensor("frequency", a[6]), {B}, dev);
    s.presence = need_as<float>("presence", tensor("presence", a[7]), {B}, dev);
    s.bias_ids = need_as<int>("bias_ids", bias_ids, {B, n_bias}, dev);
    s.bias_values = need_as<float>("bias_values", bias_values, {B, n_bias}, dev);
    s.mask = (const uint32_t*)need_as<int>("mask", mask, {n_masks, (V + 31) / 32}, dev);
    s.mask_index = need_as<int>("mask_index", mask_index, {B, R}, dev);
    // lists of no entries
    if (L == 0) s.history = s.lengths = s.prompt_lengths = nullptr;
    if (D == 0) s.draft_tokens = nullptr;
    if (n_bias == 0) s.bias_ids = nullptr, s.bias_values = nullptr;
    if (n_masks == 0) s.mask = nullptr, s.mask_index = nullptr;
    // an id map of no entries maps nothing: an address that is aligned, and not read
    static const int32_t kNoIds = 0;
    if (id_map != nullptr && n_ids == 0) s.id_map = &kNoIds;
    s.B = (int)B;
    s.R = (int)R;
    s.V = (int)V;
    s.max_history = (int)L;
    s.D = (int)D;
    s.n_ids = (int)n_ids;
    s.n_bias = (int)n_bias;
    s.n_masks = (int)n_masks;
    s.logits = x.data_ptr();
    s.out = out.data_ptr();
    const OnDevice on(dev);
    check(asymspec_shape_logits(&s, stream_of(a[14])));
    written(out);
    PyObject* r = a[given_out != nullptr ? 13 : 0];
    Py_INCREF(r);
    return r;
  });
}

// N, V, dtype of a draw's logits
struct DrawShape {
  int64_t N, V;
  int type;
  explicit DrawShape(const Tensor& x) : type(logit_type(x)) {
    if (x.dim() != 2 || (x.size(1) > 1 && x.stride(1) != 1)) refuse("logits must be [N, V], its rows contiguous");
    N = x.size(0);
    V = x.size(1);
    if (N > kMostInt || V > kMostInt) check(ASYMSPEC_E_ARG);
  }
  size_t bytes() const {
    const size_t b = asymspec_draw_workspace_size((int)N, (int)V, type);
    if (b == 0) check(ASYMSPEC_E_ARG);
    return b;
  }
};

// logits, temperature, uniforms, out, stream
PyObject* draw_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const Tensor& x = given("logits", a[0]);
    const DrawShape d(x);
    const at::Device dev = x.device();
    const int64_t N = d.N;
    const Tensor &tau = given("temperature", a[1]), &u = given("uniforms", a[2]);
    const float* tp = need_as<float>("temperature", &tau, {N}, dev);
    const float* up = need_as<float>("uniforms", &u, {N}, dev, false);
    Outs out(a[3], 2);
    out.is(at::kInt, N);
    out.is(at::kFloat, N);
    const OnDevice on(dev);
    const size_t bytes = d.bytes();
    // A small workspace shares the outputs' allocation, which lives as long as they
    // do; a large one, which a draw of some time has, is given back at once.
    const bool small = bytes <= (16u << 10);
    void* ws = out.make(dev, small ? bytes : 0);
    Tensor own_ws;
    if (!small) {
      own_ws = at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(dev));
      ws = own_ws.data_ptr();
    }
    int* token = out.ptr<int>("token", 0, dev, false);
    float* prob = out.ptr<float>("q", 1, dev, false);
    check(asymspec_draw_tokens(x.data_ptr(), d.type, (int)N, (int)d.V, x.stride(0), tp, up, u.stride(0), token,
                               out.at[0]->stride(0), prob, out.at[1]->stride(0), ws, bytes, stream_of(a[4])));
    return out.result();
  });
}

// accept_len, next_token, draft_tokens, history, lengths, finished, stop_tokens,
// max_lengths, out, stream
PyObject* commit_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const Tensor &d = given("draft_tokens", a[2]), &h = given("history", a[3]);
    if (d.dim() != 2 || (d.size(1) > 1 && d.stride(1) != 1)) refuse("draft_tokens must be [B, K], its rows contiguous");
    if (h.dim() != 2) refuse("history must be [B, L]");
    const int64_t B = d.size(0), K = d.size(1), L = h.size(1);
    const at::Device dev = h.device();
    const Tensor* stops = tensor("stop_tokens", a[6]);
    const int64_t n_stop = stops != nullptr ? stops->numel() : 0;
    if (B < 1 || B > kMostInt || K > kMostInt || L > kMostInt || n_stop > kMostInt) check(ASYMSPEC_E_ARG);
    const int* acc = need_as<int>("accept_len", &given("accept_len", a[0]), {B}, dev);
    const int* nxt = need_as<int>("next_token", &given("next_token", a[1]), {B}, dev);
    const int* dp = need_as<int>("draft_tokens", &d, {B, K}, dev, false);
    int* hp = need_as<int>("history", &h, {B, L}, dev);
    const int* len = need_as<int>("lengths", &given("lengths", a[4]), {B}, dev);
    const int* fin = need_as<int>("finished", tensor("finished", a[5]), {B}, dev);
    const int* sp = need_as<int>("stop_tokens", stops, {n_stop}, dev);
    const int* most = need_as<int>("max_lengths", tensor("max_lengths", a[7]), {B}, dev);
    Outs out(a[8], 4);
    out.is(at::kInt, B);
    out.is(at::kInt, B);
    out.is(at::kInt, B, K + 1);
    out.is(at::kInt, B);
    const OnDevice on(dev);
    out.make(dev);
    int* lo = out.ptr<int>("out[0]", 0, dev);
    int* fo = out.ptr<int>("out[1]", 1, dev);
    int* to = out.ptr<int>("out[2]", 2, dev);
    int* co = out.ptr<int>("out[3]", 3, dev);
    check(asymspec_commit_tokens(acc, nxt, K > 0 ? dp : nullptr, d.stride(0), hp, (int)L, len, fin,
                                 n_stop > 0 ? sp : nullptr, (int)n_stop, most, (int)B, (int)K, lo, fo, to, co,
                                 stream_of(a[9])));
    written(h);
    return out.result();
  });
}

// lengths, new_tokens, block_table, n_blocks, free_ring, free_state, block_size,
// width (0: none), total (0: none), release, out, stream
PyObject* plan_slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const Tensor &table = given("block_table", a[2]), &ring = given("free_ring", a[4]);
    if (table.dim() != 2 || ring.dim() != 1) refuse("block_table must be [B, max_blocks] and free_ring [pool]");
    const int64_t B = table.size(0), top = table.size(1), N = ring.size(0);
    if (B < 1 || B > kMostInt || top > kMostInt || N > kMostInt) check(ASYMSPEC_E_ARG);
    const int64_t bs = number("block_size", a[6], 1, kMostInt);
    const int64_t width = number("width", a[7], 0, kMostInt), total = number("total", a[8], 0, kMostInt);
    const Tensor* fresh_tokens = tensor("new_tokens", a[1]);
    if ((width == 0) == (total == 0)) refuse("give either width or total");
    if (fresh_tokens == nullptr && width == 0) refuse("total needs new_tokens");
    const at::Device dev = table.device();
    const int* len = need_as<int>("lengths", &given("lengths", a[0]), {B}, dev);
    const int* add = need_as<int>("new_tokens", fresh_tokens, {B}, dev);
    int* tp = need_as<int>("block_table", &table, {B, top}, dev);
    const int* held = need_as<int>("n_blocks", &given("n_blocks", a[3]), {B}, dev);
    int* rp = need_as<int>("free_ring", &ring, {N}, dev);
    const int* state = need_as<int>("free_state", &given("free_state", a[5]), {2}, dev);
    const int* rel = need_as<int>("release", tensor("release", a[9]), {B}, dev);
    Outs out(a[10], width > 0 ? 4 : 5);
    if (width > 0) out.is(at::kLong, B, width);
    else out.is(at::kLong, total);
    out.is(at::kInt, B);
    out.is(at::kInt, B);
    out.is(at::kInt, 2);
    if (width == 0) out.is(at::kInt, B + 1);
    int64_t* slots = nullptr;
    int *is_short = nullptr, *held_out = nullptr, *state_out = nullptr, *starts = nullptr;
    auto addresses = [&]() {
      slots = out.ptr<int64_t>("out[0]", 0, dev);
      is_short = out.ptr<int>("out[1]", 1, dev);
      held_out = out.ptr<int>("out[2]", 2, dev);
      state_out = out.ptr<int>("out[3]", 3, dev);
      if (width == 0) starts = out.ptr<int>("out[4]", 4, dev);
    };
    if (!out.made()) addresses();
    if (asym_step::slots_overlap(len, add, rel, tp, (int)top, held, rp, (int)N, state, (int)B, (int)width, (int)total,
                                 slots, starts, is_short, held_out, state_out))
      refuse("block_table, free_ring and out are written and must overlap no other tensor of the call");
    const OnDevice on(dev);
    out.make(dev);
    if (out.made()) addresses();
    check(asymspec_plan_slots(len, add, rel, tp, (int)top, held, rp, (int)N, state, (int)bs, (int)B, (int)width,
                              (int)total, slots, starts, is_short, held_out, state_out, stream_of(a[11])));
    written(table);
    written(ring);
    return out.result();
  });
}

// the class of the errors that a status becomes
PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error);
  g_error = cls;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"shape_logits", (PyCFunction)(void (*)(void))shape_logits, METH_FASTCALL, nullptr},
    {"draw_tokens", (PyCFunction)(void (*)(void))draw_tokens, METH_FASTCALL, nullptr},
    {"commit_tokens", (PyCFunction)(void (*)(void))commit_tokens, METH_FASTCALL, nullptr},
    {"plan_slots", (PyCFunction)(void (*)(void))plan_slots, METH_FASTCALL, nullptr},
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__step(void) { return PyModule_Create(&module); }
