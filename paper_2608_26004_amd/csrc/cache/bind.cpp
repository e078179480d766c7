// Python binding of the operators of a quantised paged cache: part of _step.so, in the
// manner of step/bind.cpp.  cache.py holds the Python signatures and their
// documentation.

#include "../step/binding.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <map>
#include <tuple>

#include "asymspec_cache.h"

namespace {

using namespace asym_bind;

// A cache's four tensors.
struct Cache {
  asymspec_cache c{};
  const Tensor* t[4];
  explicit Cache(PyObject* o) {
    static const char* names[] = {"keys", "key_scales", "values", "value_scales"};
    if ((!PyTuple_Check(o) && !PyList_Check(o)) || PySequence_Fast_GET_SIZE(o) != 4)
      refuse("cache must be a tuple of tensors (keys, key_scales, values, value_scales)", PyExc_TypeError);
    for (int i = 0; i < 4; ++i) t[i] = &given(names[i], PySequence_Fast_GET_ITEM(o, i));
    const Tensor &data = *t[0], &scales = *t[1];
    if (data.dim() != 4 || scales.dim() != 4) refuse("keys must be [blocks, heads, block_size, dim * bits / 8]");
    const int64_t N = data.size(0), H = data.size(1), S = data.size(2), w = data.size(3), g = scales.size(3);
    if (g < 1 || (w != 32 * g && w != 16 * g))
      refuse("keys have " + std::to_string(w) + " bytes a head and " + std::to_string(g) +
             " scales: 32 bytes a scale are 8 bits, 16 are 4");
    if (N > kMostInt || H > kMostInt || S > kMostInt || g > 8) check(ASYMSPEC_E_ARG);
    const at::Device dev = device();
    void* at[4];
    for (int i = 0; i < 4; ++i) at[i] = need(names[i], t[i], at::kByte, {N, H, S, i % 2 ? g : w}, dev);
    c = asymspec_cache{at[0], at[1], at[2], at[3], (int)N, (int)H, (int)S, (int)(32 * g), w == 32 * g ? 8 : 4};
  }
  at::Device device() const { return t[0]->device(); }
};

// A tensor [B, R, heads, dim] whose heads are contiguous.
asymspec_heads heads_of(const char* name, const Tensor& x, at::IntArrayRef shape, at::ScalarType type,
                        const at::Device& dev) {
  asymspec_heads h{};
  h.at = need(name, &x, type, shape, dev, false);
  const int64_t n = x.dim();
  if (x.size(n - 1) > 1 && x.stride(n - 1) != 1) refuse(std::string(name) + " must have contiguous channels");
  h.request = x.stride(0);
  h.row = n == 4 ? x.stride(1) : 0;
  h.head = x.stride(n - 2);
  return h;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}

void sizes_fit(at::IntArrayRef sizes) {
  for (int64_t s : sizes)
    if (s > kMostInt) check(ASYMSPEC_E_ARG);
}

// q, k, positions, frequencies, interleaved, magnitude, out, stream
PyObject* rotate_heads(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const Tensor& q = given("q", a[0]);
    const Tensor* k = tensor("k", a[1]);
    asymspec_rotate r{};
    r.dtype = logit_type(q, "q");
    if (q.dim() != 4) refuse("q must be [B, R, heads, dim]");
    if (k != nullptr && k->dim() != 4) refuse("k must be [B, R, heads, dim]");
    const at::Device dev = q.device();
    const int64_t B = q.size(0), R = q.size(1), H = q.size(2), D = q.size(3), Hk = k != nullptr ? k->size(2) : 0;
    sizes_fit(q.sizes());
    if (k != nullptr) sizes_fit(k->sizes());
    r.q = heads_of("q", q, q.sizes(), q.scalar_type(), dev);
    if (k != nullptr) r.k = heads_of("k", *k, {B, R, Hk, D}, q.scalar_type(), dev);
    const Tensor &p = given("positions", a[2]), &f = given("frequencies", a[3]);
    if (p.dim() == 2) r.positions = need_as<int>("positions", &p, {B, R}, dev);
    else r.positions = need_as<int>("positions", &p, {B}, dev);
    if (f.dim() != 1) refuse("frequencies must be [n]");
    r.frequencies = need_as<double>("frequencies", &f, {f.size(0)}, dev);
    if (2 * f.size(0) > D) refuse("2n channels of " + std::to_string(f.size(0)) + " frequencies are more than a head has");
    r.every_row = p.dim() == 2;
    r.interleaved = truth(a[4]);
    r.magnitude = (float)real(a[5]);
    r.B = (int)B;
    r.R = (int)R;
    r.q_heads = (int)H;
    r.k_heads = (int)Hk;
    r.dim = (int)D;
    r.n = (int)f.size(0);
    if (k != nullptr && Hk == 0) check(ASYMSPEC_E_ARG);
    if (B < 1 || R < 1 || H < 1 || r.n < 1) check(ASYMSPEC_E_ARG);
    Outs out(a[6], k != nullptr ? 2 : 1);
    out.is(q.scalar_type(), {B, R, H, D});
    if (k != nullptr) out.is(q.scalar_type(), {B, R, Hk, D});
    const OnDevice on(dev);
    out.make(dev);
    r.q_out = heads_of("out[0]", *out.at[0], {B, R, H, D}, q.scalar_type(), dev);
    if (k != nullptr) r.k_out = heads_of("out[1]", *out.at[1], {B, R, Hk, D}, q.scalar_type(), dev);
    check(asymspec_rotate_heads(&r, stream_of(a[7])));
    return out.result();
  });
}

// k, v, slots, cache, stream
PyObject* write_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const Tensor &k = given("k", a[0]), &v = given("v", a[1]), &slots = given("slots", a[2]);
    const Cache cache(a[3]);
    const int type = logit_type(k, "k");
    const at::Device dev = cache.device();
    if (slots.dim() != 1 && slots.dim() != 2) refuse("slots must be [B, R] or [tokens]");
    sizes_fit(slots.sizes());
    const int64_t B = slots.size(0), R = slots.dim() == 2 ? slots.size(1) : 1, H = cache.c.heads, D = cache.c.dim;
    const int64_t four[] = {B, R, H, D}, three[] = {B, H, D};
    const at::IntArrayRef shape = slots.dim() == 2 ? at::IntArrayRef(four, 4) : at::IntArrayRef(three, 3);
    const asymspec_heads kh = heads_of("k", k, shape, k.scalar_type(), dev), vh = heads_of("v", v, shape, k.scalar_type(), dev);
    const int64_t* sp = (const int64_t*)need("slots", &slots, at::kLong, slots.sizes(), dev);
    if (B < 1 || R < 1) check(ASYMSPEC_E_ARG);
    const OnDevice on(dev);
    check(asymspec_write_cache(&cache.c, &kh, &vh, type, sp, (int)B, (int)R, stream_of(a[4])));
    for (const Tensor* t : cache.t) written(*t);
    Py_INCREF(a[3]);
    return a[3];
  });
}

// cache, block_table, lengths, width, first, dtype (ASYMSPEC_BF16 or ASYMSPEC_FP32), out, stream
PyObject* read_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&]() -> PyObject* {
    const Cache cache(a[0]);
    const Tensor& table = given("block_table", a[1]);
    if (table.dim() != 2) refuse("block_table must be [B, max_blocks]");
    sizes_fit(table.sizes());
    const int64_t B = table.size(0), top = table.size(1), H = cache.c.heads, D = cache.c.dim;
    const at::Device dev = cache.device();
    const int* tp = need_as<int>("block_table", &table, {B, top}, dev);
    const int* len = need_as<int>("lengths", &given("lengths", a[2]), {B}, dev);
    const int64_t W = number("width", a[3], 1, kMostInt);
    const int* first = need_as<int>("first", tensor("first", a[4]), {B}, dev);
    const int type = (int)number("dtype", a[5], 0, 1);
    const at::ScalarType st = type == ASYMSPEC_BF16 ? at::kBFloat16 : at::kFloat;
    if (B < 1 || top < 1 || H < 1) check(ASYMSPEC_E_ARG);
    // (ahead of the outputs' allocation)
    const int64_t tile = 2048 / D, tiles = B * ((W + tile - 1) / tile);
    if (tiles >= 1ll << 24 || tiles * H >= 1ll << 24) check(ASYMSPEC_E_ARG);
    Outs out(a[6], 2);
    out.is(st, {B, W, H, D});
    out.is(st, {B, W, H, D});
    const OnDevice on(dev);
    out.make(dev);
    void* kp = out.ptr<char>("out[0]", 0, dev);
    void* vp = out.ptr<char>("out[1]", 1, dev);
    check(asymspec_read_cache(&cache.c, tp, (int)top, len, first, type, (int)B, (int)W, kp, vp, stream_of(a[7])));
    return out.result();
  });
}

// Workspace of an attention on a stream: memory kept for the stream's calls, whose
// counters each of them leaves as it found them, so that a call needs no launch to clear
// them.  A call that is captured has memory of its own, which its replays clear: what
// eager calls work in, a later one may replace.
Tensor attend_workspace(size_t bytes, size_t counters, const at::Device& dev, void* stream) {
  const auto as_bytes = at::TensorOptions().dtype(at::kByte).device(dev);
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing((hipStream_t)stream, &capture) != hipSuccess) {
    (void)hipGetLastError();
    check(ASYMSPEC_E_DEVICE);
  }
  if (capture != hipStreamCaptureStatusNone) {
    Tensor t = at::empty({(int64_t)bytes}, as_bytes);
    t.narrow(0, 0, (int64_t)counters).zero_();
    return t;
  }
  // hipStreamPerThread is one handle for a stream of each host thread, to which the number
  // of the thread belongs.
  static std::atomic<uint64_t> threads{0};
  static thread_local const uint64_t this_thread = ++threads;
  const uint64_t thread = (hipStream_t)stream == hipStreamPerThread ? this_thread : 0;
  // (never destroyed: torch's allocator may be gone before this)
  static auto& kept = *new std::map<std::tuple<int, void*, uint64_t>, Tensor>;
  Tensor& t = kept[{dev.index(), stream, thread}];
  if (!t.defined() || (size_t)t.numel() < bytes) {
    // (torch gives memory that is freed to the next call on the same handle, which may be
    // another thread's while this one's are under way.  So it stays; each is a quarter larger
    // than the one before)
    if (thread != 0 && t.defined()) new Tensor(t);
    t = Tensor();
    t = at::empty({(int64_t)(bytes + bytes / 4)}, as_bytes);
    t.narrow(0, 0, ASYMSPEC_ATTEND_COUNTERS).zero_();
  }
  return t;
}

// q, cache, block_table, lengths, new_tokens, scale, window, return_lse, out, stream
PyObject* attend_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const Tensor& q = given("q", a[0]);
    const Cache cache(a[1]);
    const Tensor& table = given("block_table", a[2]);
    asymspec_attend s{};
    s.cache = cache.c;
    s.dtype = logit_type(q, "q");
    if (q.dim() != 4) refuse("q must be [B, R, heads, dim]");
    if (table.dim() != 2) refuse("block_table must be [B, max_blocks]");
    sizes_fit(q.sizes());
    sizes_fit(table.sizes());
    const at::Device dev = cache.device();
    const int64_t B = q.size(0), R = q.size(1), H = q.size(2), D = cache.c.dim, top = table.size(1);
    s.q = heads_of("q", q, {B, R, H, D}, q.scalar_type(), dev);
    if (cache.c.heads < 1 || H % cache.c.heads != 0)
      refuse(std::to_string(H) + " heads of q are no multiple of the cache's " + std::to_string(cache.c.heads));
    s.block_table = need_as<int>("block_table", &table, {B, top}, dev);
    s.lengths = need_as<int>("lengths", &given("lengths", a[3]), {B}, dev);
    s.new_tokens = need_as<int>("new_tokens", tensor("new_tokens", a[4]), {B}, dev);
    s.scale = a[5] == Py_None ? (float)(1.0 / std::sqrt((double)D)) : (float)real(a[5]);
    s.window = (int)number("window", a[6], 0, kMostInt);
    const bool with_lse = truth(a[7]);
    s.B = (int)B;
    s.R = (int)R;
    s.q_heads = (int)H;
    s.max_blocks = (int)top;
    const size_t bytes = asymspec_attend_workspace_size(&s);
    if (bytes == 0) check(ASYMSPEC_E_ARG);
    // (without lse `out` is a tensor)
    struct Held {
      PyObject* o;
      ~Held() { Py_XDECREF(o); }
    } one{a[8] != Py_None && !with_lse ? PyTuple_Pack(1, a[8]) : nullptr};
    if (one.o == nullptr && PyErr_Occurred()) throw Raised{};
    Outs out(one.o != nullptr ? one.o : a[8], with_lse ? 2 : 1);
    out.is(q.scalar_type(), {B, R, H, D});
    if (with_lse) out.is(at::kFloat, {B, R, H});
    const OnDevice on(dev);
    out.make(dev);
    void* const stream = stream_of(a[9]);
    const size_t runs = (size_t)B * s.cache.heads * ((R * (H / s.cache.heads) + 15) / 16);
    const size_t counters = std::min<size_t>(128 * std::max<size_t>(runs, 2048), ASYMSPEC_ATTEND_COUNTERS);
    const Tensor ws = attend_workspace(bytes, counters, dev, stream);
    s.out = out.ptr<char>("out", 0, dev);
    if (with_lse) s.lse = out.ptr<float>("lse", 1, dev);
    check(asymspec_attend_cache(&s, ws.data_ptr(), (size_t)ws.numel(), stream));
    PyObject* r = out.result();
    if (with_lse) return r;
    PyObject* first = PyTuple_GET_ITEM(r, 0);
    Py_INCREF(first);
    Py_DECREF(r);
    return first;
  });
}

}  // namespace

extern PyMethodDef asym_cache_methods[];
PyMethodDef asym_cache_methods[] = {
    {"rotate_heads", (PyCFunction)(void (*)(void))rotate_heads, METH_FASTCALL, nullptr},
    {"write_cache", (PyCFunction)(void (*)(void))write_cache, METH_FASTCALL, nullptr},
    {"read_cache", (PyCFunction)(void (*)(void))read_cache, METH_FASTCALL, nullptr},
    {"attend_cache", (PyCFunction)(void (*)(void))attend_cache, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
