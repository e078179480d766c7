// Python binding of the operators around the decision step: torch tensors in,
// the C ABI of asymspec_step.h on the caller's stream, torch tensors out.
//
// These calls take 3 to 10 us on the device, and a serving loop issues a handful
// of them a step, so what the host does around a launch is what they cost.  A
// dozen tensors checked one attribute at a time from Python take longer than the
// kernel (16 to 18 us a call); here a call is bound by its launch and its outputs'
// allocation.  step.py holds the Python signatures and their documentation.

#include "binding.h"

#include "asymspec_step.h"
#include "span.h"

// the functions of cache/bind.cpp, ended by one without a name
extern PyMethodDef asym_cache_methods[];

namespace {

using namespace asym_bind;

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

PyMODINIT_FUNC PyInit__step(void) {
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddFunctions(m, asym_cache_methods) != 0) Py_CLEAR(m);
  return m;
}
