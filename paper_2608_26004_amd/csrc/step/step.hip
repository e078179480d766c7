// The operators around the decision step (asymspec_step.h): host checks and
// launches.  The kernels stand in shape.h, draw.h, commit.h and slots.h.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cstring>

#include "asymspec_step.h"
#include "commit.h"
#include "draw.h"
#include "shape.h"
#include "slots.h"
#include "span.h"

namespace asym_step {

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Compute units of the current device, or 0 when it is no gfx950.
static int device_cus() {
  static std::atomic<int> cus[64];       // 0: not looked at; -1: not a gfx950
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
    (void)hipGetLastError();
    return 0;
  }
  int n = cus[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    hipDeviceProp_t pr;
    if (hipGetDeviceProperties(&pr, dev) != hipSuccess) {
      (void)hipGetLastError();
      return 0;
    }
    n = std::strncmp(pr.gcnArchName, "gfx950", 6) == 0 ? pr.multiProcessorCount : -1;
    cus[dev].store(n, std::memory_order_relaxed);
  }
  return std::max(n, 0);
}

// A launch has fewer than 2^32 threads.
static bool fits(long long grid, int threads) { return grid <= 0xFFFFFFFFll / threads; }

// Enqueues a kernel of one argument.
template <class Args>
static int launch(void (*kernel)(Args), unsigned grid, int threads, size_t lds, void* stream, Args& args) {
  void* p[] = {&args};
  if (hipLaunchKernel((const void*)kernel, dim3(grid), dim3(threads), p, lds, (hipStream_t)stream) == hipSuccess)
    return ASYMSPEC_OK;
  (void)hipGetLastError();
  return ASYMSPEC_E_DEVICE;
}

// Elements from the first to behind the last of a [B][R][V] tensor, or -1 when a
// stride is negative or the tensor larger than any memory.
static int64_t extent(int64_t B, int64_t R, int64_t V, int64_t sb, int64_t sr) {
  if (sb < 0 || sr < 0) return -1;
  const __int128 n = (__int128)(B - 1) * sb + (__int128)(R - 1) * sr + V;
  return n > ((__int128)1 << 56) ? -1 : (int64_t)n;
}

// Whether its rows lie apart, in one order or the other.
static bool rows_apart(int64_t B, int64_t R, int64_t V, int64_t sb, int64_t sr) {
  const bool request_major = (R == 1 || sr >= V) && (B == 1 || sb >= (R - 1) * sr + V);
  const bool row_major = (B == 1 || sb >= V) && (R == 1 || sr >= (B - 1) * sb + V);
  return request_major || row_major;
}

template <int DT>
static int shape_launch(ShapeArgs& A, unsigned grid, size_t lds, void* st) {
  const bool in_place = A.s.logits == A.s.out, masked = A.s.mask != nullptr;
  auto* kernel = in_place ? (masked ? shape_kernel<DT, true, true> : shape_kernel<DT, true, false>)
                          : (masked ? shape_kernel<DT, false, true> : shape_kernel<DT, false, false>);
  return launch(kernel, grid, kShapeThreads, lds, st, A);
}

template <int DT>
static int draw_launch(DrawArgs& A, void* st) {
  // With a table as many workgroups as are resident at once (two a unit), each with
  // chunks of one row.
  const int wide = std::max(1, 2 * device_cus() / A.N);
  A.C = std::min((A.S + wide - 1) / wide, kTableMost);
  A.P = (A.S + A.C - 1) / A.C;
  int rc;
  if (DT == ASYMSPEC_BF16 && A.C >= kTableChunks) {
    rc = launch(draw_table_kernel, (unsigned)(A.N * A.P), kTableThreads, 0, st, A);
  } else {
    const unsigned grid = (unsigned)(((long long)A.N * A.S + kDrawThreads / 64 - 1) / (kDrawThreads / 64));
    rc = launch(draw_part_kernel<DT>, grid, kDrawThreads, 0, st, A);
  }
  return rc != ASYMSPEC_OK ? rc : launch(draw_pick_kernel<DT>, (unsigned)A.N, 64, 0, st, A);
}

// Workspace of a draw; chunks of a row in *S.  0 for invalid arguments.
static size_t draw_bytes(int N, int V, int dtype, int* S) {
  if (N < 1 || V < 1 || V >= (1 << 30) || (dtype != ASYMSPEC_BF16 && dtype != ASYMSPEC_FP32)) return 0;
  *S = (V + kDrawChunk - 1) / kDrawChunk;
  if (!fits((long long)N * *S + kDrawThreads / 64, 64)) return 0;
  return (size_t)N * *S * sizeof(DrawPart);
}

}  // namespace asym_step

using namespace asym_step;

extern "C" {

int asymspec_shape_logits(const asymspec_shape* shape, void* stream) {
  if (shape == nullptr) return ASYMSPEC_E_ARG;
  ShapeArgs A;
  A.s = *shape;
  asymspec_shape& s = A.s;
  if (s.dtype != ASYMSPEC_BF16 && s.dtype != ASYMSPEC_FP32) return ASYMSPEC_E_ARG;
  if (s.B < 1 || s.R < 1 || s.R > ASYMSPEC_SHAPE_MAX_ROWS || s.V < 1 || s.V >= (1 << 30)) return ASYMSPEC_E_ARG;
  if (s.logits == nullptr || s.out == nullptr) return ASYMSPEC_E_ARG;
  // the row strides of one row, and the request strides of one request, do not matter
  if (s.R == 1) s.row_stride = s.out_row_stride = 0;
  if (s.B == 1) s.request_stride = s.out_request_stride = 0;
  const size_t el = s.dtype == ASYMSPEC_BF16 ? 2 : 4;
  const int64_t n_in = extent(s.B, s.R, s.V, s.request_stride, s.row_stride);
  const int64_t n_out = extent(s.B, s.R, s.V, s.out_request_stride, s.out_row_stride);
  if (n_in < 0 || n_out < 0 || !rows_apart(s.B, s.R, s.V, s.out_request_stride, s.out_row_stride)) return ASYMSPEC_E_ARG;
  if (s.logits == s.out) {
    if (s.request_stride != s.out_request_stride || s.row_stride != s.out_row_stride) return ASYMSPEC_E_ARG;
  } else if ((uintptr_t)s.logits < (uintptr_t)s.out + (uintptr_t)n_out * el &&
             (uintptr_t)s.out < (uintptr_t)s.logits + (uintptr_t)n_in * el) {
    return ASYMSPEC_E_ARG;
  }
  if (s.history != nullptr) {
    if (s.lengths == nullptr || s.max_history < 1 || s.max_history > ASYMSPEC_SHAPE_MAX_HISTORY) return ASYMSPEC_E_ARG;
  } else {
    s.lengths = s.prompt_lengths = nullptr;
    s.max_history = 0;
  }
  if (s.draft_tokens == nullptr) s.D = 0;
  if (s.D < 0 || s.D > kShapeMaxDrafts || (s.D > 0 && s.D < s.R - 1)) return ASYMSPEC_E_ARG;
  if (s.D > 0 && s.B > 1 && (s.draft_stride < 0 || s.draft_stride > (1ll << 40))) return ASYMSPEC_E_ARG;
  if (s.B == 1) s.draft_stride = 0;
  if (s.id_map != nullptr && s.n_ids < 0) return ASYMSPEC_E_ARG;
  if ((s.bias_ids == nullptr) != (s.bias_values == nullptr)) return ASYMSPEC_E_ARG;
  if (s.bias_ids == nullptr) s.n_bias = 0;
  if (s.n_bias < 0 || s.n_bias > ASYMSPEC_SHAPE_MAX_BIAS) return ASYMSPEC_E_ARG;
  if ((s.mask == nullptr) != (s.mask_index == nullptr)) return ASYMSPEC_E_ARG;
  if (s.mask != nullptr && s.n_masks < 0) return ASYMSPEC_E_ARG;
  auto workgroups = [&](int T) { return (long long)s.B * ((s.V + T - 1) / T); };
  if (!fits(workgroups(kShapeMaxTokens), kShapeThreads)) return ASYMSPEC_E_ARG;
  if (!aligned(s.logits, el) || !aligned(s.out, el)) return ASYMSPEC_E_ALIGN;
  for (const void* p : {(const void*)s.history, (const void*)s.lengths, (const void*)s.prompt_lengths,
                        (const void*)s.draft_tokens, (const void*)s.id_map, (const void*)s.repetition,
                        (const void*)s.frequency, (const void*)s.presence, (const void*)s.bias_ids,
                        (const void*)s.bias_values, (const void*)s.mask, (const void*)s.mask_index})
    if (!aligned(p, 4)) return ASYMSPEC_E_ALIGN;
  const int cus = device_cus();
  if (cus == 0) return ASYMSPEC_E_DEVICE;
  // A workgroup's lists cost the same however few tokens it has, and some copy or mask
  // while others list.  So parts grow until a workgroup has enough to do: 20 KB of rows to
  // copy, 40 KB under masks, and what there is where only listed vectors change; but not
  // to two workgroups a unit or fewer.  Copies: 96 x 6 rows of 50257 fp32 tokens 60 us
  // with 24 KB, 65 with 48; 128 x 1 of 151936 bf16 24 with 16 KB, 36 with 8; 16 x 3 of 256000
  // behind 16000 20 with 24 KB (1008 workgroups), 26 with 12 or with 48 (512).  Masks:
  // 128 x 7 rows of 151936 115 us with 56 KB, 131 with 28, 122 with 112.  Neither: 8 x 3 behind
  // 4096 8.9 us with 600 workgroups, 10.0 with 304, 9.6 with 1192.
  const int64_t want = s.logits != s.out ? 20 << 10 : s.mask != nullptr ? 40 << 10 : INT64_MAX;
  int T = kShapeMinTokens;
  while (T < kShapeMaxTokens && ((s.R * T * (int64_t)el < want && workgroups(2 * T) > 2ll * cus) ||
                                 !fits(workgroups(T), kShapeThreads)))
    T *= 2;
  A.lgT = __builtin_ctz((unsigned)T);
  A.parts = (s.V + T - 1) / T;
  const long long grid = workgroups(T);
  const size_t lds = s.dtype == ASYMSPEC_BF16 ? ShapeLds<8>::bytes(T, s.n_bias) : ShapeLds<4>::bytes(T, s.n_bias);
  return s.dtype == ASYMSPEC_BF16 ? shape_launch<ASYMSPEC_BF16>(A, (unsigned)grid, lds, stream)
                                  : shape_launch<ASYMSPEC_FP32>(A, (unsigned)grid, lds, stream);
}

size_t asymspec_draw_workspace_size(int N, int V, int dtype) {
  int S;
  return draw_bytes(N, V, dtype, &S);
}

int asymspec_draw_tokens(const void* logits, int dtype, int N, int V, int64_t row_stride,
                         const float* temperature, const float* uniforms, int64_t uniform_stride,
                         int32_t* token, int64_t token_stride, float* prob, int64_t prob_stride,
                         void* workspace, size_t workspace_bytes, void* stream) {
  DrawArgs A;
  const size_t bytes = draw_bytes(N, V, dtype, &A.S);
  if (bytes == 0) return ASYMSPEC_E_ARG;
  if (logits == nullptr || temperature == nullptr || token == nullptr || workspace == nullptr) return ASYMSPEC_E_ARG;
  const int64_t far = 1ll << 40;
  if (N > 1) {
    if (row_stride < 0 || row_stride > far) return ASYMSPEC_E_ARG;
    if (uniforms != nullptr && (uniform_stride < 0 || uniform_stride > far)) return ASYMSPEC_E_ARG;
    // each row has a place of its own
    if (token_stride < 1 || token_stride > far) return ASYMSPEC_E_ARG;
    if (prob != nullptr && (prob_stride < 1 || prob_stride > far)) return ASYMSPEC_E_ARG;
  }
  if (!aligned(logits, dtype == ASYMSPEC_BF16 ? 2 : 4) || !aligned(temperature, 4) || !aligned(uniforms, 4) ||
      !aligned(token, 4) || !aligned(prob, 4) || !aligned(workspace, 16))
    return ASYMSPEC_E_ALIGN;
  if (workspace_bytes < bytes) return ASYMSPEC_E_WORKSPACE;
  if (device_cus() == 0) return ASYMSPEC_E_DEVICE;
  A.logits = logits;
  A.row_stride = N > 1 ? row_stride : 0;
  A.tau = temperature;
  A.u = uniforms;
  A.u_stride = uniform_stride;
  A.token = token;
  A.token_stride = token_stride;
  A.prob = prob;
  A.prob_stride = prob_stride;
  A.part = (DrawPart*)workspace;
  A.N = N;
  A.V = V;
  return dtype == ASYMSPEC_BF16 ? draw_launch<ASYMSPEC_BF16>(A, stream) : draw_launch<ASYMSPEC_FP32>(A, stream);
}

int asymspec_commit_tokens(const int32_t* accept_len, const int32_t* next_token, const int32_t* draft_tokens,
                           int64_t draft_stride, int32_t* history, int max_history, const int32_t* lengths,
                           const int32_t* finished, const int32_t* stop_tokens, int n_stop,
                           const int32_t* max_lengths, int B, int K, int32_t* lengths_out, int32_t* finished_out,
                           int32_t* tokens_out, int32_t* counts_out, void* stream) {
  if (B < 1 || !fits((long long)B + kCommitPer, 64) || K < 0 || K > 63 || max_history < 1 || n_stop < 0)
    return ASYMSPEC_E_ARG;
  if (accept_len == nullptr || next_token == nullptr || history == nullptr || lengths == nullptr ||
      lengths_out == nullptr || finished_out == nullptr || tokens_out == nullptr || counts_out == nullptr)
    return ASYMSPEC_E_ARG;
  if ((K > 0 && draft_tokens == nullptr) || (n_stop > 0 && stop_tokens == nullptr)) return ASYMSPEC_E_ARG;
  if (K > 0 && B > 1 && (draft_stride < 0 || draft_stride > (1ll << 40))) return ASYMSPEC_E_ARG;
  for (const void* p : {(const void*)accept_len, (const void*)next_token, (const void*)draft_tokens,
                        (const void*)history, (const void*)lengths, (const void*)finished, (const void*)stop_tokens,
                        (const void*)max_lengths, (const void*)lengths_out, (const void*)finished_out,
                        (const void*)tokens_out, (const void*)counts_out})
    if (!aligned(p, 4)) return ASYMSPEC_E_ALIGN;
  if (device_cus() == 0) return ASYMSPEC_E_DEVICE;
  CommitArgs A;
  A.accept_len = accept_len; A.next_token = next_token; A.draft_tokens = draft_tokens;
  A.draft_stride = B > 1 ? draft_stride : 0;
  A.history = history; A.lengths = lengths; A.finished = finished; A.stop_tokens = stop_tokens;
  A.max_lengths = max_lengths; A.lengths_out = lengths_out; A.finished_out = finished_out;
  A.tokens_out = tokens_out; A.counts_out = counts_out;
  A.max_history = max_history; A.n_stop = n_stop; A.B = B; A.K = K;
  return launch(commit_kernel, (unsigned)((B + kCommitPer - 1) / kCommitPer), kCommitThreads, 0, stream, A);
}

int asymspec_plan_slots(const int32_t* lengths, const int32_t* new_tokens, const int32_t* release,
                        int32_t* block_table, int max_blocks, const int32_t* n_blocks, int32_t* free_ring,
                        int ring_size, const int32_t* free_state, int block_size, int B, int width, int total,
                        int64_t* slots, int32_t* starts, int32_t* short_out, int32_t* n_blocks_out,
                        int32_t* free_state_out, void* stream) {
  if (B < 1 || B > ASYMSPEC_SLOTS_MAX_REQUESTS || block_size < 1 || max_blocks < 1 || ring_size < 1 || width < 0)
    return ASYMSPEC_E_ARG;
  if (lengths == nullptr || block_table == nullptr || n_blocks == nullptr || free_ring == nullptr ||
      free_state == nullptr || slots == nullptr || short_out == nullptr || n_blocks_out == nullptr ||
      free_state_out == nullptr)
    return ASYMSPEC_E_ARG;
  if (width == 0 && (total < 1 || new_tokens == nullptr)) return ASYMSPEC_E_ARG;
  if ((long long)B * max_blocks > 0x7FFFFFFFll || (long long)B * width > 0x7FFFFFFFll) return ASYMSPEC_E_ARG;
  // every workgroup reads the state that the call starts from
  if (n_blocks_out == n_blocks || free_state_out == free_state) return ASYMSPEC_E_ARG;
  for (const void* p : {(const void*)lengths, (const void*)new_tokens, (const void*)release, (const void*)block_table,
                        (const void*)n_blocks, (const void*)free_ring, (const void*)free_state, (const void*)starts,
                        (const void*)short_out, (const void*)n_blocks_out, (const void*)free_state_out})
    if (!aligned(p, 4)) return ASYMSPEC_E_ALIGN;
  if (!aligned(slots, 8)) return ASYMSPEC_E_ALIGN;
  const int cus = device_cus();
  if (cus == 0) return ASYMSPEC_E_DEVICE;
  if (slots_overlap(lengths, new_tokens, release, block_table, max_blocks, n_blocks, free_ring, ring_size, free_state, B,
                    width, total, slots, starts, short_out, n_blocks_out, free_state_out))
    return ASYMSPEC_E_ARG;
  SlotsArgs A;
  A.lengths = lengths; A.new_tokens = new_tokens; A.release = release; A.table = block_table;
  A.n_blocks = n_blocks; A.ring = free_ring; A.state = free_state; A.slots = slots; A.starts = starts;
  A.short_out = short_out; A.n_blocks_out = n_blocks_out; A.state_out = free_state_out;
  A.max_blocks = max_blocks; A.ring_size = ring_size; A.block_size = block_size;
  A.B = B; A.width = width; A.total = total;
  const long long places = width > 0 ? (long long)B * width : total;
  // An entry a thread, up to two workgroups per compute unit: the slots, the blocks
  // taken (an eighth of them is plenty) and those given back, which the host does
  // not know: a request that ends gives all it has, so one table in 32.
  const long long entries = places + places / 8 + (long long)B * max_blocks / 32;
  const long long grid = std::min<long long>(entries / kSlotsThreads + 1, 2ll * cus);
  return launch(slots_kernel, (unsigned)grid, kSlotsThreads, (size_t)(4 * (B + 1)) * 4, stream, A);
}

}  // extern "C"
