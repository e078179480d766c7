// The operators of a quantised paged cache (asymspec_cache.h): host checks and
// launches.  The kernels stand in rotate.h, move.h and attend.h.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "../step/launch.h"
#include "../step/span.h"
#include "asymspec_cache.h"
#include "attend.h"
#include "attend_host.h"
#include "move.h"
#include "rotate.h"

namespace asym_cache {

using asym_step::aligned;
using asym_step::device_cus;
using asym_step::launch;
using asym_step::Span;

constexpr int64_t kFar = 1ll << 40;               // of a stride
constexpr long long kMostTokens = (1ll << 31) - 16;
constexpr int kMostHeads = 4096;
constexpr int kUnits = 256;                       // compute units of the chip
constexpr int kMostRuns = ASYMSPEC_ATTEND_COUNTERS / 4;
constexpr size_t kWorkspaceAlign = 16;

static int element(int dtype) { return dtype == ASYMSPEC_BF16 ? 2 : 4; }
static bool typed(int dtype) { return dtype == ASYMSPEC_BF16 || dtype == ASYMSPEC_FP32; }

static bool valid(const asymspec_cache& c) {
  if (c.blocks < 1 || c.heads < 1 || c.heads > kMostHeads || c.block_size < 1 || c.dim < kBlock || c.dim % kBlock != 0 ||
      c.dim > ASYMSPEC_CACHE_MAX_DIM || (c.bits != 8 && c.bits != 4))
    return false;
  return (__int128)c.blocks * c.heads * c.block_size < ((__int128)1 << 31);
}
static int addresses(const asymspec_cache& c) {
  for (const void* p : {c.keys, c.key_scales, c.values, c.value_scales}) {
    if (p == nullptr) return ASYMSPEC_E_ARG;
    if (!aligned(p, 16)) return ASYMSPEC_E_ALIGN;
  }
  return ASYMSPEC_OK;
}
static size_t data_bytes(const asymspec_cache& c) {
  return (size_t)c.blocks * c.heads * c.block_size * (c.dim * c.bits / 8);
}
static size_t scale_bytes(const asymspec_cache& c) { return (size_t)c.blocks * c.heads * c.block_size * (c.dim / kBlock); }

// Strides that are not used become 0; false where one is not valid.
static bool strides(asymspec_heads& x, int B, int R, int heads) {
  if (B == 1) x.request = 0;
  if (R == 1) x.row = 0;
  if (heads == 1) x.head = 0;
  return x.request >= 0 && x.row >= 0 && x.head >= 0 && x.request <= kFar && x.row <= kFar && x.head <= kFar;
}
static Span span(const asymspec_heads& x, int B, int R, int heads, int dim, int el) {
  const int64_t n = (B - 1) * x.request + (R - 1) * x.row + (heads - 1) * x.head + dim;
  return Span(x.at, (size_t)n * el);
}
// Whether no two heads of a tensor share a channel: with the strides in order, each is
// beyond what the smaller ones reach.
static bool apart(const asymspec_heads& x, int B, int R, int heads, int dim) {
  struct Axis { int64_t stride; int64_t n; } axis[3] = {{x.request, B}, {x.row, R}, {x.head, heads}};
  std::sort(axis, axis + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  __int128 reach = dim;
  for (const Axis& a : axis) {
    if (a.n == 1) continue;
    if (a.stride < reach) return false;
    reach += (__int128)a.stride * (a.n - 1);
  }
  return true;
}
static bool same(const asymspec_heads& a, const asymspec_heads& b) {
  return a.at == b.at && a.request == b.request && a.row == b.row && a.head == b.head;
}
static bool meet(const Span& a, const Span& b) { return a.from < b.to && b.from < a.to; }

// Inputs from here on pass the caches by: smaller ones are often still there from the
// kernel that wrote them.  (Rotations of 29 MB 11.4 us with the caches, 13.6 past them;
// of 115 MB 38.5 and 38.2; of 229 MB 83 and 70.  Writes of 59 MB in 4 bits 14.8 and 16.1;
// of 118 MB 30.2 and 27.7.)
constexpr int64_t kOnce = 96 << 20;

template <int DT, bool INTER>
static int rotate_launch(RotateArgs& A, unsigned grid, size_t lds, bool vec, bool once, void* stream) {
  auto* kernel = !vec ? rotate_kernel<DT, INTER, false, false>
                      : once ? rotate_kernel<DT, INTER, true, true> : rotate_kernel<DT, INTER, true, false>;
  return launch(kernel, grid, kRotateThreads, lds, stream, A);
}

template <int DT, int BITS>
static int write_launch(MoveArgs& M, unsigned grid, bool once, void* stream) {
  return launch(once ? write_kernel<DT, BITS, true> : write_kernel<DT, BITS, false>, grid, kMoveThreads, 0, stream, M);
}

// How tokens (of `requests`, each on its own) and heads are shared: as many tokens as a
// workgroup has lanes for, and two heads, or one where that leaves fewer than four
// workgroups to a unit.  Returns the workgroups, or -1 where they are too many.
static long long move_parts(MoveArgs& M, int requests) {
  const uint32_t lanes = (uint32_t)M.c.dim / 8, heads = (uint32_t)M.c.heads;
  M.tile = kMoveThreads / lanes;
  const long long per = ((long long)M.tokens + M.tile - 1) / M.tile, tiles = per * requests;
  M.heads = tiles * heads >= 4ll * kUnits * kMoveHeads ? kMoveHeads : 1;
  const uint32_t groups = (heads + M.heads - 1) / M.heads;
  M.by_lanes = Div(lanes);
  M.by_size = Div((uint32_t)M.c.block_size);
  M.by_groups = Div(groups);
  M.by_tiles = Div((uint32_t)per);
  return tiles < (1ll << 24) && tiles * heads < (1ll << 24) ? tiles * groups : -1;
}

// Where the parts begin: behind the counters, on a line, as they need.
static char* attend_parts(void* workspace) {
  return (char*)(((uintptr_t)workspace + kMostRuns * 4 + kLine - 1) / kLine * kLine);
}

// Row tiles of 16 rows, and the workspace of an attention; 0 for invalid sizes.  sums_at: of
// the sums, behind the parts' beginning.
static size_t attend_sizes(const asymspec_attend& a, AttendArgs* A, int* tiles, size_t* sums_at) {
  const asymspec_cache& c = a.cache;
  if (!valid(c) || !typed(a.dtype)) return 0;
  if (c.dim != 64 && c.dim != 96 && c.dim != 128 && c.dim != 192 && c.dim != 256) return 0;
  if (a.B < 1 || a.B > ASYMSPEC_ATTEND_MAX_REQUESTS || a.R < 1 || a.R > ASYMSPEC_ATTEND_MAX_ROWS) return 0;
  if (a.q_heads < c.heads || a.q_heads % c.heads != 0 || a.q_heads / c.heads > 64) return 0;
  if (a.max_blocks < 1 || (long long)a.max_blocks * c.block_size >= (1ll << 31) - 256) return 0;
  A->group = a.q_heads / c.heads;
  A->rows = a.R * A->group;
  *tiles = A->rows > 16 ? attend_most_tiles(c.bits, a.dtype == ASYMSPEC_BF16, c.dim) : 1;
  A->row_tiles = (A->rows + 16 * *tiles - 1) / (16 * *tiles);
  A->most = a.max_blocks * c.block_size;
  const long long runs = (long long)a.B * c.heads, n = runs * ((A->rows + 15) / 16), per = A->most / kUnit + 2;
  if (n > kMostRuns || n * per >= (1ll << 31)) return 0;
  const long long units = runs * A->row_tiles * per;
  A->workgroups = (int)std::min<long long>(units, kUnits * attend_waves(c.bits, a.dtype == ASYMSPEC_BF16, c.dim, *tiles));
  // With all workgroups that fit, not one a compute unit, codes stream at 5.2 TB/s
  // instead of 4.5; a run's join grows by its parts' bytes, at some 40 a ns.  So the
  // latter where 3.2e-8 us a byte of codes is less than 2.4e-5 us a byte of parts.  (8
  // requests of 16384 positions in 4 bits, two heads: 16 rows 26 us and 20, 32 rows 37
  // and 28; with 8 heads, 12 rows 33 and 42.)
  const double codes = kUnit * 2.0 * (c.dim * c.bits / 8 + c.dim / kBlock);
  const double parts = (A->workgroups - kAttendFew) * 4.0 * std::min(16 * *tiles, A->rows) * c.dim / (double)(runs * A->row_tiles);
  A->few = parts > 0 ? (float)(codes / (750 * parts)) : 1e9f;
  const size_t slots = 2 * (size_t)A->workgroups * 16 * *tiles;
  *sums_at = slots * sizeof(f2);
  return kMostRuns * 4 + (kLine - kWorkspaceAlign) + *sums_at + slots * c.dim * 4;
}

}  // namespace asym_cache

using namespace asym_cache;

extern "C" {

int asymspec_rotate_heads(const asymspec_rotate* rotate, void* stream) {
  if (rotate == nullptr) return ASYMSPEC_E_ARG;
  RotateArgs A;
  A.r = *rotate;
  asymspec_rotate& r = A.r;
  if (!typed(r.dtype) || r.B < 1 || r.R < 1 || r.q_heads < 1 || r.k_heads < 0 || r.q_heads + (long long)r.k_heads > kMostHeads)
    return ASYMSPEC_E_ARG;
  if (r.dim < 2 || r.dim > 1024 || r.n < 1 || r.n > r.dim / 2 || (long long)r.B * r.R >= (1ll << 24)) return ASYMSPEC_E_ARG;
  if (r.q.at == nullptr || r.q_out.at == nullptr || r.positions == nullptr || r.frequencies == nullptr) return ASYMSPEC_E_ARG;
  if (r.k_heads > 0 && (r.k.at == nullptr || r.k_out.at == nullptr)) return ASYMSPEC_E_ARG;
  if (r.k_heads == 0) r.k = r.k_out = asymspec_heads{};
  const int el = element(r.dtype);
  if (!strides(r.q, r.B, r.R, r.q_heads) || !strides(r.q_out, r.B, r.R, r.q_heads) ||
      !strides(r.k, r.B, r.R, std::max(r.k_heads, 1)) || !strides(r.k_out, r.B, r.R, std::max(r.k_heads, 1)))
    return ASYMSPEC_E_ARG;
  if (!apart(r.q_out, r.B, r.R, r.q_heads, r.dim) || (r.k_heads > 0 && !apart(r.k_out, r.B, r.R, r.k_heads, r.dim)))
    return ASYMSPEC_E_ARG;
  {
    const Span q = span(r.q, r.B, r.R, r.q_heads, r.dim, el), qo = span(r.q_out, r.B, r.R, r.q_heads, r.dim, el);
    if (!same(r.q, r.q_out) && meet(q, qo)) return ASYMSPEC_E_ARG;
    if (r.k_heads > 0) {
      const Span k = span(r.k, r.B, r.R, r.k_heads, r.dim, el), ko = span(r.k_out, r.B, r.R, r.k_heads, r.dim, el);
      if (!same(r.k, r.k_out) && meet(k, ko)) return ASYMSPEC_E_ARG;
      // An output and the other's tensors: apart, or (the queries and keys of one
      // projection) beside each other in every request or row of one tensor.
      auto clash = [&](const asymspec_heads& out, int heads, const Span& so, const asymspec_heads& x, int x_heads, const Span& sx) {
        if (!meet(so, sx)) return false;
        const int64_t bytes = (intptr_t)x.at - (intptr_t)out.at, at = bytes / el;
        if (bytes % el != 0) return true;
        auto beside = [at](int64_t width, int64_t x_width, int64_t period) {
          return at >= 0 ? width <= at && at + x_width <= period : x_width <= -at && -at + width <= period;
        };
        const int64_t w = (heads - 1) * out.head + r.dim, xw = (x_heads - 1) * x.head + r.dim;
        if (r.B > 1 && out.request == x.request && beside((r.R - 1) * out.row + w, (r.R - 1) * x.row + xw, out.request))
          return false;
        // (of rows and requests, the nearer ones are the parts of the others)
        if (r.R == 1 || out.row != x.row || (r.B > 1 && out.request != x.request)) return true;
        if (r.B == 1) return !beside(w, xw, out.row);
        const int64_t inner = std::min(out.row, out.request), outer = std::max(out.row, out.request);
        return !(beside(w, xw, inner) && outer >= inner * (out.row < out.request ? r.R : r.B));
      };
      if (clash(r.q_out, r.q_heads, qo, r.k, r.k_heads, k) || clash(r.q_out, r.q_heads, qo, r.k_out, r.k_heads, ko) ||
          clash(r.k_out, r.k_heads, ko, r.q, r.q_heads, q))
        return ASYMSPEC_E_ARG;
    }
    const Span table[] = {Span(r.positions, (size_t)r.B * (r.every_row ? r.R : 1) * 4), Span(r.frequencies, (size_t)r.n * 8)};
    for (const Span& t : table)
      if (meet(qo, t) || (r.k_heads > 0 && meet(span(r.k_out, r.B, r.R, r.k_heads, r.dim, el), t))) return ASYMSPEC_E_ARG;
  }
  for (const void* p : {r.q.at, r.k.at, r.q_out.at, r.k_out.at})
    if (!aligned(p, el)) return ASYMSPEC_E_ALIGN;
  if (!aligned(r.positions, 4) || !aligned(r.frequencies, 8)) return ASYMSPEC_E_ALIGN;
  const int cus = device_cus();
  if (cus == 0) return ASYMSPEC_E_DEVICE;
  A.tokens = (uint32_t)((long long)r.B * r.R);
  const int ve = 16 / el, rest = r.dim - 2 * r.n;
  const bool vec = (r.interleaved ? 2 * r.n : r.n) % ve == 0 && rest % ve == 0;
  const bool copies = !same(r.q, r.q_out) || (r.k_heads > 0 && !same(r.k, r.k_out));
  A.tail = copies ? (uint32_t)(vec ? rest / ve : rest) : 0;
  A.pieces = (uint32_t)(vec ? (r.interleaved ? 2 * r.n : r.n) / ve : r.n) + A.tail;
  // A workgroup has one token, or as many as give a quarter of its threads an angle, as
  // long as a unit has four workgroups.  (16384 tokens of 40 heads of 128 channels: one
  // token 58 us, two 61, four 64.)
  A.T = 1;
  while (A.T < kRotateMostTokens && A.T * r.n < kRotateThreads / 4 && A.tokens > 4u * (uint32_t)cus * (uint32_t)A.T) A.T *= 2;
  A.by_n = Div((uint32_t)r.n);
  A.by_R = Div((uint32_t)r.R);
  A.by_pieces = Div(A.pieces);
  A.by_heads = Div((uint32_t)(r.q_heads + r.k_heads));
  const long long grid = (A.tokens + (long long)A.T - 1) / A.T;
  const size_t lds = (size_t)A.T * r.n * sizeof(float2);
  const bool once = (int64_t)A.tokens * (r.q_heads + r.k_heads) * r.dim * el >= kOnce;
  if (r.dtype == ASYMSPEC_BF16)
    return r.interleaved ? rotate_launch<ASYMSPEC_BF16, true>(A, (unsigned)grid, lds, vec, once, stream)
                         : rotate_launch<ASYMSPEC_BF16, false>(A, (unsigned)grid, lds, vec, once, stream);
  return r.interleaved ? rotate_launch<ASYMSPEC_FP32, true>(A, (unsigned)grid, lds, vec, once, stream)
                       : rotate_launch<ASYMSPEC_FP32, false>(A, (unsigned)grid, lds, vec, once, stream);
}

int asymspec_write_cache(const asymspec_cache* cache, const asymspec_heads* k, const asymspec_heads* v, int dtype,
                         const int64_t* slots, int B, int R, void* stream) {
  if (cache == nullptr || k == nullptr || v == nullptr || slots == nullptr || !typed(dtype)) return ASYMSPEC_E_ARG;
  MoveArgs M{};
  M.c = *cache;
  M.k = *k;
  M.v = *v;
  if (!valid(M.c) || B < 1 || R < 1 || (long long)B * R >= kMostTokens) return ASYMSPEC_E_ARG;
  if (M.k.at == nullptr || M.v.at == nullptr) return ASYMSPEC_E_ARG;
  if (!strides(M.k, B, R, M.c.heads) || !strides(M.v, B, R, M.c.heads)) return ASYMSPEC_E_ARG;
  int rc = addresses(M.c);
  if (rc != ASYMSPEC_OK) return rc;
  if (!aligned(M.k.at, element(dtype)) || !aligned(M.v.at, element(dtype)) || !aligned(slots, 8)) return ASYMSPEC_E_ALIGN;
  const Span s[] = {Span(M.c.keys, data_bytes(M.c)), Span(M.c.key_scales, scale_bytes(M.c)),
                    Span(M.c.values, data_bytes(M.c)), Span(M.c.value_scales, scale_bytes(M.c)),
                    span(M.k, B, R, M.c.heads, M.c.dim, element(dtype)), span(M.v, B, R, M.c.heads, M.c.dim, element(dtype)),
                    Span(slots, (size_t)B * R * 8)};
  if (asym_step::overlap(s, 4, 7)) return ASYMSPEC_E_ARG;
  if (device_cus() == 0) return ASYMSPEC_E_DEVICE;
  M.slots = slots;
  M.tokens = (uint32_t)((long long)B * R);
  M.by_R = Div((uint32_t)R);
  const long long grid = move_parts(M, 1);
  if (grid < 0) return ASYMSPEC_E_ARG;
  const bool four = M.c.bits == 4, once = 2ll * M.tokens * M.c.heads * M.c.dim * element(dtype) >= kOnce;
  if (dtype == ASYMSPEC_BF16)
    return four ? write_launch<ASYMSPEC_BF16, 4>(M, (unsigned)grid, once, stream)
                : write_launch<ASYMSPEC_BF16, 8>(M, (unsigned)grid, once, stream);
  return four ? write_launch<ASYMSPEC_FP32, 4>(M, (unsigned)grid, once, stream)
              : write_launch<ASYMSPEC_FP32, 8>(M, (unsigned)grid, once, stream);
}

int asymspec_read_cache(const asymspec_cache* cache, const int32_t* block_table, int max_blocks, const int32_t* lengths,
                        const int32_t* first, int dtype, int B, int width, void* k, void* v, void* stream) {
  if (cache == nullptr || block_table == nullptr || lengths == nullptr || !typed(dtype)) return ASYMSPEC_E_ARG;
  MoveArgs M{};
  M.c = *cache;
  if (!valid(M.c) || B < 1 || width < 1 || max_blocks < 1 || (k == nullptr && v == nullptr)) return ASYMSPEC_E_ARG;
  if (width >= kMostTokens) return ASYMSPEC_E_ARG;
  int rc = addresses(M.c);
  if (rc != ASYMSPEC_OK) return rc;
  if (!aligned(block_table, 4) || !aligned(lengths, 4) || !aligned(first, 4) || !aligned(k, 16) || !aligned(v, 16))
    return ASYMSPEC_E_ALIGN;
  const size_t out = (size_t)B * width * M.c.heads * M.c.dim * element(dtype);
  const Span s[] = {Span(k, k != nullptr ? out : 0), Span(v, v != nullptr ? out : 0), Span(M.c.keys, data_bytes(M.c)),
                    Span(M.c.key_scales, scale_bytes(M.c)), Span(M.c.values, data_bytes(M.c)),
                    Span(M.c.value_scales, scale_bytes(M.c)), Span(block_table, (size_t)B * max_blocks * 4),
                    Span(lengths, (size_t)B * 4), Span(first, first != nullptr ? (size_t)B * 4 : 0)};
  if (asym_step::overlap(s, 2, 9)) return ASYMSPEC_E_ARG;
  M.table = block_table;
  M.lengths = lengths;
  M.first = first;
  M.max_blocks = max_blocks;
  M.k.at = k;
  M.v.at = v;
  M.tokens = (uint32_t)width;
  const long long grid = move_parts(M, B);
  if (grid < 0) return ASYMSPEC_E_ARG;
  if (device_cus() == 0) return ASYMSPEC_E_DEVICE;
  auto* kernel = dtype == ASYMSPEC_BF16 ? (M.c.bits == 4 ? read_kernel<ASYMSPEC_BF16, 4> : read_kernel<ASYMSPEC_BF16, 8>)
                                        : (M.c.bits == 4 ? read_kernel<ASYMSPEC_FP32, 4> : read_kernel<ASYMSPEC_FP32, 8>);
  return launch(kernel, (unsigned)grid, kMoveThreads, 0, stream, M);
}

size_t asymspec_attend_workspace_size(const asymspec_attend* attend) {
  if (attend == nullptr) return 0;
  AttendArgs A;
  int tiles;
  size_t sums_at;
  return attend_sizes(*attend, &A, &tiles, &sums_at);
}

int asymspec_attend_cache(const asymspec_attend* attend, void* workspace, size_t workspace_bytes, void* stream) {
  if (attend == nullptr) return ASYMSPEC_E_ARG;
  AttendArgs A;
  A.a = *attend;
  asymspec_attend& a = A.a;
  int tiles;
  size_t sums_at;
  const size_t bytes = attend_sizes(a, &A, &tiles, &sums_at);
  if (bytes == 0) return ASYMSPEC_E_ARG;
  if (a.q.at == nullptr || a.out == nullptr || a.block_table == nullptr || a.lengths == nullptr || workspace == nullptr)
    return ASYMSPEC_E_ARG;
  if (a.window < 0 || !strides(a.q, a.B, a.R, a.q_heads)) return ASYMSPEC_E_ARG;
  const int rc = addresses(a.cache);
  if (rc != ASYMSPEC_OK) return rc;
  const int el = element(a.dtype);
  if (!aligned(a.q.at, el) || !aligned(a.out, 16) || !aligned(a.lse, 4) || !aligned(a.block_table, 4) ||
      !aligned(a.lengths, 4) || !aligned(a.new_tokens, 4) || !aligned(workspace, kWorkspaceAlign))
    return ASYMSPEC_E_ALIGN;
  if (workspace_bytes < bytes) return ASYMSPEC_E_WORKSPACE;
  const size_t rows = (size_t)a.B * a.R * a.q_heads, b4 = (size_t)a.B * 4;
  const Span s[] = {Span(a.out, rows * a.cache.dim * el), Span(a.lse, a.lse != nullptr ? rows * 4 : 0), Span(workspace, bytes),
                    span(a.q, a.B, a.R, a.q_heads, a.cache.dim, el), Span(a.cache.keys, data_bytes(a.cache)),
                    Span(a.cache.key_scales, scale_bytes(a.cache)), Span(a.cache.values, data_bytes(a.cache)),
                    Span(a.cache.value_scales, scale_bytes(a.cache)), Span(a.block_table, b4 * a.max_blocks),
                    Span(a.lengths, b4), Span(a.new_tokens, a.new_tokens != nullptr ? b4 : 0)};
  if (asym_step::overlap(s, 3, 11)) return ASYMSPEC_E_ARG;
  if (device_cus() == 0) return ASYMSPEC_E_DEVICE;
  A.done = (uint32_t*)workspace;
  A.stats = (f2*)attend_parts(workspace);
  A.sums = (float*)(attend_parts(workspace) + sums_at);
  // (what a row does not see has a score of -infinity, of which 0 times is no number: a scale
  // of 0 is the smallest number there is, 2^-149, and takes scores up to 2^128 below 2^-21)
  A.c = std::fabs(a.scale) * kLog2E;
  uint32_t bits;
  std::memcpy(&bits, &A.c, sizeof(bits));
  if (bits == 0) bits = 1;
  std::memcpy(&A.c, &bits, sizeof(bits));
  A.flip = std::signbit(a.scale) ? (a.dtype == ASYMSPEC_BF16 ? 0x80008000u : 0x80000000u) : 0;
  A.by_size = Div((uint32_t)a.cache.block_size);
  A.by_group = Div((uint32_t)A.group);
  const bool four = a.cache.bits == 4;
  if (a.dtype == ASYMSPEC_BF16)
    return four ? attend_part<4, ASYMSPEC_BF16>(A, tiles, stream) : attend_part<8, ASYMSPEC_BF16>(A, tiles, stream);
  return four ? attend_part<4, ASYMSPEC_FP32>(A, tiles, stream) : attend_part<8, ASYMSPEC_FP32>(A, tiles, stream);
}

}  // extern "C"
