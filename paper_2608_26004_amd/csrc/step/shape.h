// Penalties for repeated tokens, biases and grammar masks on logit rows.
//
// For a row behind a history h and some drafts, a token's logit depends on how
// often the token stands there, on its bias and on its mask bit (the formula
// is in asymspec_step.h).  All of that but the drafts and the mask is the same
// for the R rows of a request, and most tokens have none of it.
//
// One workgroup owns T tokens of one request, in all its rows.  It keeps one
// word per token in LDS (count, prompt flag, draft flag, bias entry), filled by
// integer atomics from the request's lists: integers, so their order does not
// change a result, and no dense table of counts per vocabulary is kept, cleared
// or read.  A token in several lists is then handled once, by one thread, and
// rounded once.
//
// Vectors of VE tokens with a nonzero word are listed.  The waves then take 64
// vectors of one row at a time, a few rows after the others: first those without a
// word, which the mask alone concerns (in place, -inf is written over what is not
// allowed, without reading; out of place the rest is copied, too), then the listed
// ones, over which the formula is evaluated.  Every vector is one lane's in each row,
// so nothing in the rows is ordered by a barrier.
//
// What bounds it: a 128-byte line that is touched costs a line read and a line
// written, whatever part of it changes (measured: 2 to 64 bytes of every other 64
// take the same time, 5.2e12 B/s of lines), and a line written whole 4.0e12 B/s.  And
// instructions, scalar ones as well: at 128 x 7 rows of 151936 bf16 tokens one more
// for each 16-byte vector is 0.4 us.  So what concerns a row is the wave's and stays
// in scalar registers, and the formula (some 300 operations a vector) runs over the
// list with no lane idle.  Measured there, behind 8192 tokens: 113 to 115 us with masks (a
// quarter of them nearly empty, the others 2% of the tokens; at those rates the lines touched
// would take 81, and a kernel that knows them beforehand and does nothing else takes 89 to
// 93), about 75 of them the masks', 20 the lists', 8 the formula's.  Where it took 123,
// reading and blending vectors that are masked in part, where now 2-byte stores of -inf
// go: 137; all masks ahead of the lists: 133 (lines with both changes are then touched
// twice); listing tokens in place of vectors, a lane each: 156.

#ifndef ASYMSPEC_STEP_SHAPE_H_
#define ASYMSPEC_STEP_SHAPE_H_

#include "row.h"

namespace asym_step {

constexpr int kShapeThreads = 512;
constexpr int kShapeMinTokens = 1024, kShapeMaxTokens = 8192;   // T: tokens of a workgroup, a power of two
constexpr int kShapeMaxDrafts = 64;
constexpr int kShapeUnroll = 4;                                 // vectors of a lane in flight
static_assert(kShapeThreads >= kShapeMaxDrafts && kShapeThreads >= ASYMSPEC_SHAPE_MAX_ROWS, "one thread each");

// A token's word.  Counts stay below 2^20 (ASYMSPEC_SHAPE_MAX_HISTORY), bias
// entries below 2^10 (ASYMSPEC_SHAPE_MAX_BIAS): the fields cannot overflow.
constexpr uint32_t kCount = (1u << 20) - 1u;
constexpr uint32_t kInPrompt = 1u << 20;
constexpr uint32_t kInDrafts = 1u << 21;
constexpr int kBiasShift = 22;      // bias entry + 1, or 0
static_assert(ASYMSPEC_SHAPE_MAX_HISTORY <= (int)kCount, "a count must fit its field");
static_assert(ASYMSPEC_SHAPE_MAX_BIAS < (1 << (32 - kBiasShift)), "a bias entry must fit its field");

struct ShapeArgs {
  asymspec_shape s;
  int lgT, parts;    // log2 of a workgroup's tokens, workgroups of a request
};

// LDS of a workgroup, ahead of the words [T] and the bias values [n_bias].
template <int VE>
struct ShapeLds {
  static constexpr int kGroups = kShapeMaxTokens / VE;
  uint32_t n_list, pad[3];
  int drafts[kShapeMaxDrafts];                  // as ids of this vocabulary
  int mask_row[ASYMSPEC_SHAPE_MAX_ROWS];        // -1: no mask
  unsigned long long has_word[kGroups / 64];    // bit g % 64 of g / 64: vector g is listed
  uint16_t list[kGroups];
  static size_t bytes(int T, int n_bias) { return sizeof(ShapeLds) + ((size_t)T + n_bias) * 4; }
};
static_assert(sizeof(ShapeLds<8>) % 16 == 0 && sizeof(ShapeLds<4>) % 16 == 0, "the words follow, aligned");

struct ShapeCtx {
  float rep, freq, pres;
  const float* bias;        // the request's bias values, of the entries here, in LDS
  const int* drafts;        // in LDS
};
typedef int i4 __attribute__((ext_vector_type(4)));

// One logit behind its word (0: as it was); the first n_drafts drafts precede it.  All
// lanes go the same way: of 64 vectors with a word nearly every place has one in some lane.
STEP_DEV float shape_one(float l, uint32_t w, int token, int n_drafts, const ShapeCtx& c) {
  int cnt = (int)(w & kCount);
  if (__any((w & kInDrafts) != 0u)) {
    const bool mine = (w & kInDrafts) != 0u;
    for (int j = 0; j < n_drafts; j += 4) {
      const i4 d = *(const i4*)(c.drafts + j);
#pragma unroll
      for (int i = 0; i < 4; ++i) cnt += mine && d[i] == token && j + i < n_drafts ? 1 : 0;
    }
  }
  float v = l > 0.0f ? l / c.rep : l * c.rep;
  v = cnt > 0 || (w & kInPrompt) ? v : l;
  v = cnt > 0 ? (v - c.freq * (float)cnt) - c.pres : v;
  if (__any((w >> kBiasShift) != 0u)) {
    const float bias = c.bias[max((int)(w >> kBiasShift) - 1, 0)];
    v = (w >> kBiasShift) ? v + bias : v;
  }
  return v;
}

template <int DT, bool kInPlace, bool kMasked>
// (8 waves a SIMD hide the chains of loads: with 7, 20 us more)
__global__ __launch_bounds__(kShapeThreads) __attribute__((amdgpu_waves_per_eu(8))) void shape_kernel(ShapeArgs A) {
  typedef typename Row<DT>::T E;
  constexpr int VE = Row<DT>::VE, kWaves = kShapeThreads / 64;
  constexpr uint32_t kAll = (1u << VE) - 1u;
  extern __shared__ __align__(16) uint32_t shape_lds[];
  ShapeLds<VE>& S = *(ShapeLds<VE>*)shape_lds;
  uint32_t* words = shape_lds + sizeof(S) / 4;

  const asymspec_shape& s = A.s;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = (int)(blockIdx.x / (unsigned)A.parts);
  const int T = 1 << A.lgT;
  const int x0 = (int)(blockIdx.x % (unsigned)A.parts) << A.lgT;
  const int n = min(T, s.V - x0);                         // tokens here
  ShapeCtx c;
  c.rep = s.repetition ? s.repetition[b] : 1.0f;
  c.freq = s.frequency ? s.frequency[b] : 0.0f;
  c.pres = s.presence ? s.presence[b] : 0.0f;
  float* biases = (float*)(words + T);
  c.bias = biases;
  c.drafts = S.drafts;
  // such penalties change no logit, so the lists behind them are not read
  const bool counts = !(c.rep == 1.0f && c.freq == 0.0f && c.pres == 0.0f);

  // The lists' first entries are on their way while the words are cleared.
  constexpr int kAhead = 2;                               // vectors of 4 tokens
  typedef uint32_t u4any __attribute__((ext_vector_type(4), aligned(4)));
  const int* h = s.history ? s.history + (size_t)b * s.max_history : nullptr;
  const int len = counts && h ? min(max(s.lengths[b], 0), s.max_history) : 0;
  const int plen = len > 0 && s.prompt_lengths ? s.prompt_lengths[b] : 0;
  u4 tok[kAhead];
  auto fetch = [&](int p0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int p = p0 + (k * kShapeThreads + tid) * 4;
      if (p + 4 <= s.max_history) {
        // (the first ones do not wait for the length)
        if (k == 0 || p < len) tok[k] = *(const u4any*)(h + p);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) tok[k][e] = p + e < len ? (uint32_t)h[p + e] : 0u;
      }
    }
  };
  if (h) fetch(0);
  constexpr int kBias = (ASYMSPEC_SHAPE_MAX_BIAS + kShapeThreads - 1) / kShapeThreads;
  uint32_t bias_id[kBias];
  float bias[kBias];
  if (s.n_bias > 0) {
#pragma unroll
    for (int k = 0; k < kBias; ++k) {
      const int i = tid + k * kShapeThreads;
      const size_t at = (size_t)b * s.n_bias + i;
      bias_id[k] = i < s.n_bias ? (uint32_t)s.bias_ids[at] : ~0u;
      bias[k] = i < s.n_bias ? s.bias_values[at] : 0.0f;
    }
  }
  uint32_t draft = ~0u;
  if (counts && tid < s.D) draft = (uint32_t)s.draft_tokens[b * s.draft_stride + tid];
  if (kMasked && tid < s.R) {
    const int k = s.mask_index[(size_t)b * s.R + tid];
    S.mask_row[tid] = (unsigned)k < (unsigned)s.n_masks ? k : -1;
  }
  // (no token has a word)
  const bool lists = counts || s.n_bias > 0;
  if (lists) {
    for (int i = tid; i < T / 4; i += kShapeThreads) ((u4*)words)[i] = u4{0u, 0u, 0u, 0u};
  } else if (tid < ShapeLds<VE>::kGroups / 64) {
    S.has_word[tid] = 0ull;
  }
  if (tid == 0) S.n_list = 0u;
  __syncthreads();

  // the words: bias entries first, while they are zero: the largest word is that of
  // the last entry
  if (s.n_bias > 0) {
#pragma unroll
    for (int k = 0; k < kBias; ++k) {
      const uint32_t x = bias_id[k] - (uint32_t)x0;
      if (x < (uint32_t)n) {
        atomicMax(&words[x], (uint32_t)(tid + k * kShapeThreads + 1) << kBiasShift);
        biases[tid + k * kShapeThreads] = bias[k];
      }
    }
    __syncthreads();
  }
  if (counts) {
    auto id = [&](uint32_t x) {     // of this vocabulary; above 2^31: none
      return s.id_map ? (x < (uint32_t)s.n_ids ? (uint32_t)s.id_map[x] : ~0u) : x;
    };
    if (tid < s.D) {
      const uint32_t t = id(draft), x = t - (uint32_t)x0;
      S.drafts[tid] = (int)t;
      if (x < (uint32_t)n) atomicOr(&words[x], kInDrafts);
    }
    for (int p0 = 0; p0 < len; p0 += kAhead * kShapeThreads * 4) {
      if (p0 > 0) fetch(p0);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int p = p0 + (k * kShapeThreads + tid) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (p + e < len) {
            const uint32_t x = id(tok[k][e]) - (uint32_t)x0;
            if (x < (uint32_t)n) {
              if (p + e < plen) atomicOr(&words[x], kInPrompt);
              else atomicAdd(&words[x], 1u);
            }
          }
        }
      }
    }
  }

  // the vectors with a word
  const int groups = n / VE;                              // whole vectors
  if (lists) __syncthreads();
  for (int g0 = lists ? 0 : groups; g0 < groups; g0 += kShapeThreads) {
    const int g = g0 + tid;
    bool has = false;
    if (g < groups) {
      const u4* w = (const u4*)(words + g * VE);
      u4 any = w[0];
      if (VE == 8) any |= w[1];
      has = (any[0] | any[1] | any[2] | any[3]) != 0u;
    }
    const unsigned long long m = __ballot(has);
    uint32_t at = 0;
    if (lane == 0) {
      if (m != 0ull) at = atomicAdd(&S.n_list, (uint32_t)__popcll(m));
      if (g < groups) S.has_word[g >> 6] = m;
    }
    at = (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
    if (has) S.list[at + __popcll(m & ((1ull << lane) - 1ull))] = (uint16_t)g;
  }
  if (lists) __syncthreads();

  const char* in = (const char*)((const E*)s.logits + b * s.request_stride + x0);
  char* out = (char*)((E*)s.out + b * s.out_request_stride + x0);
  const int64_t in_row = s.row_stride * (int64_t)sizeof(E), out_row = s.out_row_stride * (int64_t)sizeof(E);
  const size_t mask_bytes = (size_t)((s.V + 31) / 32) * 4;
  const char* mask = (const char*)s.mask + x0 / 8;
  // the mask bits ahead of this part in row r, or null
  auto mask_of = [&](int r) -> const char* {
    const int k = kMasked ? __builtin_amdgcn_readfirstlane(S.mask_row[r]) : -1;
    return k < 0 ? nullptr : mask + (size_t)k * mask_bytes;
  };
  auto bits_of = [&](const char* m, uint32_t g) -> uint32_t {
    return VE == 8 ? (uint32_t)(uint8_t)m[g] : ((uint32_t)(uint8_t)m[g >> 1] >> (4u * (g & 1u))) & 15u;
  };
  const int d0 = s.D - (s.R - 1);                         // drafts ahead of row 0

  auto shape_vec = [&](u4& v, uint32_t g, int r) {
    const int nd = s.D ? d0 + r : 0;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      // (ahead of its drafts a token is as it was, whatever bits it has)
      const float l = Row<DT>::get(v, e), f = shape_one(l, words[g * VE + e], x0 + (int)g * VE + e, nd, c);
      if (__float_as_uint(f) != __float_as_uint(l)) Row<DT>::put(v, e, f);
    }
  };
  // A few rows at a time: as many as give each wave its vectors in flight.
  const int m = __builtin_amdgcn_readfirstlane((int)S.n_list), wsegs = (m + 63) / 64;
  const int segs = !kInPlace || kMasked ? (groups + 63) / 64 : 0;
  const int together = segs > 0 ? max(1, kShapeUnroll * kWaves / segs) : s.R;
  // i / segs for i < segs * R <= 2^11
  const uint32_t inv = segs > 0 ? ((1u << 18) + (uint32_t)segs - 1u) / (uint32_t)segs : 0u;
  int turn = wave;                                        // of the listed vectors
  for (int r0 = 0; r0 < s.R; r0 += together) {
    const int r1 = min(s.R, r0 + together);
    if constexpr (!kInPlace || kMasked) {
      for (int i0 = wave; i0 < segs * (r1 - r0); i0 += kShapeUnroll * kWaves) {
        u4 v[kShapeUnroll];
        uint32_t allowed[kShapeUnroll], g[kShapeUnroll];
        int row[kShapeUnroll];
        bool mine[kShapeUnroll];
#pragma unroll
        for (int u = 0; u < kShapeUnroll; ++u) {
          const int i = i0 + u * kWaves, k = (int)(((uint32_t)i * inv) >> 18), seg = i - k * segs;
          row[u] = r0 + k;
          g[u] = (uint32_t)(seg * 64 + lane);
          mine[u] = false;
          allowed[u] = kAll;
          if (row[u] < r1) {
            const char* mb = mask_of(row[u]);
            if (!kInPlace || mb != nullptr) mine[u] = g[u] < (uint32_t)groups && !((S.has_word[seg] >> lane) & 1ull);
            if (mb != nullptr && mine[u]) allowed[u] = bits_of(mb, g[u]);
          }
        }
#pragma unroll
        for (int u = 0; u < kShapeUnroll; ++u) {
          if (kInPlace) mine[u] = mine[u] && allowed[u] != kAll;
          else if (mine[u] && allowed[u] != 0u) v[u] = load_vec<DT>((const E*)(in + row[u] * in_row + g[u] * 16u));
        }
#pragma unroll
        for (int u = 0; u < kShapeUnroll; ++u) {
          if (mine[u]) {
            E* o = (E*)(out + row[u] * out_row + g[u] * 16u);
            if (kMasked && allowed[u] == 0u) {
              store_vec<DT>(o, Row<DT>::neg_inf());
            } else if (kInPlace) {
              for (uint32_t off = ~allowed[u] & kAll; off != 0u; off &= off - 1u)
                o[__ffs(off) - 1] = Row<DT>::put1(-__builtin_huge_valf());
            } else {
              if (kMasked) Row<DT>::mask(v[u], allowed[u]);
              store_vec<DT>(o, v[u]);
            }
          }
        }
      }
    }
    // the listed ones, in turn
    for (; turn < wsegs * (r1 - r0); turn += kWaves) {
      const int k = turn / wsegs, r = r0 + k, at = (turn - k * wsegs) * 64 + lane;
      const char* mb = mask_of(r);
      if (at >= m) continue;
      const uint32_t g = S.list[at];
      const uint32_t allowed = mb != nullptr ? bits_of(mb, g) : kAll;
      u4 v = Row<DT>::neg_inf();
      if (allowed != 0u) {
        v = load_vec<DT>((const E*)(in + r * in_row + g * 16u));
        shape_vec(v, g, r);
        if (kMasked) Row<DT>::mask(v, allowed);
      }
      store_vec<DT>((E*)(out + r * out_row + g * 16u), v);
    }
    turn -= wsegs * (r1 - r0);
  }

  // the tokens behind the last whole vector of a row
  for (int i = tid; i < (n - groups * VE) * s.R; i += kShapeThreads) {
    const int r = i % s.R, e = i / s.R, x = groups * VE + e;
    const uint32_t w = lists ? words[x] : 0u;
    const int k = kMasked ? S.mask_row[r] : -1;
    const bool on = k < 0 || ((uint8_t)mask[(size_t)k * mask_bytes + x / 8] >> (x % 8)) & 1;
    E v = ((const E*)(in + r * in_row))[x];
    const float l = Row<DT>::get1(v), f = on && w != 0u ? shape_one(l, w, x0 + x, s.D ? d0 + r : 0, c) : l;
    if (!on) v = Row<DT>::put1(-__builtin_huge_valf());
    else if (__float_as_uint(f) != __float_as_uint(l)) v = Row<DT>::put1(f);
    if (!kInPlace || !on || w != 0u) ((E*)(out + r * out_row))[x] = v;
  }
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_SHAPE_H_
