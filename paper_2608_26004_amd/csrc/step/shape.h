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
// rounded once.  In place, 16-byte pieces whose words are all zero and whose
// tokens are all allowed are neither read nor written; pieces with no allowed
// token are written without being read.

#ifndef ASYMSPEC_STEP_SHAPE_H_
#define ASYMSPEC_STEP_SHAPE_H_

#include "row.h"

namespace asym_step {

constexpr int kShapeThreads = 512;
constexpr int kShapeMinTokens = 1024, kShapeMaxTokens = 8192;   // T: tokens of a workgroup, a power of two
constexpr int kShapeMaxDrafts = 64;

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
  int T, parts;      // tokens of a workgroup, workgroups of a request
};

struct ShapeCtx {
  float rep, freq, pres;
  const float* bias;        // the request's bias values
  const int* drafts;        // in LDS, as ids of this vocabulary
};

// One allowed logit with a nonzero word; the first n_drafts drafts precede it.
STEP_DEV float shape_one(float v, uint32_t w, int token, int n_drafts, const ShapeCtx& c) {
  int cnt = (int)(w & kCount);
  if (w & kInDrafts)
    for (int j = 0; j < n_drafts; ++j) cnt += c.drafts[j] == token ? 1 : 0;
  if (cnt > 0 || (w & kInPrompt)) v = v > 0.0f ? v / c.rep : v * c.rep;
  if (cnt > 0) v = (v - c.freq * (float)cnt) - c.pres;
  if (w >> kBiasShift) v = v + c.bias[(w >> kBiasShift) - 1u];
  return v;
}

// One vector of tokens x0 .. x0 + VE - 1: bit e of `allowed` is token x0 + e.
template <int DT>
STEP_DEV void shape_vec(u4& v, const uint32_t* words, uint32_t allowed, int x0, int n_drafts, const ShapeCtx& c) {
#pragma unroll
  for (int e = 0; e < Row<DT>::VE; ++e) {
    const uint32_t w = words[e];
    if (!((allowed >> e) & 1u)) {
      Row<DT>::put(v, e, -__builtin_huge_valf());
    } else if (w != 0u) {
      Row<DT>::put(v, e, shape_one(Row<DT>::get(v, e), w, x0 + e, n_drafts, c));
    }
  }
}

template <int DT, bool kInPlace, bool kMasked>
__global__ __launch_bounds__(kShapeThreads) void shape_kernel(ShapeArgs A) {
  typedef typename Row<DT>::T E;
  constexpr int VE = Row<DT>::VE;
  constexpr int kPer = kShapeMaxTokens / VE / kShapeThreads;      // vectors per thread and row, at most
  extern __shared__ __align__(16) uint32_t shape_lds[];
  uint32_t* words = shape_lds;                                  // [T]
  int* drafts = (int*)(shape_lds + A.T);                        // [kShapeMaxDrafts]
  uint32_t* n_list = shape_lds + A.T + kShapeMaxDrafts;         // [1] (and padding)
  uint16_t* list = (uint16_t*)(n_list + 4);               // [T / VE]

  const asymspec_shape& s = A.s;
  const int tid = (int)threadIdx.x;
  const int b = (int)(blockIdx.x / (unsigned)A.parts);
  const int x0 = (int)(blockIdx.x % (unsigned)A.parts) * A.T;
  const int n = min(A.T, s.V - x0);                       // tokens here
  ShapeCtx c;
  c.rep = s.repetition ? s.repetition[b] : 1.0f;
  c.freq = s.frequency ? s.frequency[b] : 0.0f;
  c.pres = s.presence ? s.presence[b] : 0.0f;
  c.bias = s.bias_values ? s.bias_values + (size_t)b * s.n_bias : nullptr;
  c.drafts = drafts;
  // such penalties change no logit, so the lists behind them are not read
  const bool counts = !(c.rep == 1.0f && c.freq == 0.0f && c.pres == 0.0f);

  for (int i = tid; i < A.T / 4; i += kShapeThreads) ((u4*)words)[i] = u4{0u, 0u, 0u, 0u};
  if (tid == 0) *n_list = 0u;
  __syncthreads();
  // the bias entries first, while the words are zero: the largest word is that
  // of the last entry
  for (int k = tid; k < s.n_bias; k += kShapeThreads) {
    const uint32_t x = (uint32_t)s.bias_ids[(size_t)b * s.n_bias + k] - (uint32_t)x0;
    if (x < (uint32_t)n) atomicMax(&words[x], (uint32_t)(k + 1) << kBiasShift);
  }
  __syncthreads();
  if (counts) {
    auto here = [&](int x) {        // place in `words`, or out of range
      if (s.id_map) x = (unsigned)x < (unsigned)s.n_ids ? s.id_map[x] : -1;
      return x < 0 ? -1 : x - x0;
    };
    if (tid < s.D) {
      const int x = here(s.draft_tokens[b * s.draft_stride + tid]);
      drafts[tid] = x + x0;
      if ((unsigned)x < (unsigned)n) atomicOr(&words[x], kInDrafts);
    }
    if (s.history) {
      const int len = min(max(s.lengths[b], 0), s.max_history);
      const int plen = s.prompt_lengths ? s.prompt_lengths[b] : 0;
      const int* h = s.history + (size_t)b * s.max_history;
      for (int p = tid; p < len; p += kShapeThreads) {
        const int x = here(h[p]);
        if ((unsigned)x < (unsigned)n) {
          if (p < plen) atomicOr(&words[x], kInPrompt);
          else atomicAdd(&words[x], 1u);
        }
      }
    }
    __syncthreads();
  }

  const E* in = (const E*)s.logits + b * s.request_stride + x0;
  E* out = (E*)s.out + b * s.out_request_stride + x0;
  const int groups = (n + VE - 1) / VE;
  const int d0 = s.D - (s.R - 1);                         // drafts ahead of row 0

  // one group of one row; the row's last group may be partial
  auto group = [&](int r, int g, uint32_t allowed, bool active) {
    const E* pi = in + r * s.row_stride + g * VE;
    E* po = out + r * s.out_row_stride + g * VE;
    const int x = x0 + g * VE;
    const int nd = s.D ? d0 + r : 0;
    if (g * VE + VE <= n) {
      u4 v;
      if (kMasked && allowed == 0u) {
        v = Row<DT>::neg_inf();
      } else {
        v = load_vec<DT>(pi);
        if (active || (kMasked && allowed != (1u << VE) - 1u))
          shape_vec<DT>(v, words + g * VE, allowed, x, nd, c);
      }
      store_vec<DT>(po, v);
    } else {
      for (int e = 0; e < n - g * VE; ++e) {
        const uint32_t w = words[g * VE + e];
        E v = pi[e];
        const E old = v;
        if (!((allowed >> e) & 1u)) v = Row<DT>::put1(-__builtin_huge_valf());
        else if (w != 0u) v = Row<DT>::put1(shape_one(Row<DT>::get1(v), w, x + e, nd, c));
        if (!kInPlace || v != old) po[e] = v;
      }
    }
  };
  auto is_active = [&](int g) {
    const u4* w = (const u4*)(words + g * VE);
    u4 any = w[0];
    if (VE == 8) any |= w[1];
    return (any[0] | any[1] | any[2] | any[3]) != 0u;
  };

  if (kInPlace && !kMasked) {
    // few groups have anything to do: listed, then spread over the threads
    for (int g = tid; g < groups; g += kShapeThreads)
      if (is_active(g)) list[atomicAdd(n_list, 1u)] = (uint16_t)g;
    __syncthreads();
    const int m = (int)*n_list;
    for (int i = tid; i < m * s.R; i += kShapeThreads) {
      const int r = i / m;
      group(r, list[i - r * m], 0xFFu, true);
    }
  } else {
    bool active[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int g = tid + k * kShapeThreads;
      active[k] = g < groups && is_active(g);
    }
    const int W = (s.V + 31) / 32;
    for (int r = 0; r < s.R; ++r) {
      const uint8_t* m = nullptr;
      if (kMasked) {
        const int k = s.mask_index[(size_t)b * s.R + r];
        if ((unsigned)k < (unsigned)s.n_masks) m = (const uint8_t*)(s.mask + (size_t)k * W) + x0 / 8;
      }
      uint32_t allowed[kPer];
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int g = tid + k * kShapeThreads;
        allowed[k] = (1u << VE) - 1u;
        if (kMasked && m != nullptr && g < groups)
          allowed[k] = VE == 8 ? m[g] : (m[g >> 1] >> (4 * (g & 1))) & 15u;
      }
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int g = tid + k * kShapeThreads;
        if (g < groups && (!kInPlace || active[k] || (kMasked && allowed[k] != (1u << VE) - 1u)))
          group(r, g, allowed[k], active[k]);
      }
    }
  }
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_SHAPE_H_
