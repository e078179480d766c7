// A draw from each of N logit rows: the lowest index of the largest logit, or
// an inverse-CDF draw from softmax(l / tau) with the caller's uniform.
//
// The token is a whole number that has to come out the same however the row is
// summed, also where a uniform falls next to a step of the distribution: with
// fp32 weights the steps of a 10^5-token row are uncertain by about as much as
// the smallest of them is wide.  So the weights and their sums are fp64: steps
// are then uncertain by 1e-13 of the sum.
//
// Two kernels.  draw_part: one wave per chunk of 1024 tokens keeps its chunk in
// registers, finds its largest logit m and sums exp((l - m) / tau); no wave
// waits for another.  draw_pick: one wave per row joins the chunks' sums in
// their order, finds the chunk that the draw falls into, and reads that chunk
// again to find the token.  A row is split because the exponentials bound it: one
// compute unit alone would take about 20 us over 151936 tokens.
//
// draw_part runs 20 vector operations a token and about 100 a chunk, 26 a token in
// all, at 33e12 lane operations a second as this chip issues fp64 ones: 103 us for
// 512 rows of 256000 bf16 tokens (262 MB, 51 us at a copy's rate; 95 us with the rows
// in cache), 15 us for 128 of 151936; draw_pick 4 to 5 us.  Greedy rows take a read's
// time.  Chunks of 2048 tokens take 4% less on the large batch, but 0.7 us more on one
// row and in draw_pick; two chunks a wave, or waves that stay and fetch their next
// chunk ahead, take 4 to 6% more (a SIMD then holds seven waves in place of eight).

#ifndef ASYMSPEC_STEP_DRAW_H_
#define ASYMSPEC_STEP_DRAW_H_

#include "../device.h"
#include "row.h"

namespace asym_step {

constexpr int kDrawThreads = 256;             // 4 chunks
constexpr int kDrawPer = 16;                  // tokens of a lane
constexpr int kDrawChunk = 64 * kDrawPer;     // tokens of a chunk

struct DrawPart {
  double sum;      // of exp((l - m) / tau) over the chunk; 0 without any weight
  float m;         // the chunk's largest logit
  int32_t arg;     // greedy rows: its first index in the row
};

struct DrawArgs {
  const void* logits;
  int64_t row_stride;
  const float* tau;
  const float* u;
  int64_t u_stride;
  int32_t* token;
  int64_t token_stride;
  float* prob;
  int64_t prob_stride;
  DrawPart* part;    // [N][S]
  int N, V, S;       // S: chunks of a row
};

// The weights exp((l - m) / tau) = 2^t, t = k (l - m), of logits l <= m, to 2e-14
// relative: 2^n times a polynomial in f = t - n, |f| <= 1/2, of degree 9
// (interpolated at the Chebyshev points of the interval, so near the best of its
// degree).  n comes out of an addition of 1.5 * 2^52, whose sum holds it in its
// low word.  A logit of -inf or not a number has weight 0, as has what is below
// 2^-1074.  Below m = +inf a weight is 1 or 0: flat() turns such logits into ones
// that give that.
//
// The coefficients are kept in scalar registers, where a fused multiply-add reads
// them in place; as literals each costs two moves (512 rows of 256000 bf16 tokens:
// 145 us against 121).
struct DrawScale {
  double c[10], k, m, least;
  bool inf;
  STEP_DEV DrawScale(float tau, float top)
      : c{0x1.000000000003dp+0,  0x1.62e42fefa39f7p-1,  0x1.ebfbdff8149f2p-3,  0x1.c6b08d7044119p-5,
          0x1.3b2ab72b175eep-7,  0x1.5d87fe908f88ap-10, 0x1.43088e257f341p-13, 0x1.ffcb76789860fp-17,
          0x1.63ef969a64d3cp-20, 0x1.b6571de2f2351p-24} {
#pragma unroll
    for (int i = 0; i < 9; ++i) asm("" : "+s"(c[i]));
    asm("" : "+v"(c[9]));      // (an instruction reads one scalar at most)
    // (an infinite temperature is a very large one: it leaves -inf without weight)
    const double t = __builtin_fmin((double)tau, 0x1p200);
    double r = __builtin_amdgcn_rcp(t);       // and two steps of Newton's method
    r = __builtin_fma(r, __builtin_fma(-t, r, 1.0), r);
    r = __builtin_fma(r, __builtin_fma(-t, r, 1.0), r);
    k = 1.4426950408889634074 * r;
    inf = top == __builtin_huge_valf();
    m = inf ? 0.0 : (double)top;
    least = -762.0 * t;        // 2^-1099
  }
  STEP_DEV float flat(float l) const { return l == __builtin_huge_valf() ? 0.0f : -__builtin_huge_valf(); }
  // (of a logit that went through flat() where inf)
  STEP_DEV double weight(double l) const {
    const double d = __builtin_fmax(l - m, least);
    const double s = __builtin_fma(k, d, 0x1.8p52), n = s - 0x1.8p52;
    const double f = __builtin_fma(k, d, -n);
    double p = __builtin_fma(c[9], f, c[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) p = __builtin_fma(p, f, c[i]);
    return __builtin_ldexp(p, (int)(uint32_t)__builtin_bit_cast(uint64_t, s));
  }
};

// A lane's 16 tokens of the chunk at x0 of a row: vectors first, first + step, ...
// of the chunk.  Past the row's end -inf.
template <int DT>
STEP_DEV void draw_load(const typename Row<DT>::T* row, int x0, int V, int first, int step,
                        u4 (&v)[kDrawPer / Row<DT>::VE]) {
  constexpr int VE = Row<DT>::VE, NV = kDrawPer / VE;
  if (x0 + kDrawChunk <= V) {       // the same for the whole wave: nothing between the loads
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = load_vec<DT>(row + x0 + (first + i * step) * VE);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = Row<DT>::neg_inf();
      const int x = x0 + (first + i * step) * VE;
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (x + e < V) Row<DT>::put_bits(v[i], e, row[x + e]);
    }
  }
}
template <int DT>
STEP_DEV void draw_decode(const u4 (&v)[kDrawPer / Row<DT>::VE], float (&l)[kDrawPer]) {
  constexpr int VE = Row<DT>::VE;
#pragma unroll
  for (int i = 0; i < kDrawPer; ++i) l[i] = Row<DT>::get(v[i / VE], i % VE);
}

template <int DT>
__global__ __launch_bounds__(kDrawThreads) void draw_part_kernel(DrawArgs A) {
  constexpr int VE = Row<DT>::VE;
  const int lane = (int)threadIdx.x & 63;
  const unsigned id = blockIdx.x * (kDrawThreads / 64) + (unsigned)__builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const unsigned row = id / (unsigned)A.S;
  if (row >= (unsigned)A.N) return;
  const int x0 = (int)(id - row * (unsigned)A.S) * kDrawChunk;
  const float tau = A.tau[row];
  u4 v[kDrawPer / VE];
  draw_load<DT>((const typename Row<DT>::T*)A.logits + row * A.row_stride, x0, A.V, lane, 64, v);
  float l[kDrawPer];
  draw_decode<DT>(v, l);
  // The maximum as fp64, which the weights need too: the conversion makes every
  // not-a-number a quiet one, which fmax leaves out.
  double top = -__builtin_huge_val();
#pragma unroll
  for (int i = 0; i < kDrawPer; ++i) top = __builtin_fmax(top, (double)l[i]);
  const float m = asym::wave_max((float)top);
  double sum = 0.0;
  int arg = 0;
  if (!(tau > 0.0f)) {
    arg = 0x7FFFFFFF;
#pragma unroll
    for (int i = kDrawPer - 1; i >= 0; --i)
      if (l[i] == m) arg = x0 + ((i / VE) * 64 + lane) * VE + i % VE;
    arg = asym::wave_min_i(arg);
  } else if (m > -__builtin_huge_valf()) {
    const DrawScale k(tau, m);
    if (k.inf) {
#pragma unroll
      for (int i = 0; i < kDrawPer; ++i) l[i] = k.flat(l[i]);
    }
    double part[2] = {0.0, 0.0};
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i) part[i & 1] += k.weight((double)l[i]);
    double before;
    asym::wave_scan_d(part[0] + part[1], sum, before);
  }
  if (lane == 63) A.part[id] = DrawPart{sum, m, arg};
}

template <int DT>
__global__ __launch_bounds__(64) void draw_pick_kernel(DrawArgs A) {
  constexpr int VE = Row<DT>::VE;
  const int lane = (int)threadIdx.x, row = (int)blockIdx.x;
  const DrawPart* P = A.part + (size_t)row * A.S;
  const float inf = __builtin_huge_valf();
  const float tau = A.tau[row];
  float u = A.u ? A.u[row * A.u_stride] : 0.0f;
  if (!(u > 0.0f)) u = 0.0f;
  int32_t* token = A.token + row * A.token_stride;
  float* prob = A.prob ? A.prob + row * A.prob_stride : nullptr;

  // The chunk that the draw falls into: each lane has a run of chunks, kept in
  // registers where it is short (rows of up to 2^18 tokens), else read each time.
  constexpr int kKeep = 4;
  const int per = (A.S + 63) / 64;
  const int lo = min(A.S, lane * per), hi = min(A.S, lo + per);
  DrawPart kept[kKeep];
#pragma unroll
  for (int j = 0; j < kKeep; ++j) kept[j] = per <= kKeep && lo + j < hi ? P[lo + j] : DrawPart{0.0, -inf, 0x7FFFFFFF};
  auto each = [&](auto&& f) {       // f(chunk, its part), in order
    if (per <= kKeep) {
#pragma unroll
      for (int j = 0; j < kKeep; ++j) f(lo + j, kept[j]);
    } else {
      for (int s = lo; s < hi; ++s) {
        DrawPart q = P[s];
        f(s, q);
      }
    }
  };
  float mine_m = -inf;
  int arg = 0x7FFFFFFF;
  each([&](int, const DrawPart& q) {
    if (q.m > mine_m) {
      mine_m = q.m;
      arg = q.arg;
    }
  });
  const float m = asym::wave_max(mine_m);
  if (!(tau > 0.0f) || m == -inf) {
    arg = asym::wave_min_i(mine_m == m ? arg : 0x7FFFFFFF);
    if (lane == 0) {
      *token = m == -inf ? 0 : arg;
      if (prob) *prob = m == -inf ? 0.0f : 1.0f;
    }
    return;
  }
  const DrawScale k(tau, m);
  auto weight_of = [&](const DrawPart& q) { return q.sum * k.weight((double)(k.inf ? k.flat(q.m) : q.m)); };
  double mine = 0.0, upto, ahead;
  each([&](int, DrawPart& q) {
    const double w = weight_of(q);
    q.sum = w;              // (of a kept part: its weight from here on)
    mine += w;
  });
  asym::wave_scan_d(mine, upto, ahead);
  const double total = __shfl(upto, 63, 64);
  const double target = (double)u * total;
  // the first lane whose sums pass the target; without one (a uniform of 1) the
  // last lane with weight
  const unsigned long long past = __ballot(upto > target && mine > 0.0), some = __ballot(mine > 0.0);
  const bool none = past == 0ull;
  const int from = none ? 63 - __clzll((long long)(some | 1ull)) : __ffsll(past) - 1;
  int at = lo;
  double before = ahead;
  {
    double c = ahead;
    bool found = false;
    each([&](int s, const DrawPart& q) {
      const double w = per <= kKeep ? q.sum : weight_of(q);
      if (w > 0.0 && !found) {
        at = s;
        before = c;
        found = !none && c + w > target;
      }
      c += w;
    });
  }
  at = __shfl(at, from, 64);
  before = __shfl(before, from, 64);

  // The token in it: each lane has 16 consecutive ones.  The first lane whose
  // sums pass the target holds it; if rounding, or a uniform of 1, puts the target
  // behind all of them, the last lane with weight, and its last such token.
  const typename Row<DT>::T* p = (const typename Row<DT>::T*)A.logits + row * A.row_stride;
  const int x0 = at * kDrawChunk + lane * kDrawPer;
  u4 v[kDrawPer / VE];
  draw_load<DT>(p, at * kDrawChunk, A.V, lane * (kDrawPer / VE), 1, v);
  float l[kDrawPer];
  draw_decode<DT>(v, l);
  if (k.inf) {
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i) l[i] = k.flat(l[i]);
  }
  double w[kDrawPer];
  double sum = 0.0, incl, excl;
#pragma unroll
  for (int i = 0; i < kDrawPer; ++i) {
    w[i] = k.weight((double)l[i]);
    sum += w[i];
  }
  asym::wave_scan_d(sum, incl, excl);
  const unsigned long long over = none ? 0ull : __ballot(before + incl > target && sum > 0.0);
  const unsigned long long has = __ballot(sum > 0.0);
  const int who = over != 0ull ? __ffsll(over) - 1 : 63 - __clzll((long long)(has | 1ull));
  if (lane == who) {
    double c = before + excl, wt = 0.0;
    int t = 0;
    bool found = false;
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i) {
      if (w[i] > 0.0 && !found) {
        t = x0 + i;
        wt = w[i];
        found = over != 0ull && c + w[i] > target;
      }
      c += w[i];
    }
    *token = t;
    if (prob) *prob = (float)(wt / total);
  }
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_DRAW_H_
