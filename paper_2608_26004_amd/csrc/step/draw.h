// A draw from each of N logit rows: the lowest index of the largest logit, or
// an inverse-CDF draw from softmax(l / tau) with the caller's uniform.
//
// The token is a whole number that has to come out the same however the row is
// summed, also where a uniform falls next to a step of the distribution: with
// fp32 weights the steps of a 10^5-token row are uncertain by about as much as
// the smallest of them is wide.  So the weights and their sums are fp64: steps
// are then uncertain by 1e-15 of the sum.
//
// Two kernels.  draw_part: one workgroup per (row, chunk of 4096 tokens) keeps
// its chunk in registers, finds its maximum m and sums exp((l - m) / tau).
// draw_pick: one workgroup per row joins the chunks' sums in their order, finds
// the chunk that the draw falls into, and reads that chunk again to find the
// token.

#ifndef ASYMSPEC_STEP_DRAW_H_
#define ASYMSPEC_STEP_DRAW_H_

#include "row.h"

namespace asym_step {

constexpr int kDrawThreads = 256;
constexpr int kDrawPer = 16;                                // tokens of a thread
constexpr int kDrawChunk = kDrawThreads * kDrawPer;         // tokens of a chunk

struct DrawPart {
  double sum;      // of exp((l - m) / tau) over the chunk
  float m;         // the chunk's largest logit (-inf: no weight)
  int32_t arg;     // its first index in the row
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

// exp((l - m) / tau) for -inf < l <= m; k = 1 / tau.  Never not a number: below
// m = +inf, and for any k, an infinite difference has no weight.
STEP_DEV double draw_weight(float l, float m, double k) {
  if (l == m) return 1.0;
  const double d = (double)l - (double)m;
  return d > -__builtin_huge_val() ? exp(d * k) : 0.0;
}

// Tokens x0 .. x0 + kDrawPer - 1 of a row as fp32; past its end, and where it
// is not a number, -inf.
template <int DT>
STEP_DEV void draw_load(const typename Row<DT>::T* row, int x0, int V, float* l) {
  constexpr int VE = Row<DT>::VE;
  if (x0 + kDrawPer <= V) {
    u4 v[kDrawPer / VE];
#pragma unroll
    for (int i = 0; i < kDrawPer / VE; ++i) v[i] = load_vec<DT>(row + x0 + i * VE);
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i) l[i] = Row<DT>::get(v[i / VE], i % VE);
  } else {
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i) l[i] = x0 + i < V ? Row<DT>::get1(row[x0 + i]) : -__builtin_huge_valf();
  }
#pragma unroll
  for (int i = 0; i < kDrawPer; ++i)
    if (l[i] != l[i]) l[i] = -__builtin_huge_valf();
}

// The larger logit, and of two equal ones the lower index.
STEP_DEV void draw_max(float& m, int& arg, float m2, int arg2) {
  if (m2 > m || (m2 == m && arg2 < arg)) {
    m = m2;
    arg = arg2;
  }
}

template <int DT>
__global__ __launch_bounds__(kDrawThreads) void draw_part_kernel(DrawArgs A) {
  __shared__ float sm[kDrawThreads / 64];
  __shared__ int sa[kDrawThreads / 64];
  __shared__ double ss[kDrawThreads / 64];
  const int tid = (int)threadIdx.x, wave = tid >> 6;
  const int row = (int)(blockIdx.x / (unsigned)A.S), s = (int)(blockIdx.x % (unsigned)A.S);
  const typename Row<DT>::T* p = (const typename Row<DT>::T*)A.logits + row * A.row_stride;
  const int x0 = s * kDrawChunk + tid * kDrawPer;
  float l[kDrawPer];
  draw_load<DT>(p, x0, A.V, l);
  float m = l[0];
  int arg = x0;
#pragma unroll
  for (int i = 1; i < kDrawPer; ++i)
    if (l[i] > m) {
      m = l[i];
      arg = x0 + i;
    }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) draw_max(m, arg, __shfl_xor(m, off, 64), __shfl_xor(arg, off, 64));
  if ((tid & 63) == 0) {
    sm[wave] = m;
    sa[wave] = arg;
  }
  __syncthreads();
  m = sm[0];
  arg = sa[0];
#pragma unroll
  for (int w = 1; w < kDrawThreads / 64; ++w) draw_max(m, arg, sm[w], sa[w]);
  const float tau = A.tau[row];
  double sum = 0.0;
  if (tau > 0.0f && m > -__builtin_huge_valf()) {
    const double k = 1.0 / (double)tau;
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i)
      if (l[i] > -__builtin_huge_valf()) sum += draw_weight(l[i], m, k);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if ((tid & 63) == 0) ss[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kDrawThreads / 64; ++w) sum += ss[w];
  }
  if (tid == 0) A.part[(size_t)row * A.S + s] = DrawPart{sum, m, arg};
}

// Inclusive sums over the workgroup's threads, in their order.
STEP_DEV double draw_scan(double v, double* lds, double& total) {
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double o = __shfl_up(v, off, 64);
    if (lane >= off) v += o;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = v;
  __syncthreads();
  double before = 0.0;
  total = 0.0;
#pragma unroll
  for (int w = 0; w < kDrawThreads / 64; ++w) {
    if (w < wave) before += lds[w];
    total += lds[w];
  }
  return before + v;
}

template <int DT>
__global__ __launch_bounds__(kDrawThreads) void draw_pick_kernel(DrawArgs A) {
  __shared__ float sm[kDrawThreads / 64];
  __shared__ int sa[kDrawThreads / 64];
  __shared__ double lds[kDrawThreads / 64];
  __shared__ int found, last;
  __shared__ double found_before;
  const int tid = (int)threadIdx.x, row = (int)blockIdx.x;
  const DrawPart* P = A.part + (size_t)row * A.S;
  const float inf = __builtin_huge_valf();
  // the row's largest logit
  float m = -inf;
  int arg = 0x7FFFFFFF;
  for (int s = tid; s < A.S; s += kDrawThreads) draw_max(m, arg, P[s].m, P[s].arg);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) draw_max(m, arg, __shfl_xor(m, off, 64), __shfl_xor(arg, off, 64));
  if ((tid & 63) == 0) {
    sm[tid >> 6] = m;
    sa[tid >> 6] = arg;
  }
  if (tid == 0) {
    found = 0x7FFFFFFF;
    last = -1;
  }
  __syncthreads();
  m = sm[0];
  arg = sa[0];
#pragma unroll
  for (int w = 1; w < kDrawThreads / 64; ++w) draw_max(m, arg, sm[w], sa[w]);
  int32_t* token = A.token + row * A.token_stride;
  float* prob = A.prob ? A.prob + row * A.prob_stride : nullptr;
  const float tau = A.tau[row];
  if (!(tau > 0.0f) || m == -inf) {
    if (tid == 0) {
      *token = m == -inf ? 0 : arg;
      if (prob) *prob = m == -inf ? 0.0f : 1.0f;
    }
    return;
  }
  const double k = 1.0 / (double)tau;
  // the chunk that the draw falls into: each thread has a run of chunks
  const int per = (A.S + kDrawThreads - 1) / kDrawThreads;
  const int lo = min(A.S, tid * per), hi = min(A.S, lo + per);
  auto chunk_sum = [&](int s) { return P[s].m > -inf ? P[s].sum * draw_weight(P[s].m, m, k) : 0.0; };
  double mine = 0.0;
  for (int s = lo; s < hi; ++s) mine += chunk_sum(s);
  double total;
  const double upto = draw_scan(mine, lds, total);
  float u = A.u ? A.u[row * A.u_stride] : 0.0f;
  if (!(u > 0.0f)) u = 0.0f;
  const double target = (double)u * total;
  {
    double c = upto - mine;
    int f = -1, z = -1;
    double fb = 0.0;
    for (int s = lo; s < hi; ++s) {
      const double w = chunk_sum(s);
      if (w > 0.0) z = s;
      if (f < 0 && c + w > target && w > 0.0) {
        f = s;
        fb = c;
      }
      c += w;
    }
    if (f >= 0) atomicMin(&found, f);
    if (z >= 0) atomicMax(&last, z);
    __syncthreads();
    if (f >= 0 && found == f) found_before = fb;
    // no sum exceeds the target: the last token with weight
    const bool none = found == 0x7FFFFFFF;
    __syncthreads();
    if (none && tid == 0) {
      found = last;
      found_before = -__builtin_huge_val();
    }
    __syncthreads();
  }
  const int s = max(found, 0);      // (the chunk of the largest logit has weight, so one was found)
  const double before = found_before;
  __syncthreads();
  if (tid == 0) {
    found = 0x7FFFFFFF;
    last = -1;
  }
  const typename Row<DT>::T* p = (const typename Row<DT>::T*)A.logits + row * A.row_stride;
  const int x0 = s * kDrawChunk + tid * kDrawPer;
  float l[kDrawPer];
  draw_load<DT>(p, x0, A.V, l);
  double w[kDrawPer];
  mine = 0.0;
#pragma unroll
  for (int i = 0; i < kDrawPer; ++i) {
    w[i] = l[i] > -inf ? draw_weight(l[i], m, k) : 0.0;
    mine += w[i];
  }
  double unused;
  const double up = draw_scan(mine, lds, unused);
  double c = before + (up - mine);
  int f = -1, z = -1;
#pragma unroll
  for (int i = 0; i < kDrawPer; ++i) {
    c += w[i];
    if (w[i] > 0.0) z = x0 + i;
    if (f < 0 && w[i] > 0.0 && c > target) f = x0 + i;
  }
  if (f >= 0) atomicMin(&found, f);
  if (z >= 0) atomicMax(&last, z);
  __syncthreads();
  const int t = found != 0x7FFFFFFF ? found : last;
#pragma unroll
  for (int i = 0; i < kDrawPer; ++i)
    if (x0 + i == t) {
      *token = t;
      if (prob) *prob = (float)(w[i] / total);
    }
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_DRAW_H_
