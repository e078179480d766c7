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
// compute unit alone would take about 20 us over 151936 tokens.  bf16 rows of which
// a workgroup has many tokens go through draw_table in place of draw_part.
//
// draw_part runs 17 vector operations a token, 14 of them fp64, and about 75 a chunk, at
// the 30e12 lane operations a second that this chip reaches with fp64 multiply-adds: 96 us
// for 512 rows of 256000 bf16 tokens (262 MB, 51 us at a copy's rate).  Greedy rows take
// a read's time.  Chunks of 2048 tokens take 4% less on the large batch, but 0.7 us more
// on one row and in draw_pick; two chunks a wave, or waves that stay and fetch their next
// chunk ahead, take 4 to 6% more (a SIMD then holds seven waves in place of eight).
// draw_table takes 55 to 61 us there, near a read's time; for 128 rows of 151936 tokens 13 us
// against 16, 1 to 2 of them the table's making.  draw_pick takes 4 to 5 us.  fp32 rows, all
// in draw_part: 65 us for 256 of 256000 (the same bytes), 47 greedy (partly from the cache).

#ifndef ASYMSPEC_STEP_DRAW_H_
#define ASYMSPEC_STEP_DRAW_H_

#include "../device.h"
#include "row.h"

namespace asym_step {

constexpr int kDrawThreads = 256;             // 4 chunks
constexpr int kDrawPer = 16;                  // tokens of a lane
constexpr int kDrawChunk = 64 * kDrawPer;     // tokens of a chunk

struct DrawPart {
  double sum;      // of the chunk's weights; 0 without any
  float m;         // the chunk's largest logit; -inf without any
  int32_t arg;     // greedy rows: its first index in the row; else kPlain where the weights
                   // are 2^(k l - rint(k m)), kTabled where 2^(k l), and 0 where 2^(k (l - m))
};
constexpr int32_t kPlain = 1, kTabled = 2;

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
  int C, P;          // with a table: chunks of a workgroup, workgroups of a row
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
  STEP_DEV double weight(double l) const { return raised(__builtin_fmax(l - m, least), 0x1.8p52); }
  // 2^(k d - M), |k d| and |M| below 2^30, magic = 1.5 * 2^52 - M
  STEP_DEV double raised(double d, double magic) const {
    const double s = __builtin_fma(k, d, magic), n = s - magic;
    const double f = __builtin_fma(k, d, -n);
    double p = __builtin_fma(c[9], f, c[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) p = __builtin_fma(p, f, c[i]);
    return __builtin_ldexp(p, (int)(uint32_t)__builtin_bit_cast(uint64_t, s));
  }
  // A chunk's sum at the row's level m.  (Scaled at the end: the step between the two
  // levels alone may be beyond fp64's range.)
  STEP_DEV double of_part(const DrawPart& q) const {
    if ((q.arg != kPlain && q.arg != kTabled) || inf) return q.sum * weight((double)(inf ? flat(q.m) : q.m));
    // times 2^(rint(k q.m) - k m), or 2^(-k m)
    const double at = q.arg == kPlain ? __builtin_rint(k * (double)q.m) : 0.0;
    const double d = __builtin_fmax(__builtin_fma(-k, m, at), -2200.0);
    const double n = __builtin_rint(d), f = d - n;
    double p = __builtin_fma(c[9], f, c[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) p = __builtin_fma(p, f, c[i]);
    return __builtin_ldexp(q.sum * p, (int)n);
  }
};

// Reductions over a wave, one instruction a step where the values have 32 bits: lanes
// that a step leaves out take the operation's identity, so that it needs no move.  The
// result is the wave's (a sum's is in lane 63).
template <int CTRL, int ROWMASK = 0xF>
STEP_DEV int draw_dpp(int old, int x) {
  return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWMASK, 0xF, false);
}
STEP_DEV int draw_max_i(int x) {
  constexpr int kLeast = (int)0x80000000;
  x = max(x, draw_dpp<0xB1>(kLeast, x));
  x = max(x, draw_dpp<0x4E>(kLeast, x));
  x = max(x, draw_dpp<0x141>(kLeast, x));
  x = max(x, draw_dpp<0x140>(kLeast, x));
  x = max(x, draw_dpp<0x142, 0xA>(kLeast, x));
  x = max(x, draw_dpp<0x143, 0xC>(kLeast, x));
  return __builtin_amdgcn_readlane(x, 63);
}
STEP_DEV uint32_t draw_max_u(uint32_t x) {
  x = max(x, (uint32_t)draw_dpp<0xB1>(0, (int)x));
  x = max(x, (uint32_t)draw_dpp<0x4E>(0, (int)x));
  x = max(x, (uint32_t)draw_dpp<0x141>(0, (int)x));
  x = max(x, (uint32_t)draw_dpp<0x140>(0, (int)x));
  x = max(x, (uint32_t)draw_dpp<0x142, 0xA>(0, (int)x));
  x = max(x, (uint32_t)draw_dpp<0x143, 0xC>(0, (int)x));
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
template <int CTRL>
STEP_DEV double draw_dpp_d(double x) {      // (each lane has a source)
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)b, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)lo | ((uint64_t)hi << 32));
}
STEP_DEV double draw_sum_d(double x) {
  x += draw_dpp_d<0xB1>(x);
  x += draw_dpp_d<0x4E>(x);
  x += draw_dpp_d<0x141>(x);
  x += draw_dpp_d<0x140>(x);
  x += asym::dpp_d0<0x142, 0xA>(x);
  return x + asym::dpp_d0<0x143, 0xC>(x);
}

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

// The part of the chunk at x0, whose tokens a wave holds in v (lane l those of vectors
// l, l + 64, ...); its sum in lane 63.
template <int DT>
STEP_DEV DrawPart draw_chunk(const u4 (&v)[kDrawPer / Row<DT>::VE], int x0, float tau, int lane) {
  constexpr int VE = Row<DT>::VE;
  float l[kDrawPer];
  draw_decode<DT>(v, l);
  // The largest and least logits, by their bits: as integers with a sign the largest
  // one is the largest logit if one is positive; without a sign the least logit, if
  // one is negative.
  int hi = (int)__float_as_uint(l[0]);
  uint32_t lo = __float_as_uint(l[0]);
#pragma unroll
  for (int i = 1; i < kDrawPer; ++i) {
    hi = max(hi, (int)__float_as_uint(l[i]));
    lo = max(lo, __float_as_uint(l[i]));
  }
  hi = draw_max_i(hi);
  lo = draw_max_u(lo);
  const bool nan = hi > (int)kInfBits || lo > kNegInfBits;
  float m = __uint_as_float((uint32_t)hi);
  if (nan) {
    // The conversion to fp64 makes every not-a-number a quiet one, which fmax leaves out.
    double top = -__builtin_huge_val();
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i) top = __builtin_fmax(top, (double)l[i]);
    m = asym::wave_max((float)top);
  } else if (hi < 0) {
    int least = hi;
#pragma unroll
    for (int i = 0; i < kDrawPer; ++i) least = min(least, (int)__float_as_uint(l[i]));
    m = __uint_as_float((uint32_t)asym::wave_min_i(least));
  }
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
    double part[2] = {0.0, 0.0};
    const double km = k.k * (double)m, kl = k.k * (double)((int)lo < 0 ? __uint_as_float(lo) : 0.0f);
    if (__builtin_amdgcn_readfirstlane(!nan && kl - km > -1000.0 && __builtin_fabs(kl) < 0x1p30)) {
      // No weight underflows, so none needs a bound, and k l is below 2^30, so that no
      // difference to m is needed, either: three operations less of 20.
      const double magic = 0x1.8p52 - __builtin_rint(km);
#pragma unroll
      for (int i = 0; i < kDrawPer; ++i) part[i & 1] += k.raised((double)l[i], magic);
      arg = kPlain;
    } else {
      if (k.inf) {
#pragma unroll
        for (int i = 0; i < kDrawPer; ++i) l[i] = k.flat(l[i]);
      }
#pragma unroll
      for (int i = 0; i < kDrawPer; ++i) part[i & 1] += k.weight((double)l[i]);
    }
    sum = draw_sum_d(part[0] + part[1]);
  }
  return DrawPart{sum, m, arg};
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
  const DrawPart q = draw_chunk<DT>(v, x0, tau, lane);
  if (lane == 63) A.part[id] = q;
}

// The same for bf16 rows of many chunks: a logit has 16 bits, so a workgroup computes the
// weights 2^(k l) of all logits with 2^-12 <= |l| < 128 once, into a table of 4864 entries in
// LDS, and looks its chunks' tokens up: 7 operations a token in place of 17, two tokens at a
// time where they have 16 bits.  2^(k l) itself is in fp64's range, so the sum does not wait
// for the chunk's largest logit; that is found beside it (a token's half operation, and 8
// a chunk; 1% of the time of 512 rows of 256000) for the row's level, to which draw_pick
// brings the sums: at 2^(k l) those of a long row could pass fp64's range, and what has
// weight would depend on where the logits lie.  Masked tokens have an entry without weight,
// smaller logits and zeros (one chunk in 16 has one, at a deviation of 3) are computed where
// they stand.  A chunk with other logits, or with |k l| >= 1000, goes the other way
// afterwards, as do those behind two such at a wave's start, rows whose temperature makes
// that likely, and greedy rows.  That order costs rows of such logits throughout: 512 x 256000 of deviation 300 take 114 us (98 in draw_part; 163
// in the table's kernel if every chunk were tried first), 128 x 151936 32 (20).
constexpr int kTableThreads = 1024;       // (with 512 and two tables more a unit 18.1 us for 128 rows, 17.0 so)
constexpr int kTableMost = 64 * (kTableThreads / 64);             // chunks of a workgroup: one bit each a wave
constexpr uint32_t kTableLow = 0x3980u, kTableHigh = 0x4300u;     // bits of 2^-12 and 128
constexpr int kTable = 2 * (int)(kTableHigh - kTableLow);         // entry 2 * (bits - kTableLow) + sign
constexpr int kTableInf = 2 * (0x7F80 - (int)kTableLow) + 1;       // where -inf would stand
constexpr float kTableTau = 0x1p-5f;                              // under it |l| < 21 alone would do
// Chunks of a workgroup that pay for its table (rows of 151936 tokens: 64 of them, 19
// chunks each, 14.2 us with a table and 14.3 without; 96, 30 chunks each, 15.1 and 16.9;
// 2048 rows of 17 chunks 34.0 and 33.0).
constexpr int kTableChunks = 20;
typedef uint16_t h2 __attribute__((ext_vector_type(2)));
typedef int16_t s2 __attribute__((ext_vector_type(2)));

// The largest logit of a chunk without a not-a-number, from each lane's largest bits as
// integers with a sign: if none is positive, the least bits are the largest logit's.
STEP_DEV float draw_top(const u4 (&v)[2], s2 hi) {
  int top = draw_max_i(max((int)hi[0], (int)hi[1]));
  if (top < 0) {
    s2 lo = hi;
#pragma unroll
    for (int i = 0; i < 8; ++i) lo = __builtin_elementwise_min(lo, __builtin_bit_cast(s2, (uint32_t)v[i / 4][i % 4]));
    top = ~draw_max_i(max(~(int)lo[0], ~(int)lo[1]));
  }
  return __uint_as_float((uint32_t)top << 16);
}

__global__ __launch_bounds__(kTableThreads) __attribute__((amdgpu_waves_per_eu(8))) void draw_table_kernel(DrawArgs A) {
  constexpr int DT = ASYMSPEC_BF16, VE = 8, NV = kDrawPer / VE, kWaves = kTableThreads / 64;
  __shared__ double table[kTable + 1];      // and no weight
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = (int)(blockIdx.x / (unsigned)A.P), c0 = (int)(blockIdx.x % (unsigned)A.P) * A.C;
  const int c1 = min(A.S, c0 + A.C);
  const uint16_t* p = (const uint16_t*)A.logits + row * A.row_stride;
  const float tau = A.tau[row];
  const bool tabled = tau >= kTableTau && tau < 0x1p30f;
  DrawPart* out = A.part + (size_t)row * A.S;
  unsigned long long left = ~0ull;        // chunks of the wave that go the other way
  if (tabled) {
    u4 v[NV] = {}, next[NV] = {};
    if (c0 + wave < c1) draw_load<DT>(p, (c0 + wave) * kDrawChunk, A.V, lane, 64, v);
    const DrawScale k(tau, 0.0f);
    for (int i = tid; i < kTable; i += kTableThreads) {
      const uint32_t bits = kTableLow + (uint32_t)(i >> 1) + ((uint32_t)(i & 1) << 15);
      const double l = (double)__uint_as_float(bits << 16);
      table[i] = __builtin_fabs(k.k * l) < 1000.0 ? k.raised(l, 0x1.8p52) : __builtin_nan("");
    }
    if (tid == 0) table[kTable] = 0.0;
    __syncthreads();
    left = 0ull;
    unsigned long long bit = 1ull;
    for (int c = c0 + wave; c < c1; c += kWaves, bit <<= 1) {
      if (c + kWaves < c1) draw_load<DT>(p, (c + kWaves) * kDrawChunk, A.V, lane, 64, next);
      h2 at[kDrawPer / 2], most = {0, 0};
      s2 hi = {-0x8000, -0x8000};
#pragma unroll
      for (int i = 0; i < kDrawPer / 2; ++i) {
        const uint32_t two = v[i / 4][i % 4];
        const h2 w = __builtin_bit_cast(h2, two);
        hi = __builtin_elementwise_max(hi, __builtin_bit_cast(s2, two));
        at[i] = (w - (uint16_t)kTableLow) * (uint16_t)2 + (w >> (uint16_t)15);
        most = __builtin_elementwise_max(most, at[i]);
      }
      double part[2] = {0.0, 0.0};
      bool bad = false;
      auto add = [&]() {
#pragma unroll
        for (int i = 0; i < kDrawPer / 2; ++i) {
          part[0] += table[at[i][0]];
          part[1] += table[at[i][1]];
        }
      };
      if (__all(most[0] < kTable && most[1] < kTable)) {
        add();
      } else {
        // Masked tokens have the entry without weight: 0 in `other` like those in the table.
        h2 other = {0, 0};
#pragma unroll
        for (int i = 0; i < kDrawPer / 2; ++i) {
          const h2 past = __builtin_elementwise_sub_sat(at[i], h2{kTable - 1, kTable - 1});
          other |= __builtin_elementwise_min(past, past ^ (uint16_t)(kTableInf - (kTable - 1)));
          at[i] = __builtin_elementwise_min(at[i], h2{kTable, kTable});
        }
        add();
        if (__any((other[0] | other[1]) != 0)) {
          // the smallest ones and zeros are computed
#pragma unroll
          for (int i = 0; i < kDrawPer; ++i) {
            const uint32_t bits = i & 1 ? v[i / VE][i % VE / 2] >> 16 : v[i / VE][i % VE / 2] & 0xFFFFu;
            const bool tiny = (bits & 0x7FFFu) < kTableLow;
            bad = bad || !(at[i / 2][i % 2] < kTable || tiny || bits == 0xFF80u);
            if (__any(tiny)) part[i & 1] += tiny ? k.raised((double)__uint_as_float(bits << 16), 0x1.8p52) : 0.0;
          }
        }
      }
      part[0] += part[1];
      if (__any(bad || part[0] != part[0])) {
        left |= bit;
        if (left == 3ull) {         // the first two: so will the others
          left = ~0ull;
          break;
        }
      } else {
        const double sum = draw_sum_d(part[0]);
        const float top = draw_top(v, hi);
        if (lane == 63) out[c] = DrawPart{sum, top, kTabled};
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] = next[i];
    }
  }
  for (int c = c0 + wave; c < c1; c += kWaves, left >>= 1) {
    if (left & 1ull) {
      u4 v[NV];
      draw_load<DT>(p, c * kDrawChunk, A.V, lane, 64, v);
      float t = tau;
      asm volatile("" : "+s"(t));      // (nothing of it is kept from chunk to chunk: no register is left for that)
      const DrawPart q = draw_chunk<DT>(v, c * kDrawChunk, t, lane);
      if (lane == 63) out[c] = q;
    }
  }
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
  // A chunk counts if its largest logit has a weight of 2^-1074, fp64's smallest number,
  // or more: below that a chunk's sum can come out as more than nothing where none of its
  // tokens has any weight.
  const float least_m = k.inf ? inf : (float)(k.m + k.least * (744.4400719213812 / 762.0));
  auto weight_of = [&](const DrawPart& q) { return q.m >= least_m ? k.of_part(q) : 0.0; };
  double mine = 0.0, upto, ahead;
  each([&](int, DrawPart& q) {
    const double w = weight_of(q);
    q.sum = w;              // (of a kept part: its weight from here on)
    mine += w;
  });
  asym::wave_scan_d(mine, upto, ahead);
  const double total = __shfl(upto, 63, 64);
  const double target = (double)u * total;
  // the first lane whose sums pass the target; without one, and with a uniform of 1 (which
  // a lane's sums can pass, too: they may be rounded to more than the total), the last
  // lane with weight
  const unsigned long long past = __ballot(u < 1.0f && upto > target && mine > 0.0), some = __ballot(mine > 0.0);
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
