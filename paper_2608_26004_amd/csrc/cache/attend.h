// attend_cache: softmax(scale q k^T) v over a paged cache in 8 or 4 bits, in one pass.
//
// Work is cut along the cache: a unit is 128 positions of one head of the cache, for
// all rows of the step and all query heads that read it (16 or 32 of these rows at a
// time: a row tile, and a run is what a request's head has for one).  A workgroup takes
// neighbouring units of a run, of which each of its four waves has 32 positions (or, where
// runs are many and short, each wave takes whole runs by itself).  A wave
// keeps a running reference and sum for each row, so that nothing is exchanged until the
// units end; there the waves' parts meet in LDS, and parts of different workgroups in
// memory, where the last one to leave its part joins them, many of them in two steps (in the
// workgroups' order, whoever is last, so that the answer is always the same).
//
// Both products run on 16x16x32 bf16 matrix instructions: a code times its scale is
// exact in bf16.  For the scores a lane decodes what it loaded, with the order of the
// channels permuted alike on both sides so that a lane's piece of a key is contiguous;
// the scores come out as the second product's operand needs its probabilities (one row a
// lane, eight positions), so that those never move between lanes.  A lane loads the same
// channels of eight positions of the values and pairs them by byte permutes.  The sum of
// the probabilities is a product with ones, of the parts that meet the values.
//
// Bound by memory where requests are long: 128 requests of 7 x 4 rows and 4096 to 8192
// positions, 8 heads of 128 channels in 8 bits, 1.67 GB, take 288 us (5.8 TB/s; a copy
// reaches 5.1), two of 131072 to 262144 positions in 4 bits 93 (4.6 TB/s).  The loads
// alone take 267 and 79 us there, the arithmetic alone 200 and 70: decoding and the
// exponentials keep the vector units 65% busy, the matrix ones 27%.  Where work is small the
// ends weigh as much: 8 requests of 8192 to 16384 positions, 12 rows, 32.5 us, of it 5 the
// waves' parts, 4 the join; one row over 2048 positions 9.8, of it 4 to 5 the join.
//
// What was slower: codes loaded ahead in registers (they spill); two sets of 32 positions
// in flight (104 us for 99 in the second case); eight waves a workgroup (301 for 295 in the first);
// parts made visible by an agent's fences (100 us more a call).  The scaled
// matrix instructions that take codes as they are would save the decoding of keys, but their sums
// hold only 2^-13 of the terms.

#ifndef ASYMSPEC_CACHE_ATTEND_H_
#define ASYMSPEC_CACHE_ATTEND_H_

#include "attend_host.h"
#include "format.h"

namespace asym_cache {

constexpr int kAttendThreads = 256;
constexpr int kUnit = 128;                        // positions of a unit: 32 a wave
constexpr int kAttendFew = 256;                   // workgroups: one a compute unit
constexpr int kMostWorkgroups = 1024;             // four a compute unit at most
constexpr int kLine = 128;                        // bytes of a line of the caches
constexpr uint32_t kNoRow = 0xFFFFFFFFu;
constexpr uint32_t kOnes = 0x3F803F80u;           // two bf16
constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct AttendArgs {
  asymspec_attend a;
  uint32_t* done;       // parts that are left, of each run or group of its parts; zero between calls
  float* sums;          // [2 workgroups][16 MT][dim]: parts of runs, from a line's beginning on
  f2* stats;            // [2 workgroups][16 MT]: reference, sum; the same
  int group;            // query heads of a head of the cache
  int rows;             // R * group
  int row_tiles;        // of 16 MT rows
  int most;             // positions that a table holds
  int workgroups;
  float few;            // one over the units below which 256 workgroups are enough
  float c;              // |scale| log2 e, above 0
  uint32_t flip;        // sign bits of a scale below 0, for the queries
  Div by_size, by_group;
};

// A head's channels in pieces of 128, 64 or 32, of which a lane holds a quarter of a
// key's (contiguous), or a sixteenth of a value's.
template <int D> struct Pieces {
  static constexpr int N = (D == 64 || D == 128) ? 1 : 2;
  static constexpr int width(int i) { return D == 96 ? (i == 0 ? 64 : 32) : D == 192 ? (i == 0 ? 128 : 64) : D == 64 ? 64 : 128; }
  static constexpr int base(int i) { return i == 0 ? 0 : width(0); }
};

// What a request has for its rows: units from `first` on that hold its positions
// [lo, hi), and its number of rows.
struct Range {
  int len, fresh, lo, hi, first, units;
  STEP_DEV Range(const AttendArgs& A, int b)
      : Range(A, min(max(A.a.lengths[b], 0), 0x7FFFFF00),
              A.a.new_tokens != nullptr ? min(max(A.a.new_tokens[b], 0), A.a.R) : A.a.R) {}
  STEP_DEV Range(const AttendArgs& A, int len_, int fresh_) : len(len_), fresh(fresh_) {
    hi = min(len + fresh, A.most);
    lo = A.a.window > 0 ? max(0, len - A.a.window + 1) : 0;
    first = lo / kUnit;
    units = fresh > 0 && hi > lo ? (hi + kUnit - 1) / kUnit - first : 0;
  }
};

STEP_DEV float lanes_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// f over the lanes up to each one, of numbers from 0 on.
template <class F>
STEP_DEV int lanes_upto(int x, F&& f) {
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));      // a row's lanes
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));      // the row's before it
  return f(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));   // the half's
}

STEP_DEV uint32_t bf_pair(float a, float b) {
  const bf2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}
STEP_DEV float bf_low(uint32_t x) { return __uint_as_float(x << 16); }
STEP_DEV float bf_high(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

STEP_DEV f4 mfma(const u4& a, const u4& b, const f4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

// x less the low (0) or the high (1) half of a pair, in one instruction: x - 1 * half -
// 0 * other, exact where the half is x rounded.
template <int HALF>
STEP_DEV float less(float x, uint32_t pair) {
  // (in a register: as a constant of the instruction the low half's -1 was taken for the
  // high half's)
  uint32_t minus;
  if (HALF == 0) asm("s_mov_b32 %0, 0x0000bf80" : "=s"(minus));
  else asm("s_mov_b32 %0, 0xbf800000" : "=s"(minus));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, pair), __builtin_bit_cast(bf2, minus), x, false);
}

// 8 fp32 values as N bf16 parts that add up to them, but for 2^-8N of each.
template <int N>
STEP_DEV void split8(const float* x, u4* parts) {
  float rest[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
  for (int p = 0; p < N; ++p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      parts[p][i] = bf_pair(rest[2 * i], rest[2 * i + 1]);
      if (p + 1 < N) {
        rest[2 * i] = less<0>(rest[2 * i], parts[p][i]);
        rest[2 * i + 1] = less<1>(rest[2 * i + 1], parts[p][i]);
      }
    }
  }
}

// A one in each byte that is an e4m3 code of no number.
STEP_DEV uint32_t nan_codes(uint32_t x) { return (((x & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u; }

template <int BYTES>
STEP_DEV void load_codes(const uint8_t* p, uint32_t* r) {
  if constexpr (BYTES == 1) r[0] = *p;
  else if constexpr (BYTES == 2) r[0] = *(const uint16_t*)p;
  else if constexpr (BYTES == 4) r[0] = *(const uint32_t*)p;
  else if constexpr (BYTES == 8) {
    const u2 v = *(const u2*)p;
    r[0] = v[0], r[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const u4 v = *(const u4*)(p + 16 * i);
      r[4 * i] = v[0], r[4 * i + 1] = v[1], r[4 * i + 2] = v[2], r[4 * i + 3] = v[3];
    }
  }
}

// f(integral constant) for 0 .. N - 1
template <int N, int I = 0, class F>
STEP_DEV void count(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    count<N, I + 1>(f);
  }
}

// Which position of sixteen is row r of a score instruction's result: a lane has rows
// 4 h + i, i = 0 .. 3, and so positions 4 i + h, whose values' rows in LDS are neighbours
// for the four h that read at once.
STEP_DEV int position_of(int r) { return (r & 3) * 4 + (r >> 2); }

// 32 positions' codes and scales on their way through a wave's part of LDS, and as its
// lanes then hold them: with j = lane % 16 and h = lane / 16, a quarter of each piece of
// two keys, those of row j of either sixteen, and a sixteenth of eight values, those of
// rows 4 h + i.
//
// Memory goes to LDS past the registers, 16 bytes a lane and rows in their order.  Where
// a row is 2^k chunks of 16 bytes, a key's chunks are exchanged so that the chunks that
// 16 lanes read at once lie in different banks.  A position's scales are one to three
// parts of 1, 2 or 4 bytes, each in a dword: [part][keys, values][position].
template <int BITS, int D>
struct Codes {
  typedef Pieces<D> P;
  static constexpr int kRow = D * BITS / 8, kScales = D / kBlock;        // bytes of a position
  static constexpr int kChunks = kRow / 16;
  static constexpr int kPart = kScales % 4 == 0 ? 4 : kScales % 2 == 0 ? 2 : 1, kPartsOf = kScales / kPart;
  static constexpr int kValAt = 32 * kRow, kScaleAt = 64 * kRow, kBytes = 64 * kRow + kPartsOf * 256;
  static constexpr int kKey = D * BITS / 128, kVal = BITS / 4 * P::N;     // dwords
  uint32_t key[2][kKey], val[8][kVal] = {};
  uint32_t key_scale[2][P::N], val_scale[8][P::N];

  // Where a chunk of a position's key lies in its row.
  static STEP_DEV int chunk_at(int t, int chunk) {
    constexpr bool kExchanged = (kChunks & (kChunks - 1)) == 0;
    return kExchanged ? chunk ^ ((t & 15) * kChunks / 16) : chunk;
  }

  // row: lane's, of position lane % 32.
  static STEP_DEV void load(const asymspec_cache& c, uint32_t row, uint8_t* lds, int lane) {
#pragma unroll
    for (int n = 0; n < (32 * kChunks + 63) / 64; ++n) {
      const int s = 64 * n + lane, t = s / kChunks, at = s % kChunks;
      if (32 * kChunks % 64 != 0 && s >= 32 * kChunks) break;
      const uint64_t r = (uint32_t)__shfl(row, t);
      to_lds<16>((const uint8_t*)c.keys + (r * kRow + 16 * chunk_at(t, at)), lds + 1024 * n);
      to_lds<16>((const uint8_t*)c.values + (r * kRow + 16 * at), lds + kValAt + 1024 * n);
    }
    const uint8_t* s = (const uint8_t*)(lane < 32 ? c.key_scales : c.value_scales) + (uint64_t)row * kScales;
#pragma unroll
    for (int u = 0; u < kPartsOf; ++u) to_lds<kPart>(s + kPart * u, lds + kScaleAt + 256 * u);
  }

  template <int BYTES>
  static STEP_DEV void to_lds(const uint8_t* from, uint8_t* to) {
    typedef const __attribute__((address_space(1))) void* Global;
    typedef __attribute__((address_space(3))) void* Shared;
    // (codes are read once: told so (the 2), the caches keep no lines for them, and 128 x 7 rows
    // over 8192 positions in 8 bits take 299 us instead of 331)
    if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds((Global)from, (Shared)to, 16, 0, 2);
    else if constexpr (BYTES == 4) __builtin_amdgcn_global_load_lds((Global)from, (Shared)to, 4, 0, 0);
    else if constexpr (BYTES == 2) __builtin_amdgcn_global_load_lds((Global)from, (Shared)to, 2, 0, 0);
    else __builtin_amdgcn_global_load_lds((Global)from, (Shared)to, 1, 0, 0);
  }

  STEP_DEV void take(const uint8_t* lds, int j, int h) {
    const int t = position_of(j);
    count<P::N>([&](auto p) {
      constexpr int w = P::width(p), from = P::base(p), kOwn = w * BITS / 32, kSixteenth = w * BITS / 128;
      const int at = from * BITS / 8 + h * kOwn, block = (from + h * (w / 4)) / kBlock;
#pragma unroll
      for (int a = 0; a < 2; ++a) {
        const uint8_t* row = lds + (16 * a + t) * kRow;
        if constexpr (kOwn > 16) {
#pragma unroll
          for (int i = 0; i < kOwn / 16; ++i)
            load_codes<16>(row + 16 * chunk_at(t, at / 16 + i), &key[a][from * BITS / 128 + 4 * i]);
        } else {
          load_codes<kOwn>(row + 16 * chunk_at(t, at / 16) + at % 16, &key[a][from * BITS / 128]);
        }
        key_scale[a][p] = lds[kScaleAt + (block / kPart) * 256 + block % kPart + 4 * (16 * a + t)];
      }
      const int vblock = (from + j * (w / 16)) / kBlock;
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int a = t / 4, i = t % 4;
        load_codes<kSixteenth>(lds + kValAt + (16 * a + 4 * i + h) * kRow + from * BITS / 8 + j * kSixteenth,
                               &val[t][p * (BITS / 4)]);
        val_scale[t][p] = lds[kScaleAt + (vblock / kPart) * 256 + vblock % kPart + 4 * (32 + 16 * a + 4 * i + h)];
      }
    });
  }
};

// The kernel's arguments where they lie, loaded as they are needed: held from its start, they
// are more than the scalar registers, and spill.  (One row over 2048 positions 9.7 us, so 10.1.)
STEP_DEV const AttendArgs& arguments() {
  auto p = (const __attribute__((address_space(4))) AttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const AttendArgs*)p;
}

// The thread's number, from its wave's: neither it nor what is computed from it waits in
// registers.
STEP_DEV int thread_again(int wave) {
  int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
  asm volatile("" : "+v"(lane));
  return 64 * wave + lane;
}

// N (2 or 4) channels of a row from its sums, and its lse.
template <int DT, int N = 4>
STEP_DEV void finish(const AttendArgs& A, int b, int r, int q_head, int dim, int ch, float ref, float sum, const f4& o) {
  typedef typename Row<DT>::T T;
  const int64_t at = ((int64_t)b * A.a.R + r) * A.a.q_heads + q_head;
  const bool none = sum == 0.f;
  const float over = 1.f / sum;
  float y[4];
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] = none ? 0.f : o[e] * over;
  T* out = (T*)A.a.out + at * dim + ch;
  if constexpr (DT == ASYMSPEC_BF16 && N == 2) *(uint32_t*)out = bf_pair(y[0], y[1]);
  else if constexpr (DT == ASYMSPEC_BF16) *(u2*)out = u2{bf_pair(y[0], y[1]), bf_pair(y[2], y[3])};
  else if constexpr (N == 2) *(f2*)out = f2{y[0], y[1]};
  else *(f4*)out = f4{y[0], y[1], y[2], y[3]};
  if (ch == 0 && A.a.lse != nullptr) A.a.lse[at] = none ? -INFINITY : (ref + log2f(sum)) * kLn2;
}

// Two floats for another workgroup, which may be on another die: stored past both
// caches.  Each place has lines of its own (the first begins on one, and they are whole
// lines), which one workgroup stores and one loads in a call, behind the counter, so that
// no cache holds them from before: a line that two places share would be in a die's cache
// once one of them is joined there, and the other be read as it was then.  (An agent's
// fences write back and drop a die's whole cache, which cost 100 us a call.)
STEP_DEV void leave(float* p, float x, float y) {
  const uint64_t v = (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x);
  __hip_atomic_store((uint64_t*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}
template <class T>
STEP_DEV T left(const T* p) { return __builtin_nontemporal_load(p); }

// Which parts are joined, and where they are: a workgroup has two places, the second for a
// run that it begins.  Of `parts` workgroups, `apart` from w0 on, the first one's part is in
// its second place (`second`) and the others' in their first, or the other way about.  The
// result is the rows' answer, or a part in place `to`.
struct Join {
  int w0, parts, apart, second, other, to;
  STEP_DEV int place(int k) const { return 2 * (w0 + k * apart) + (k == 0 ? second : other); }
};

// Joins parts of a run.  A thread has eight channels of a row, and with few rows a share of
// the parts, of which it loads four at a time (two at once take up to a quarter longer, eight up
// to 2.5 us: this code runs once, and is fetched for it).
template <int DT, int D, int MT>
STEP_DEV void join(const AttendArgs& A, const Range& range, int b, int head, int row0, const Join& J, int tid,
                   uint8_t* lds) {
  constexpr int kEights = D / 8, kAtOnce = 4;
  const int rows = min(16 * MT, A.rows - row0), items = rows * kEights, parts = J.parts;
  const int shares = max(1, kAttendThreads / items);
  f4* sums = (f4*)lds;                                    // [2][threads]
  f2* stats = (f2*)(lds + kAttendThreads * 32);
  for (int i0 = 0; i0 < items; i0 += kAttendThreads) {
    const int i = i0 + tid, share = shares > 1 ? i / items : 0, item = i - share * items;
    const bool is = shares > 1 ? share < shares : i < items;
    const int row = is ? item / kEights : 0, ch = is ? (item - row * kEights) * 8 : 0;
    float top = -INFINITY, total = 0.f;
    f4 o[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    for (int k0 = is ? share : parts; k0 < parts; k0 += kAtOnce * shares) {
      f4 x[kAtOnce][2];
      f2 st[kAtOnce];
      count<kAtOnce>([&](auto c) {
        const int k = min(k0 + c * shares, parts - 1);
        const int64_t at = (int64_t)J.place(k) * (16 * MT) + row;
        st[c] = left(A.stats + at);
        const f4* from = (const f4*)(A.sums + at * D + ch);
        x[c][0] = left(from);
        x[c][1] = left(from + 1);
      });
      float next = top;
      count<kAtOnce>([&](auto c) {
        if (k0 + c * shares >= parts) st[c] = f2{-INFINITY, 0.f};
        next = fmaxf(next, st[c][0]);
      });
      const float at = next == -INFINITY ? 0.f : next, f = __builtin_amdgcn_exp2f(top - at);
      top = next;
      total *= f;
      o[0] *= f;
      o[1] *= f;
      count<kAtOnce>([&](auto c) {
        // (a part without a reference has no sums but, where its scores were no numbers, those)
        const bool none = st[c][0] == -INFINITY && st[c][1] == 0.f;
        const float f = none ? 0.f : st[c][0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st[c][0] - at);
        total += st[c][1] * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[0][e] = none ? o[0][e] : fmaf(x[c][0][e], f, o[0][e]);
          o[1][e] = none ? o[1][e] : fmaf(x[c][1][e], f, o[1][e]);
        }
      });
    }
    if (shares > 1) {
      if (is) {
        sums[tid] = o[0];
        sums[kAttendThreads + tid] = o[1];
        stats[tid] = f2{top, total};
      }
      __syncthreads();
      if (is && share == 0) {
        for (int k = 1; k < shares; ++k) {
          const f2 st = stats[k * items + item];
          const float next = fmaxf(top, st[0]), at = next == -INFINITY ? 0.f : next;
          const float f = __builtin_amdgcn_exp2f(top - at), g = __builtin_amdgcn_exp2f(st[0] - at);
          top = next;
          total = total * f + st[1] * g;
          o[0] = o[0] * f + sums[k * items + item] * g;
          o[1] = o[1] * f + sums[kAttendThreads + k * items + item] * g;
        }
      }
    }
    if (is && share == 0 && J.to >= 0) {
      const int64_t at = (int64_t)J.to * (16 * MT) + row;
      for (int e = 0; e < 2; ++e) {
        leave(A.sums + at * D + ch + 4 * e, o[e][0], o[e][1]);
        leave(A.sums + at * D + ch + 4 * e + 2, o[e][2], o[e][3]);
      }
      if (ch == 0) leave((float*)&A.stats[at], top, total);
    } else if (is && share == 0) {
      uint32_t g = (uint32_t)(row0 + row);
      const int r = (int)A.by_group.split(g);
      const bool fresh = r < range.fresh;
      for (int e = 0; e < 2; ++e)
        finish<DT>(A, b, r, head * A.group + (int)g, D, ch + 4 * e, fresh ? top : -INFINITY, fresh ? total : 0.f,
                   e == 0 ? o[0] : o[1]);
    }
  }
}

// The whole part of a / b, the same in all lanes; a is below 2^42.  (A quotient that is not
// whole is 1 / b and more below the next whole number, 2^-42 of it: a rounding does not reach it.)
STEP_DEV int over(double a, int b) { return __builtin_amdgcn_readfirstlane((int)(a / b)); }

STEP_DEV int pieces_of(int units, int most) { return most == 1 ? units : (units + most - 1) / most; }

template <int BITS, int DT, int D, int MT>
__global__ __launch_bounds__(kAttendThreads, attend_waves(BITS, DT == ASYMSPEC_BF16, D, MT)) void attend_kernel(AttendArgs) {
  const AttendArgs& A = arguments();
  typedef Pieces<D> P;
  typedef Codes<BITS, D> C;
  typedef typename Row<DT>::T T;
  constexpr int kParts = DT == ASYMSPEC_BF16 ? 1 : 3;      // of a query
  constexpr int kProb = DT == ASYMSPEC_BF16 ? 2 : 3;       // of a probability
  constexpr int kSteps = D / 32, kTiles = D / 16;          // matrix instructions along a head
  constexpr int kStride = D + 4;                           // of a row in LDS: 16 rows, all banks
  static_assert(16 * MT * sizeof(f2) % kLine == 0 && 16 * MT * D * sizeof(float) % kLine == 0, "places are whole lines");
  // codes on their way, and at the end of a run the waves' sums
  constexpr int kJoinBytes = kAttendThreads * 40;
  constexpr int kSumBytes = 4 * 16 * kStride * 4 > kJoinBytes ? 4 * 16 * kStride * 4 : kJoinBytes, kLds = kSumBytes > 4 * C::kBytes ? kSumBytes : 4 * C::kBytes;
  __shared__ __align__(16) uint8_t lds[kLds];
  float (*buf)[16][kStride] = (float (*)[16][kStride])lds;
  __shared__ float2 stat[4][16];
  __shared__ int totals[3][4], most_units[4], found[4], list[3], shared_by[2], is_last;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int heads = A.a.cache.heads, per_unit = heads * A.row_tiles;

  // The requests' first units in the list, and the request of this workgroup's first one.  Each
  // workgroup counts all requests' units, with as many threads, up to three times over: one row
  // of one head over one position takes 6.4 us for 256 requests, 8.2 for 1024, 16.8 for 4096.
  const int each = (A.a.B + kAttendThreads - 1) / kAttendThreads;
  const Range lane_first(A, min(tid * each, A.a.B - 1));    // (a thread's only one, up to 256 requests)
  const int me = blockIdx.x;
  int all = 0, items = 0, G = 0, even = 0;
  // Where there are workgroups for all runs if each has at most `most` units of one, that
  // is what they have; else (0) even shares of the list, which begin and end within runs and cost
  // a workgroup the ends of two.  (8 requests of 8192 to 16384 positions 32.5 us, with even
  // shares 33.4; windows of 1024 positions, 32 requests of 16 heads in fp32, 16.8 and 17.8.)
  int most = 0, mine = 0, start = 0;
  bool solo = false;
#pragma nounroll
  for (int i = 0; i < 3; ++i) {
    const int m = i == 0 ? 1 : i == 1 ? even : even + 1 + even / 16;
    int own = tid * each < A.a.B ? pieces_of(lane_first.units, m) * per_unit : 0, longest = lane_first.units;
    for (int k = 1; k < each; ++k)
      if (tid * each + k < A.a.B) {
        const int n = Range(A, tid * each + k).units;
        own += pieces_of(n, m) * per_unit;
        longest = max(longest, n);
      }
    const int upto = lanes_upto(own, [](int x, int y) { return x + y; });
    longest = lanes_upto(longest, [](int x, int y) { return max(x, y); });
    if (lane == 63) totals[i][wave] = upto, most_units[wave] = longest;
    __syncthreads();
    int ahead = upto - own;
    items = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int t = totals[i][w];
      if (w < wave) ahead += t;
      items += t;
    }
    items = __builtin_amdgcn_readfirstlane(items);
    if (i == 0) {
      all = items;
      // a part more of a run is as many bytes more for the one that joins them
      G = __builtin_amdgcn_readfirstlane(min((float)all * A.few < 1.f ? min(A.workgroups, kAttendFew) : A.workgroups, all));
      even = G > 0 ? over((double)all + G - 1, G) : 0;
      // Many short runs: a wave does whole ones by itself, 4 steps of 32 positions a unit and
      // some 4 for the rest, where a workgroup takes one step a unit and the time of 8 to
      // load queries and tables and to join its waves.  (122 requests of 8 positions, 5 heads of
      // 256 channels in 8 bits: 10.0 us, by workgroups 20.2; 256 of 100, 16 heads of 128 in
      // 4 bits 23 and 33; but 90 of 700, 8 heads 26.1 and 20.4, and the rule takes workgroups.)
      const int longest = max(max(most_units[0], most_units[1]), max(most_units[2], most_units[3]));
      const float runs = (float)(A.a.B * per_unit), waves = 4.f * (float)A.workgroups;
      solo = __builtin_amdgcn_readfirstlane(
          all > G && ceilf(runs / waves) * (float)(longest + 1) * waves < (float)all + 8.f * runs);
      if (even == 1) most = 1;
    } else if (items > G) {
      continue;
    } else {
      most = m;
    }
    mine = own;
    start = ahead;
    if (even <= 1 || solo || i > 0) break;
  }
  int u = 0, end = 0;
  if (solo) {
    const int slot = 4 * me + wave, runs = A.a.B * per_unit;
    u = over((double)slot * runs, 4 * A.workgroups);
    end = over((double)(slot + 1) * runs, 4 * A.workgroups);
  } else if (most == 0 && me < G) {
    u = over((double)me * all, G);
    end = over((double)(me + 1) * all, G);
  }
  const int item = most > 0 ? me : u;
  if (!solo && item >= start && item < start + mine) {
    Range r = lane_first;
    int b = tid * each;
    for (int n; item >= start + (n = pieces_of(r.units, max(most, 1)) * per_unit);) {
      start += n;
      r = Range(A, ++b);
    }
    found[0] = b, found[1] = start, found[2] = r.len, found[3] = r.fresh;
  }
  __syncthreads();
  int b = __builtin_amdgcn_readfirstlane(found[0]), base = __builtin_amdgcn_readfirstlane(found[1]);
  Range range(A, __builtin_amdgcn_readfirstlane(found[2]), __builtin_amdgcn_readfirstlane(found[3]));
  // (what a run's end needs waits in LDS)
  if (most > 0 && me < items) {
    const int n = range.units, pieces = __builtin_amdgcn_readfirstlane(pieces_of(n, most));
    const int run = over(me - base, pieces), piece = (me - base) - run * pieces;
    if (tid == 0) shared_by[0] = me - piece, shared_by[1] = pieces;
    base = 0;                                             // (units of this request)
    u = run * n + over((double)n * piece, pieces);
    end = run * n + over((double)n * (piece + 1), pieces);
  } else if (tid == 0) {
    list[0] = all, list[1] = G;
  }
  if (tid == 0) list[2] = most;

  if (solo) b = -1;
  while (u < end) {
    const int lane = thread_again(wave) & 63, j = lane & 15, h = lane >> 4;
    int run, from;
    if (solo) {
      const int at = over(u, per_unit);
      if (at != b) range = Range(A, b = at);
      run = u - b * per_unit;
      from = 0;
      if (range.units == 0) {
        ++u;
        continue;
      }
    } else {
      if (u >= base + range.units * per_unit) {
        base += range.units * per_unit;
        range = Range(A, ++b);
        continue;
      }
      run = over(u - base, range.units);
      from = (u - base) - run * range.units;
    }
    const int n = range.units, to = solo ? n : min(n, from + (end - u));
    const int head = run / A.row_tiles, row0 = (run - head * A.row_tiles) * (16 * MT);
    u += solo ? 1 : to - from;

    // the queries of this lane's rows, and the positions that these see
    u4 q[MT][kParts][kSteps];
    int see_lo[MT], see_hi[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      uint32_t g = (uint32_t)(row0 + 16 * m + j);
      const bool is = (int)g < A.rows;
      const int r = is ? (int)A.by_group.split(g) : 0;
      if (!is) g = 0;
      see_hi[m] = range.len + r;
      see_lo[m] = A.a.window > 0 ? range.len + r - A.a.window + 1 : 0;
      const T* x = (const T*)A.a.q.at + (b * A.a.q.request + r * A.a.q.row + (head * A.group + (int)g) * A.a.q.head);
      count<P::N>([&](auto p) {
        constexpr int w = P::width(p), base_ch = P::base(p);
#pragma unroll
        for (int s = 0; s < w / 32; ++s) {
          const T* y = x + base_ch + h * (w / 4) + 8 * s;
          if constexpr (DT == ASYMSPEC_BF16) {
            q[m][0][base_ch / 32 + s] = asym_step::load_vec<DT>(y) ^ A.flip;
          } else {
            float f[8];
            u4 parts[kParts];
            load8<DT>(y, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(__float_as_uint(f[e]) ^ A.flip);
            split8<kParts>(f, parts);
#pragma unroll
            for (int k = 0; k < kParts; ++k) q[m][k][base_ch / 32 + s] = parts[k];
          }
        }
      });
    }
    // positions that every row sees
    const int full_hi = range.len, full_lo = A.a.window > 0 ? range.len + range.fresh - A.a.window : 0;

    f4 acc[MT][kTiles];
    f4 sum[MT];                                            // (each of its four the same)
    float ref[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      ref[m] = -INFINITY;
      sum[m] = f4{0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < kTiles; ++e) acc[m][e] = f4{0, 0, 0, 0};
    }

    // Row of the cache of the lane's position, of 32 from p on: the table's entry, and
    // what becomes of it once it is there.
    auto entry = [&](int p) -> int {
      const int position = p + (lane & 31);
      return position < A.most ? A.a.block_table[(int64_t)b * A.a.max_blocks + A.by_size.of((uint32_t)position)] : -1;
    };
    auto row_of = [&](int block, int p) -> uint32_t {
      uint32_t offset = (uint32_t)(p + (lane & 31));
      A.by_size.split(offset);
      if ((uint32_t)block >= (uint32_t)A.a.cache.blocks) return kNoRow;
      return ((uint32_t)block * (uint32_t)heads + (uint32_t)head) * (uint32_t)A.a.cache.block_size + offset;
    };
    uint8_t* const own = lds + wave * C::kBytes;

    // What 32 positions add.
    auto use = [&](C& c, int p, uint32_t row, uint32_t there) {
      const bool full = there == 0xFFFFFFFFu && p + 31 <= full_hi && p >= full_lo;

      // scores of positions 16 a + 4 i + h
      f4 s[MT][2];
#pragma unroll
      for (int m = 0; m < MT; ++m) s[m][0] = s[m][1] = f4{0, 0, 0, 0};
      count<P::N>([&](auto pc) {
        constexpr int w = P::width(pc), base_ch = P::base(pc);
        const float scale[2] = {scale_of(c.key_scale[0][pc]), scale_of(c.key_scale[1][pc])};
#pragma unroll
        for (int st = 0; st < w / 32; ++st) {
          u4 k[2];
#pragma unroll
          for (int a = 0; a < 2; ++a) k[a] = decode8<BITS>(&c.key[a][base_ch * BITS / 128 + st * (BITS / 4)], scale[a]);
          // (two sums in turn: a matrix instruction waits for the one before it on its own)
#pragma unroll
          for (int x = 0; x < kParts; ++x)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
              for (int a = 0; a < 2; ++a) s[m][a] = mfma(k[a], q[m][x][base_ch / 32 + st], s[m][a]);
        }
      });
      // the largest of the scale bytes
      uint32_t most_key = 0, most_val = 0;
#pragma unroll
      for (int x = 0; x < P::N; ++x) {
#pragma unroll
        for (int a = 0; a < 2; ++a) most_key = max(most_key, c.key_scale[a][x]);
#pragma unroll
        for (int t = 0; t < 8; ++t) most_val = max(most_val, c.val_scale[t][x]);
      }
      bool bad_val = most_val > most_scale<BITS>();
      if (BITS == 8 && !full) {
        // (where all rows see all positions, the products spread a code that is not a
        // number as they should)
        uint32_t any = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int x = 0; x < C::kVal; ++x) any |= nan_codes(c.val[t][x]);
        bad_val |= any != 0;
      }
      if (__any(most_key > most_scale<BITS>())) {
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          uint32_t of = 0;
#pragma unroll
          for (int x = 0; x < P::N; ++x) {
            const uint64_t lanes = __ballot(c.key_scale[a][x] > most_scale<BITS>());
            of |= (uint32_t)(lanes | lanes >> 16 | lanes >> 32 | lanes >> 48) & 0xFFFFu;
          }
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if ((of >> (4 * h + i)) & 1u) s[m][a][i] = NAN;
        }
      }
      if (!full) {
        const uint32_t mine = there >> h;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            const int k = 16 * (t / 4) + 4 * (t % 4), at = p + h + k;
            if (!((mine >> k) & 1u) || at > see_hi[m] || at < see_lo[m]) s[m][t / 4][t % 4] = -INFINITY;
          }
      }

      // probabilities beside the row's reference, which follows its largest score once
      // that is 2^8 above it
      u4 prob[MT][kProb];
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        float top = s[m][0][0];
#pragma unroll
        for (int t = 1; t < 8; ++t) top = fmaxf(top, s[m][t / 4][t % 4]);
        top *= A.c;
        if (__any(top > ref[m] + 8.f)) {
          const float next = fmaxf(ref[m], lanes_max(top));
          const float f = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref[m] - next);
          ref[m] = next;
          sum[m] *= f;
#pragma unroll
          for (int e = 0; e < kTiles; ++e) acc[m][e] *= f;
        }
        const float at = ref[m] == -INFINITY ? 0.f : ref[m];
        float w[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) w[t] = __builtin_amdgcn_exp2f(fmaf(s[m][t / 4][t % 4], A.c, -at));
        split8<kProb>(w, prob[m]);
        // (the sum of what is multiplied with the values)
#pragma unroll
        for (int k = 0; k < kProb; ++k) sum[m] = mfma(u4{kOnes, kOnes, kOnes, kOnes}, prob[m][k], sum[m]);
      }

      float vs[8][P::N];
#pragma unroll
      for (int t = 0; t < 8; ++t)
#pragma unroll
        for (int x = 0; x < P::N; ++x) vs[t][x] = scale_of(c.val_scale[t][x]);
      if (__any(bad_val)) {
        // Where a row sees a value that is not a number, the sum becomes one; where it
        // does not, the value must not count: a probability of 0 would not hide it.
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int x = 0; x < P::N; ++x)
            if (c.val_scale[t][x] > most_scale<BITS>()) vs[t][x] = 0.f;
        if (BITS == 8) {
#pragma unroll
          for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int x = 0; x < C::kVal; ++x) c.val[t][x] &= ~(nan_codes(c.val[t][x]) * 0xFFu);
        }
        const uint32_t safe = row == kNoRow ? 0 : row;
        for (int k = 0; k < 32; ++k) {
          if (!((there >> k) & 1u)) continue;
          const uint32_t r = __shfl(safe, k);
          const uint8_t* scales = (const uint8_t*)A.a.cache.value_scales + (uint64_t)r * (D / kBlock);
          const uint8_t* codes = (const uint8_t*)A.a.cache.values + (uint64_t)r * (D * BITS / 8);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            if (p + k > see_hi[m] || p + k < see_lo[m]) continue;
            count<P::N>([&](auto pc) {
              constexpr int w = P::width(pc), base_ch = P::base(pc);
#pragma unroll
              for (int e = 0; e < w / 16; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int ch = base_ch + (4 * h + i) * (w / 16) + e;
                  if (scales[ch / kBlock] > most_scale<BITS>() || (BITS == 8 && (codes[ch] & 0x7F) == 0x7F))
                    acc[m][base_ch / 16 + e][i] = NAN;
                }
            });
          }
        }
      }
      count<P::N>([&](auto pc) {
        constexpr int w = P::width(pc), base_ch = P::base(pc);
        count<w / 32>([&](auto e2) {
          constexpr int kSel = BITS == 4 ? e2 : e2 % 2, kReg = pc * (BITS / 4) + (BITS == 4 ? 0 : e2 / 2);
          uint32_t x[8];
#pragma unroll
          for (int t = 0; t < 8; ++t) x[t] = decode2<BITS, kSel>(c.val[t][kReg], vs[t][pc]);
          u4 even, odd;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            even[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
            odd[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
          }
#pragma unroll
          for (int k = 0; k < kProb; ++k)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              acc[m][base_ch / 16 + 2 * e2] = mfma(even, prob[m][k], acc[m][base_ch / 16 + 2 * e2]);
              acc[m][base_ch / 16 + 2 * e2 + 1] = mfma(odd, prob[m][k], acc[m][base_ch / 16 + 2 * e2 + 1]);
            }
        });
      });
    };

    // While 32 positions are used the next ones' codes are on their way to LDS, and the
    // table's entries of those behind them.
    const int step = solo ? 32 : kUnit;
    int p = solo ? range.lo & ~31 : (range.first + from) * kUnit + 32 * wave;
    const int p_end = min(range.hi, (range.first + to) * kUnit);
    if (p + 32 <= range.lo) p += step;
    if (p < p_end) {
      uint32_t row = row_of(entry(p), p);
      C::load(A.a.cache, row == kNoRow ? 0 : row, own, lane);
      int next = p + step < p_end ? entry(p + step) : -1;
      for (;;) {
        C c;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        // (a wave whose codes are there asks for the next ones ahead of the others' arithmetic)
        __builtin_amdgcn_s_setprio(3);
        c.take(own, j, h);
        const uint32_t there = (uint32_t)__ballot(row != kNoRow), used = row;
        const int at = p;
        p += step;
        if (p < p_end) {
          // (what is read of it has arrived in registers before it is written again)
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          row = row_of(next, p);
          C::load(A.a.cache, row == kNoRow ? 0 : row, own, lane);
          if (p + step < p_end) next = entry(p + step);
        }
        __builtin_amdgcn_s_setprio(0);
        use(c, at, used, there);
        if (p >= p_end) break;
      }
    }

    if (solo) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        uint32_t g = (uint32_t)(row0 + 16 * m + j);
        if ((int)g >= A.rows) continue;
        const int r = (int)A.by_group.split(g);
        const bool fresh = r < range.fresh;
        count<P::N>([&](auto pc) {
          constexpr int w = P::width(pc), base_ch = P::base(pc), N = w / 16 < 4 ? w / 16 : 4;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < w / 16; e += N) {
              f4 o{0, 0, 0, 0};
#pragma unroll
              for (int x = 0; x < N; ++x) o[x] = acc[m][base_ch / 16 + e + x][i];
              finish<DT, N>(A, b, r, head * A.group + (int)g, D, base_ch + (4 * h + i) * (w / 16) + e,
                            fresh ? ref[m] : -INFINITY, fresh ? sum[m][0] : 0.f, o);
            }
        });
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      continue;
    }

    // The four waves' parts of the run, and what becomes of them.
    const bool complete = from == 0 && to == n;
    const int tid = thread_again(wave);
    const int slot = 2 * me + (from > 0 ? 0 : 1);       // (a run that an earlier workgroup began comes first)
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      __syncthreads();
      if (h == 0) stat[wave][j] = make_float2(ref[m], sum[m][0]);
      count<P::N>([&](auto pc) {
        constexpr int w = P::width(pc), base_ch = P::base(pc);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < w / 16; ++e)
            buf[wave][j][base_ch + (4 * h + i) * (w / 16) + e] = acc[m][base_ch / 16 + e][i];
      });
      __syncthreads();
      for (int i = tid; i < 16 * (D / 4); i += kAttendThreads) {
        const int rr = i / (D / 4), ch = (i - rr * (D / 4)) * 4;
        uint32_t g = (uint32_t)(row0 + 16 * m + rr);
        if ((int)g >= A.rows) continue;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[w][rr].x);
        float total = 0.f;
        f4 o{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float f = stat[w][rr].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat[w][rr].x - top);
          // (a wave that saw nothing has no part, and a sum of one that is not a number stays)
          total += stat[w][rr].y * f;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += buf[w][rr][ch + e] * f;
        }
        if (!complete) {
          const int64_t at = (int64_t)slot * (16 * MT) + 16 * m + rr;
          leave(A.sums + at * D + ch, o[0], o[1]);
          leave(A.sums + at * D + ch + 2, o[2], o[3]);
          if (ch == 0) leave((float*)&A.stats[at], top, total);
        } else {
          const int r = (int)A.by_group.split(g);
          finish<DT>(A, b, r, head * A.group + (int)g, D, ch, r < range.fresh ? top : -INFINITY,
                     r < range.fresh ? total : 0.f, o);
        }
      }
    }
    Join J{0, 1, 1, 1, 0, -1};
    int counter = 0, w0 = 0, group = 0, groups = 1;
    if (!complete) {
      const int most = __builtin_amdgcn_readfirstlane(list[2]);
      if (most > 0) {
        w0 = __builtin_amdgcn_readfirstlane(shared_by[0]);
        J.parts = __builtin_amdgcn_readfirstlane(shared_by[1]);
        counter = w0;
      } else {
        // the workgroups of its first and last unit: the last w with w all / G <= unit (so the
        // first one begins the run, and has its part in its second place)
        const int all = __builtin_amdgcn_readfirstlane(list[0]), G = __builtin_amdgcn_readfirstlane(list[1]);
        const int u0 = base + run * n;
        w0 = over((u0 + 1.) * G - 1, all);
        J.parts = over(((double)u0 + n) * G - 1, all) - w0 + 1;
        counter = (b * heads + head) * A.row_tiles + row0 / (16 * MT);
      }
      J.w0 = w0;
      // Many parts are joined in groups first, each by the last to leave one of its own, and the
      // last group to be joined joins the groups'.  A group's result goes to its first
      // workgroup's other place, which is free: each workgroup has a part of one run alone.  (12
      // rows over 131072 positions of one head 21 us, at once 50; 4 rows over 8 heads 44.)
      if (most > 0 && J.parts > 32) {
        const int shares = max(1, kAttendThreads / (min(16 * MT, A.rows - row0) * (D / 8)));
        if (J.parts > 8 + 24 * shares) {
          group = __builtin_amdgcn_readfirstlane((int)sqrtf((float)J.parts));
          const int first = over(me - w0, group) * group;
          groups = over(J.parts + group - 1, group);
          J = Join{w0 + first, min(group, J.parts - first), 1, first == 0, 0, 2 * (w0 + first) + (first != 0)};
          counter = kMostWorkgroups + w0 + first;
        }
      }
      // (a part is in memory before it is counted, whichever wave stored it)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __syncthreads();                                      // (codes go there again)
    if (!complete) {
#pragma nounroll
      for (;;) {
        if (tid == 0) {
          // (neighbours' counters lie in different lines: many workgroups count at once)
          uint32_t* const done = A.done + ((counter & 4095) * 32 + (counter >> 12));
          is_last = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)(J.parts - 1);
          if (is_last) __hip_atomic_store(done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (!is_last) break;
        join<DT, D, MT>(A, range, b, head, row0, J, tid, lds);
        if (J.to < 0) break;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        J = Join{w0, groups, group, 0, 1, -1};
        counter = w0;
      }
      __syncthreads();
    }
  }

  // rows of requests without a unit
  for (int b = me; b < A.a.B; b += (int)gridDim.x) {
    if (Range(A, b).units > 0) continue;
    for (int i = thread_again(wave); i < A.a.R * A.a.q_heads * (D / 4); i += kAttendThreads) {
      const int at = i / (D / 4);
      finish<DT>(A, b, at / A.a.q_heads, at % A.a.q_heads, D, (i - at * (D / 4)) * 4, -INFINITY, 0.f, f4{0, 0, 0, 0});
    }
  }
}

}  // namespace asym_cache

#endif  // ASYMSPEC_CACHE_ATTEND_H_
