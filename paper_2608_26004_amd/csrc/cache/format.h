// The cache's numbers: 32 channels share a power of two, each is an e4m3 or an e2m1
// number over it.  A power of two makes every step exact but the one rounding to the
// code: the codes do not depend on the order of the arithmetic, and a code times its
// scale is exact in bf16 (at most four bits of mantissa).  gfx950 converts both ways
// with the scale in one instruction for two channels.

#ifndef ASYMSPEC_CACHE_FORMAT_H_
#define ASYMSPEC_CACHE_FORMAT_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../step/row.h"
#include "asymspec_cache.h"

namespace asym_cache {

using asym_step::Row;
using asym_step::u4;

typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s2 __attribute__((ext_vector_type(2)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 32;            // channels of a scale
constexpr uint32_t kNotFinite = 255;  // a scale byte

// Quotients by a number that the host knows, of numbers below 2^31: with 2^(l-1) < d
// <= 2^l and m = ceil(2^(31+l) / d), floor(n m / 2^(31+l)) is floor(n / d), since
// m d exceeds 2^(31+l) by less than 2^l.
struct Div {
  uint32_t d, mul, l;
  Div() = default;
  explicit Div(uint32_t by) : d(by), l(0) {
    while ((1ull << l) < d) ++l;
    mul = (uint32_t)(((1ull << (31 + l)) + d - 1) / d);
  }
  STEP_DEV uint32_t of(uint32_t n) const { return __umulhi(2 * n, mul) >> l; }
  // the quotient; the remainder stays in n
  STEP_DEV uint32_t split(uint32_t& n) const {
    const uint32_t q = of(n);
    n -= q * d;
    return q;
  }
};

STEP_DEV float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// The largest scale byte of numbers, with which the largest code is below 2^128:
// beyond it a block reads as not a number.
template <int BITS>
STEP_DEV constexpr uint32_t most_scale() { return BITS == 8 ? 246 : 252; }

// The scale byte of 32 values whose largest magnitude has these bits: the smallest e
// >= -100 with m <= 448 * 2^e = 1.75 * 2^(e+8), or m <= 6 * 2^e = 1.5 * 2^(e+2).
template <int BITS>
STEP_DEV uint32_t scale_byte(uint32_t most) {
  const int e = (int)(most >> 23) - (BITS == 8 ? 8 : 2) + ((most & 0x7FFFFFu) > (BITS == 8 ? 0x600000u : 0x400000u));
  return e > (int)most_scale<BITS>() ? kNotFinite : (uint32_t)max(e, 27);
}

// Codes of 8 channels over their scale (to the nearest, ties to even; nothing is
// beyond the largest code): 4 bytes, or 8.
template <int BITS>
STEP_DEV u2 encode8(const float* x, float scale) {
  u2 r{0, 0};
  if (BITS == 4) {
    r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[0], x[1], scale, 0);
    r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[2], x[3], scale, 1);
    r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[4], x[5], scale, 2);
    r[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r[0], x[6], x[7], scale, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s2 v{0, 0};
      v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, x[4 * i], x[4 * i + 1], scale, false);
      v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, x[4 * i + 2], x[4 * i + 3], scale, true);
      r[i] = __builtin_bit_cast(uint32_t, v);
    }
  }
  return r;
}

// Two channels of a dword of codes as bf16, the lower channel in the low half: byte
// SEL of 4-bit codes, or half SEL of 8-bit ones.
template <int BITS, int SEL>
STEP_DEV uint32_t decode2(uint32_t codes, float scale) {
  if constexpr (BITS == 4)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, SEL != 0));
}

// 8 channels as bf16.
template <int BITS>
STEP_DEV u4 decode8(const uint32_t* codes, float scale) {
  if constexpr (BITS == 4)
    return u4{decode2<4, 0>(codes[0], scale), decode2<4, 1>(codes[0], scale), decode2<4, 2>(codes[0], scale),
              decode2<4, 3>(codes[0], scale)};
  else
    return u4{decode2<8, 0>(codes[0], scale), decode2<8, 1>(codes[0], scale), decode2<8, 0>(codes[1], scale),
              decode2<8, 1>(codes[1], scale)};
}

// 16 bytes of a row, wherever they begin.  ONCE: the caches keep no line for them.
template <int DT, bool ONCE>
STEP_DEV u4 load_row(const typename Row<DT>::T* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const typename Row<DT>::U*>(p));
  else return asym_step::load_vec<DT>(p);
}

// 8 values of a row, wherever it begins.
template <int DT, bool ONCE = false>
STEP_DEV void load8(const typename Row<DT>::T* p, float* x) {
  if constexpr (DT == ASYMSPEC_BF16) {
    const u4 v = load_row<DT, ONCE>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = Row<DT>::get(v, i);
  } else {
    const u4 v = load_row<DT, ONCE>(p), w = load_row<DT, ONCE>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]), x[4 + i] = __uint_as_float(w[i]);
  }
}

}  // namespace asym_cache

#endif  // ASYMSPEC_CACHE_FORMAT_H_
