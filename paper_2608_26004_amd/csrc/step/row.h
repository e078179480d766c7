// Rows of logits as the operators around the decision step read them: 16-byte
// vectors of VE tokens, counted from the row's first token.  Rows may start
// anywhere (odd vocabularies, strided views), so the vectors are loaded and
// stored with an element's alignment only.

#ifndef ASYMSPEC_STEP_ROW_H_
#define ASYMSPEC_STEP_ROW_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "asymspec_step.h"

#define STEP_DEV __device__ __forceinline__

namespace asym_step {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kInfBits = 0x7F800000u;
constexpr uint32_t kNegInfBits = 0xFF800000u;

template <int DT> struct Row;

template <> struct Row<ASYMSPEC_BF16> {
  static constexpr int VE = 8;
  typedef uint16_t T;
  typedef uint32_t U __attribute__((ext_vector_type(4), aligned(2)));
  static STEP_DEV float get(const u4& v, int e) {
    return __uint_as_float((e & 1) ? (v[e >> 1] & 0xFFFF0000u) : (v[e >> 1] << 16));
  }
  // to the nearest bf16, ties to even: the one rounding of a result
  static STEP_DEV uint32_t bits(float f) {
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7FFFFFFFu) > kInfBits) return (u >> 16) | 0x40u;
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
  }
  static STEP_DEV void put_bits(u4& v, int e, uint32_t b) {
    v[e >> 1] = (e & 1) ? ((v[e >> 1] & 0xFFFFu) | (b << 16)) : ((v[e >> 1] & 0xFFFF0000u) | b);
  }
  static STEP_DEV void put(u4& v, int e, float f) { put_bits(v, e, bits(f)); }
  static STEP_DEV u4 neg_inf() { return u4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}; }
  // -inf in place of each token e whose bit of `allowed` is clear
  static STEP_DEV void mask(u4& v, uint32_t allowed) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = 0u - ((allowed >> (2 * i)) & 1u), hi = 0u - ((allowed >> (2 * i + 1)) & 1u);
      const uint32_t keep = (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
      v[i] = (v[i] & keep) | (0xFF80FF80u & ~keep);
    }
  }
  static STEP_DEV float get1(T b) { return __uint_as_float((uint32_t)b << 16); }
  static STEP_DEV T put1(float f) { return (T)bits(f); }
};

template <> struct Row<ASYMSPEC_FP32> {
  static constexpr int VE = 4;
  typedef uint32_t T;
  typedef uint32_t U __attribute__((ext_vector_type(4), aligned(4)));
  static STEP_DEV float get(const u4& v, int e) { return __uint_as_float(v[e]); }
  static STEP_DEV void put_bits(u4& v, int e, uint32_t b) { v[e] = b; }
  static STEP_DEV void put(u4& v, int e, float f) { v[e] = __float_as_uint(f); }
  static STEP_DEV u4 neg_inf() { return u4{kNegInfBits, kNegInfBits, kNegInfBits, kNegInfBits}; }
  static STEP_DEV void mask(u4& v, uint32_t allowed) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = ((allowed >> i) & 1u) ? v[i] : kNegInfBits;
  }
  static STEP_DEV float get1(T b) { return __uint_as_float(b); }
  static STEP_DEV T put1(float f) { return __float_as_uint(f); }
};

template <int DT>
STEP_DEV u4 load_vec(const typename Row<DT>::T* p) {
  return *reinterpret_cast<const typename Row<DT>::U*>(p);
}
template <int DT>
STEP_DEV void store_vec(typename Row<DT>::T* p, const u4& v) {
  *reinterpret_cast<typename Row<DT>::U*>(p) = v;
}

}  // namespace asym_step

#endif  // ASYMSPEC_STEP_ROW_H_
