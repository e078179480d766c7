// rotate_heads: a workgroup takes a few tokens, computes each angle's sine and cosine
// once into LDS, and turns the channels of all their heads with them, 16 bytes of each
// side of its pairs at a time.
//
// Bound by memory: 16384 tokens of 40 heads of 128 channels in bf16, 335 MB, take 55 us on
// the card (6.1 TB/s; a copy of more than the caches hold reaches 5.1), 57 a call.  An
// angle is some 60 operations of 64 and 32 bits, but one serves 40 heads here; 147456
// tokens of 2 heads of 256 channels, all turned, take 143 us for 302 MB by their angles
// (with sines in 64 bits throughout 154).  One step's rows (8 requests) take 4.4 us: a
// launch, and a chain of the position, its angle, LDS and the channels.  Loading the
// channels ahead of the angles made the large case slower.

#ifndef ASYMSPEC_CACHE_ROTATE_H_
#define ASYMSPEC_CACHE_ROTATE_H_

#include "format.h"

namespace asym_cache {

constexpr int kRotateThreads = 256;
constexpr int kRotateMostTokens = 8;

struct RotateArgs {
  asymspec_rotate r;
  uint32_t tokens;          // B * R
  int T;                    // tokens of a workgroup
  uint32_t pieces, tail;    // of a head: all, and those that are only copied
  Div by_n, by_R, by_pieces, by_heads;
};

// VEC: pieces of 16 bytes of each of the pair's sides (or of both, interleaved);
// else of one pair.  ONCE: more than the caches hold, which keep no line of what is read.
template <int DT, bool INTER, bool VEC, bool ONCE>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs A) {
  typedef typename Row<DT>::T T;
  constexpr int VE = VEC ? Row<DT>::VE : 1;
  extern __shared__ float2 turn[];                       // [T][n]
  const asymspec_rotate& r = A.r;
  const uint32_t first = blockIdx.x * (uint32_t)A.T;
  const uint32_t here = min((uint32_t)A.T, A.tokens - first);
  for (uint32_t i = threadIdx.x; i < here * (uint32_t)r.n; i += kRotateThreads) {
    uint32_t f = i;
    const uint32_t token = first + A.by_n.split(f);
    uint32_t row = token;
    const uint32_t b = A.by_R.split(row);
    const long long p = r.every_row ? (long long)r.positions[token] : (long long)r.positions[b] + row;
    // in turns, of which the whole ones leave in 64 bits; of what stays the 24 bits that
    // fp32 holds, and then the rest, below 2^-23 of a radian, to first order
    double t = (double)p * (r.frequencies[f] * 0.15915494309189533577);
    t -= rint(t);
    const float near = (float)t, rest = (float)((t - (double)near) * 6.28318530717958647693);
    float s, c;
    sincospif(2.0f * near, &s, &c);
    turn[i] = make_float2(fmaf(-s, rest, c) * r.magnitude, fmaf(c, rest, s) * r.magnitude);
  }
  __syncthreads();
  const uint32_t heads = (uint32_t)(r.q_heads + r.k_heads);
  const uint32_t all = here * heads * A.pieces;
  const uint32_t turned = A.pieces - A.tail;
  for (uint32_t i = threadIdx.x; i < all; i += kRotateThreads) {
    uint32_t piece = i;
    uint32_t head = A.by_pieces.split(piece);
    const uint32_t t = A.by_heads.split(head);
    uint32_t row = first + t;
    const uint32_t b = A.by_R.split(row);
    const bool is_q = head < (uint32_t)r.q_heads;
    if (!is_q) head -= (uint32_t)r.q_heads;
    const asymspec_heads& x = is_q ? r.q : r.k;
    const asymspec_heads& y = is_q ? r.q_out : r.k_out;
    const T* in = (const T*)x.at + (b * x.request + row * x.row + head * x.head);
    T* out = (T*)y.at + (b * y.request + row * y.row + head * y.head);
    const float2* w = turn + t * (uint32_t)r.n;
    if (piece >= turned) {
      const uint32_t c = 2u * (uint32_t)r.n + (piece - turned) * VE;
      if constexpr (VEC) asym_step::store_vec<DT>(out + c, load_row<DT, ONCE>(in + c));
      else out[c] = in[c];
    } else if constexpr (INTER) {
      if constexpr (VEC) {
        u4 v = load_row<DT, ONCE>(in + piece * VE);
#pragma unroll
        for (int e = 0; e < VE; e += 2) {
          const float2 cs = w[(piece * VE + e) / 2];
          const float p = Row<DT>::get(v, e), q = Row<DT>::get(v, e + 1);
          Row<DT>::put(v, e, p * cs.x - q * cs.y);
          Row<DT>::put(v, e + 1, p * cs.y + q * cs.x);
        }
        asym_step::store_vec<DT>(out + piece * VE, v);
      } else {
        const float2 cs = w[piece];
        const float p = Row<DT>::get1(in[2 * piece]), q = Row<DT>::get1(in[2 * piece + 1]);
        out[2 * piece] = Row<DT>::put1(p * cs.x - q * cs.y);
        out[2 * piece + 1] = Row<DT>::put1(p * cs.y + q * cs.x);
      }
    } else {
      const uint32_t c = piece * VE;
      if constexpr (VEC) {
        u4 v = load_row<DT, ONCE>(in + c), z = load_row<DT, ONCE>(in + c + r.n);
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          const float2 cs = w[c + e];
          const float p = Row<DT>::get(v, e), q = Row<DT>::get(z, e);
          Row<DT>::put(v, e, p * cs.x - q * cs.y);
          Row<DT>::put(z, e, p * cs.y + q * cs.x);
        }
        asym_step::store_vec<DT>(out + c, v);
        asym_step::store_vec<DT>(out + c + r.n, z);
      } else {
        const float2 cs = w[c];
        const float p = Row<DT>::get1(in[c]), q = Row<DT>::get1(in[c + r.n]);
        out[c] = Row<DT>::put1(p * cs.x - q * cs.y);
        out[c + r.n] = Row<DT>::put1(p * cs.y + q * cs.x);
      }
    }
  }
}

}  // namespace asym_cache

#endif  // ASYMSPEC_CACHE_ROTATE_H_
