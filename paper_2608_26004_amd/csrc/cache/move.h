// write_cache and read_cache: a lane has 8 channels of a token, keys and values of two
// heads, whose loads are under way together.  A token's place is looked up once; what a
// head adds is a constant.  Lanes run along a head's channels and then along tokens that
// are neighbours, in a block of the cache too, so that both sides move whole lines.
//
// Bound by memory: 65536 tokens of 8 heads of 128 channels from bf16 to 4 bits and back
// take 119 us for 679 MB, 16 x 8192 positions back 124 for 644 MB (5.2 TB/s and more; a
// copy reaches 5.1).  With one head's key or value a lane the index arithmetic took
// longer than that (176, 181 us); with one head a lane they take 139 and 133, with all
// eight 132 and 134; with loads that leave lines in the caches 138 and 125.

#ifndef ASYMSPEC_CACHE_MOVE_H_
#define ASYMSPEC_CACHE_MOVE_H_

#include "format.h"

namespace asym_cache {

constexpr int kMoveThreads = 256;
constexpr int kMoveHeads = 2;         // of a lane

struct MoveArgs {
  asymspec_cache c;
  asymspec_heads k, v;             // what is written, or (contiguous) read
  const int64_t* slots;            // write: [tokens]
  const int32_t *table, *lengths, *first;   // read
  uint32_t tokens;                 // write: B * R; read: width
  uint32_t tile;                   // tokens of a workgroup
  uint32_t heads;                  // of a workgroup: at most kMoveHeads
  int max_blocks;
  Div by_lanes, by_size, by_R, by_groups, by_tiles;
};

// The largest of the four lanes that share a scale.
STEP_DEV uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));
}

// Calls load(i, which, head) for the keys (which = 0) and values of each of the heads,
// and then use of the same.
template <class Load, class Use>
STEP_DEV void each_head(uint32_t from, uint32_t to, Load&& load, Use&& use) {
  static_assert(kMoveHeads == 2);
  const bool two = from + 1 < to;
  load(0, 0, from), load(1, 1, from);
  if (two) load(2, 0, from + 1), load(3, 1, from + 1);
  use(0, 0, from), use(1, 1, from);
  if (two) use(2, 0, from + 1), use(3, 1, from + 1);
}

template <int DT, int BITS, bool ONCE>
__global__ __launch_bounds__(kMoveThreads) void write_kernel(MoveArgs A) {
  typedef typename Row<DT>::T T;
  uint32_t group = blockIdx.x;
  const uint32_t tile = A.by_groups.split(group);
  uint32_t c8 = threadIdx.x;
  const uint32_t t = A.by_lanes.split(c8), token = tile * A.tile + t;
  const int64_t slot = t < A.tile && token < A.tokens ? A.slots[token] : -1;
  // (lanes that share a scale share a token)
  if (slot < 0 || slot >= (int64_t)A.c.blocks * A.c.block_size) return;
  uint32_t row = token, offset = (uint32_t)slot;
  const uint32_t b = A.by_R.split(row), block = A.by_size.split(offset);
  const T* const k = (const T*)A.k.at + (b * A.k.request + row * A.k.row) + c8 * 8;
  const T* const v = (const T*)A.v.at + (b * A.v.request + row * A.v.row) + c8 * 8;
  const uint32_t size = (uint32_t)A.c.block_size, bytes = (uint32_t)(A.c.dim * BITS / 8), scales = (uint32_t)(A.c.dim / kBlock);
  const uint64_t first = (uint64_t)block * (uint32_t)A.c.heads * size + offset;
  float f[2 * kMoveHeads][8];
  each_head(
      group * A.heads, min((group + 1) * A.heads, (uint32_t)A.c.heads),
      [&](int i, int which, uint32_t head) { load8<DT, ONCE>(which ? v + head * A.v.head : k + head * A.k.head, f[i]); },
      [&](int i, int which, uint32_t head) {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(f[i][e]) & 0x7FFFFFFFu);
        const uint32_t byte = scale_byte<BITS>(quad_max(most));
        const bool finite = byte != kNotFinite;
        u2 codes = encode8<BITS>(f[i], scale_of(finite ? byte : 127));
        if (!finite) codes = u2{0, 0};
        const uint64_t at = first + (uint64_t)head * size;
        uint8_t* data = (uint8_t*)(which ? A.c.values : A.c.keys) + at * bytes + c8 * BITS;
        if (BITS == 4) *(uint32_t*)data = codes[0];
        else *(u2*)data = codes;
        if (c8 % 4 == 0)
          ((uint8_t*)(which ? A.c.value_scales : A.c.key_scales))[at * scales + c8 / 4] = (uint8_t)byte;
      });
}

template <int DT, int BITS>
__global__ __launch_bounds__(kMoveThreads) void read_kernel(MoveArgs A) {
  typedef typename Row<DT>::T T;
  uint32_t group = blockIdx.x;
  uint32_t tile = A.by_groups.split(group);
  const uint32_t b = A.by_tiles.split(tile);
  uint32_t c8 = threadIdx.x;
  const uint32_t t = A.by_lanes.split(c8), token = tile * A.tile + t;
  if (t >= A.tile || token >= A.tokens) return;
  const int64_t position = (A.first != nullptr ? (int64_t)A.first[b] : 0) + token;
  const uint32_t size = (uint32_t)A.c.block_size, bytes = (uint32_t)(A.c.dim * BITS / 8), scales = (uint32_t)(A.c.dim / kBlock);
  int block = -1;
  uint32_t offset = (uint32_t)position;
  if (position >= 0 && position < A.lengths[b]) {
    const uint32_t page = A.by_size.split(offset);
    if (page < (uint32_t)A.max_blocks) block = A.table[(int64_t)b * A.max_blocks + page];
  }
  const bool there = (uint32_t)block < (uint32_t)A.c.blocks;
  const uint64_t first = there ? (uint64_t)block * (uint32_t)A.c.heads * size + offset : 0;
  const int64_t to = ((int64_t)b * A.tokens + token) * (uint32_t)A.c.heads * A.c.dim + c8 * 8;
  uint32_t codes[2 * kMoveHeads][2], byte[2 * kMoveHeads];
  each_head(
      group * A.heads, min((group + 1) * A.heads, (uint32_t)A.c.heads),
      [&](int i, int which, uint32_t head) {
        if (!there) return;
        const uint64_t at = first + (uint64_t)head * size;
        const uint8_t* data = (const uint8_t*)(which ? A.c.values : A.c.keys) + at * bytes + c8 * BITS;
        if (BITS == 4) {
          codes[i][0] = __builtin_nontemporal_load((const uint32_t*)data);
        } else {
          const u2 x = __builtin_nontemporal_load((const u2*)data);
          codes[i][0] = x[0], codes[i][1] = x[1];
        }
        byte[i] = ((const uint8_t*)(which ? A.c.value_scales : A.c.key_scales))[at * scales + c8 / 4];
      },
      [&](int i, int which, uint32_t head) {
        T* out = (T*)(which ? A.v.at : A.k.at);
        if (out == nullptr) return;
        u4 x{0, 0, 0, 0};
        if (there) {
          x = decode8<BITS>(codes[i], scale_of(byte[i]));
          if (byte[i] > most_scale<BITS>()) x = u4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        }
        out += to + (int64_t)head * A.c.dim;
        if constexpr (DT == ASYMSPEC_BF16) {
          *(u4*)out = x;
        } else {
          u4 lo, hi;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            lo[e] = __float_as_uint(Row<ASYMSPEC_BF16>::get(x, e));
            hi[e] = __float_as_uint(Row<ASYMSPEC_BF16>::get(x, 4 + e));
          }
          *(u4*)out = lo;
          *(u4*)(out + 4) = hi;
        }
      });
}

}  // namespace asym_cache

#endif  // ASYMSPEC_CACHE_MOVE_H_
