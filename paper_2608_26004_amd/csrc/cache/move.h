// write_cache and read_cache: 8 channels a lane.  A tile is 16 tokens, whose rows of a
// head lie one behind the other in a block; lanes run along a head's channels and then
// along the tile's tokens, so that both sides move whole lines.

#ifndef ASYMSPEC_CACHE_MOVE_H_
#define ASYMSPEC_CACHE_MOVE_H_

#include "format.h"

namespace asym_cache {

constexpr int kMoveThreads = 256;
constexpr int kMoveTile = 16;

struct MoveArgs {
  asymspec_cache c;
  asymspec_heads k, v;             // what is written, or (contiguous) read
  const int64_t* slots;            // write: [tokens]
  const int32_t *table, *lengths, *first;   // read
  uint32_t tokens;                 // write: B * R; read: width
  uint32_t tiles;                  // write: of all tokens; read: of a request's
  uint32_t items, groups;          // of a tile: lanes' parts, and workgroups that share them
  int max_blocks;
  Div by_lanes, by_heads, by_size, by_R, by_groups, by_tiles;
};

// Which part of a tile an index says: channels c8 * 8 on of token t of a head of the
// keys (0) or values.
struct Part {
  uint32_t c8, t, head, which;
  STEP_DEV Part(const MoveArgs& A, uint32_t i) {
    c8 = i;
    t = A.by_lanes.split(c8);
    head = t / kMoveTile;
    t %= kMoveTile;
    which = A.by_heads.split(head);
  }
};

// A token's row of a head, from its slot.
STEP_DEV uint64_t row_of(const MoveArgs& A, uint32_t block, uint32_t offset, uint32_t head) {
  return ((uint64_t)block * (uint32_t)A.c.heads + head) * (uint32_t)A.c.block_size + offset;
}

// The largest of the four lanes that share a scale.
STEP_DEV uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));
}

template <int DT, int BITS>
__global__ __launch_bounds__(kMoveThreads) void write_kernel(MoveArgs A) {
  typedef typename Row<DT>::T T;
  uint32_t group = blockIdx.x;
  const uint32_t tile = A.by_groups.split(group);
  for (uint32_t i = group * kMoveThreads + threadIdx.x; i < A.items; i += A.groups * kMoveThreads) {
    const Part p(A, i);
    const uint32_t token = tile * kMoveTile + p.t;
    const int64_t slot = token < A.tokens ? A.slots[token] : -1;
    // (lanes that share a scale share a token)
    if (slot < 0 || slot >= (int64_t)A.c.blocks * A.c.block_size) continue;
    uint32_t row = token;
    const uint32_t b = A.by_R.split(row);
    const asymspec_heads& x = p.which ? A.v : A.k;
    float f[8];
    load8<DT>((const T*)x.at + (b * x.request + row * x.row + p.head * x.head) + p.c8 * 8, f);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(f[e]) & 0x7FFFFFFFu);
    const uint32_t byte = scale_byte<BITS>(quad_max(most));
    const bool finite = byte != kNotFinite;
    u2 codes = encode8<BITS>(f, scale_of(finite ? byte : 127));
    if (!finite) codes = u2{0, 0};
    uint32_t offset = (uint32_t)slot;
    const uint32_t block = A.by_size.split(offset);
    const uint64_t at = row_of(A, block, offset, p.head);
    uint8_t* data = (uint8_t*)(p.which ? A.c.values : A.c.keys) + at * (uint32_t)(A.c.dim * BITS / 8) + p.c8 * BITS;
    if (BITS == 4) *(uint32_t*)data = codes[0];
    else *(u2*)data = codes;
    if (p.c8 % 4 == 0)
      ((uint8_t*)(p.which ? A.c.value_scales : A.c.key_scales))[at * (uint32_t)(A.c.dim / kBlock) + p.c8 / 4] = (uint8_t)byte;
  }
}

template <int DT, int BITS>
__global__ __launch_bounds__(kMoveThreads) void read_kernel(MoveArgs A) {
  typedef typename Row<DT>::T T;
  uint32_t group = blockIdx.x;
  uint32_t tile = A.by_groups.split(group);
  const uint32_t b = A.by_tiles.split(tile);
  const int64_t from = A.first != nullptr ? A.first[b] : 0, to = A.lengths[b];
  for (uint32_t i = group * kMoveThreads + threadIdx.x; i < A.items; i += A.groups * kMoveThreads) {
    const Part p(A, i);
    const uint32_t token = tile * kMoveTile + p.t;
    if (token >= A.tokens) continue;
    const int64_t position = from + token;
    u4 v{0, 0, 0, 0};
    if (position >= 0 && position < to) {
      uint32_t offset = (uint32_t)position;
      const uint32_t page = A.by_size.split(offset);
      const int block = page < (uint32_t)A.max_blocks ? A.table[(int64_t)b * A.max_blocks + page] : -1;
      if ((uint32_t)block < (uint32_t)A.c.blocks) {
        const uint64_t at = row_of(A, (uint32_t)block, offset, p.head);
        const uint8_t* data = (const uint8_t*)(p.which ? A.c.values : A.c.keys) +
                              at * (uint32_t)(A.c.dim * BITS / 8) + p.c8 * BITS;
        const uint32_t byte =
            ((const uint8_t*)(p.which ? A.c.value_scales : A.c.key_scales))[at * (uint32_t)(A.c.dim / kBlock) + p.c8 / 4];
        uint32_t codes[2];
        codes[0] = *(const uint32_t*)data;
        if (BITS == 8) codes[1] = *(const uint32_t*)(data + 4);
        v = decode8<BITS>(codes, scale_of(byte));
        if (byte > most_scale<BITS>()) v = u4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
      }
    }
    T* out = (T*)(p.which ? A.v.at : A.k.at);
    if (out == nullptr) continue;
    out += (((int64_t)b * A.tokens + token) * (uint32_t)A.c.heads + p.head) * A.c.dim + p.c8 * 8;
    if constexpr (DT == ASYMSPEC_BF16) {
      *(u4*)out = v;
    } else {
      u4 lo, hi;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo[e] = __float_as_uint(Row<ASYMSPEC_BF16>::get(v, e));
        hi[e] = __float_as_uint(Row<ASYMSPEC_BF16>::get(v, 4 + e));
      }
      *(u4*)out = lo;
      *(u4*)(out + 4) = hi;
    }
  }
}

}  // namespace asym_cache

#endif  // ASYMSPEC_CACHE_MOVE_H_
