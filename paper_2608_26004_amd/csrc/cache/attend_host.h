// The launches of attend_cache, an object for each part of the instances.

#ifndef ASYMSPEC_CACHE_ATTEND_HOST_H_
#define ASYMSPEC_CACHE_ATTEND_HOST_H_

namespace asym_cache {

struct AttendArgs;

// Row tiles of an instance: two where a wave's sums, queries and codes stay in its
// registers.  (16 requests of 16384 positions, 4 heads: 28 rows of dim 192 in 8 bits with
// two tiles 91 us, with one 120; but fp32 dim 128 in 4 bits 69 and 63, and where registers
// spill, as with dim 256 in 8 bits, 289 and 153.  64 rows of dim 64: four tiles 54 to 58,
// two 52 to 57.)
constexpr int attend_most_tiles(int bits, bool bf16, int dim) { return (bf16 ? dim * bits < 2048 : dim <= 64) ? 2 : 1; }

// Waves of an instance on a SIMD, whose 512 registers they share, and so workgroups on a
// compute unit: as many as need no register spilled.  (With spills dim 256 in 8 bits, 12
// rows, takes 70 us instead of 42, and in fp32 118 instead of 46.)
constexpr int attend_waves(int bits, bool bf16, int dim, int tiles) {
  return bf16 ? (tiles == 1 && dim * bits <= 512 ? 3 : dim * bits >= 2048 || dim * tiles >= 384 ? 1 : 2) : dim >= 192 ? 1 : 2;
}

template <int BITS, int DT>
int attend_part(AttendArgs& A, int tiles, void* stream);

}  // namespace asym_cache

#endif  // ASYMSPEC_CACHE_ATTEND_HOST_H_
