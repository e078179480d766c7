// The launches of attend_cache, an object for each part of the instances.

#ifndef ASYMSPEC_CACHE_ATTEND_HOST_H_
#define ASYMSPEC_CACHE_ATTEND_HOST_H_

namespace asym_cache {

struct AttendArgs;

// Row tiles of an instance: as many as a call's rows need, as long as a wave's sums,
// queries and two sets of codes stay in its registers.
constexpr int attend_most_tiles(bool bf16, int dim) { return bf16 ? (dim <= 64 ? 4 : dim <= 128 ? 2 : 1) : dim <= 64 ? 2 : 1; }

// Waves of an instance on a SIMD, whose registers they share (168 each, or 256), and so
// workgroups on a compute unit.
constexpr int attend_waves(bool bf16, int dim, int tiles) { return bf16 && dim * tiles <= 128 ? 3 : 2; }

template <int BITS, int DT>
int attend_part(AttendArgs& A, int tiles, void* stream);

}  // namespace asym_cache

#endif  // ASYMSPEC_CACHE_ATTEND_HOST_H_
