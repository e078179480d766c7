// The kernels of attend_cache for one width of codes and type of queries.

#include <hip/hip_runtime.h>

#include "../step/launch.h"
#include "attend.h"
#include "attend_host.h"

namespace asym_cache {

constexpr int kBits = ASYMSPEC_PART_BITS, kType = ASYMSPEC_PART_DT;

template <int D, int MT>
static int attend_launch(AttendArgs& A, void* stream) {
  return asym_step::launch(attend_kernel<kBits, kType, D, MT>, (unsigned)A.workgroups, kAttendThreads, 0, stream, A);
}

template <int D>
static int attend_tiles(AttendArgs& A, int tiles, void* stream) {
  if constexpr (attend_most_tiles(kBits, kType == ASYMSPEC_BF16, D) > 1)
    if (tiles > 1) return attend_launch<D, 2>(A, stream);
  return attend_launch<D, 1>(A, stream);
}

template <>
int attend_part<kBits, kType>(AttendArgs& A, int tiles, void* stream) {
  switch (A.a.cache.dim) {
    case 64: return attend_tiles<64>(A, tiles, stream);
    case 96: return attend_tiles<96>(A, tiles, stream);
    case 128: return attend_tiles<128>(A, tiles, stream);
    case 192: return attend_tiles<192>(A, tiles, stream);
    default: return attend_tiles<256>(A, tiles, stream);
  }
}

}  // namespace asym_cache
