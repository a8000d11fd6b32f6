// How keys are shared out over the splits of a sequence.  No CUDA in here, so that the
// arithmetic can be checked on the host.
#ifndef SBD_KEY_RANGES_H
#define SBD_KEY_RANGES_H

#include <stdint.h>

#ifdef __CUDACC__
#define SBD_HD __host__ __device__ __forceinline__
#else
#define SBD_HD inline
#endif

namespace sbd {

struct KeyRange {
  uint32_t begin, end;
};
// Range `split` of n < 2^31 keys in `splits` <= 16 ranges of whole granules (of 16 keys
// at most), the last ones shorter or empty.  In 32 unsigned bits: n plus a granule and
// twice the rounding of the ranges before stay below 2^32.
SBD_HD KeyRange key_range(uint32_t n, uint32_t splits, uint32_t split, uint32_t granule) {
  const uint32_t range = ((n + splits - 1) / splits + granule - 1) / granule * granule;
  const uint32_t begin = split * range < n ? split * range : n;
  return {begin, n - begin < range ? n : begin + range};
}

}  // namespace sbd

#endif  // SBD_KEY_RANGES_H
