// Bins of a row's logits by sixteenths of the temperature (sample.hip): plain arithmetic, for the
// kernels and for host code.
#pragma once

#include <math.h>
#include <stdint.h>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define AQLM_BINS_FN __host__ __device__ __forceinline__
#else
#define AQLM_BINS_FN inline
#endif

namespace aqlm {

constexpr int kSampleBins = 512;

// The least fp32 number that is not below n, |n| up to 2^30.  (From 2^24 on n itself need not be one, and
// the nearest one may lie below it.)
AQLM_BINS_FN float least_not_below(int n) {
  const float f = (float)n;
  return (int32_t)f >= n ? f : __builtin_bit_cast(float, __builtin_bit_cast(int32_t, f) + (f < 0.f ? -1 : 1));
}

// The bins: in whole numbers of f = l c below the largest's, |f| up to 2^29, or (fine) the 512 parts of one of them.  A
// bin has the f with lower <= f < upper.  (Fine: |low| below 2^14, so that 512 low is a whole number of 32 bits, and
// 512 f is exact where f - low is not: just below 0 that is 1.)
struct Bins {
  int top;  // of the largest
  bool fine;
  float low;  // fine: the lower end
  AQLM_BINS_FN int at(float f) const {
    return fine ? kSampleBins - 1 - ((int)floorf(f * kSampleBins) - (int)(low * kSampleBins)) : top - (int)floorf(f);
  }
  AQLM_BINS_FN float lower(int bin) const {
    return fine ? low + (float)(kSampleBins - 1 - bin) / kSampleBins : least_not_below(top - bin);
  }
  AQLM_BINS_FN float upper(int bin) const {
    return fine ? lower(bin) + 1.f / kSampleBins : least_not_below(top - bin + 1);
  }
  AQLM_BINS_FN int last() const { return fine ? kSampleBins - 1 : kSampleBins - 2; }
};

}  // namespace aqlm
