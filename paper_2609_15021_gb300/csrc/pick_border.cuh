// pick_border.cuh -- the search for the smallest picked rank, in plain arithmetic that the host compiles too.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define KVX_BOTH __host__ __device__ __forceinline__
#else
#define KVX_BOTH inline
#endif

namespace kvx {

constexpr int kPickBits = 11, kPickBins = 1 << kPickBits, kPickPasses = 3;

// Where the want'th largest of the ranks in [low, high] lies.  A pass counts them in up to 2^11 equal ranges of 2^shift and goes on with
// the one that it falls in, which takes 11 bits off their span: three passes leave one rank whatever the ranks are, and whether or not
// they are the same in every pass (a workspace that another call writes to).
struct Border {
  uint32_t low, high;
  int32_t want;
  uint32_t rank = UINT32_MAX;  // ranks above it are picked,
  int32_t equal = 0;           // and the first `equal` of those that have it

  KVX_BOTH int shift() const {
    const uint32_t span = high - low;
#ifdef __CUDA_ARCH__
    const int bits = 32 - __clz(span);
#else
    int bits = 0;
    while (bits < 32 && span >> bits) ++bits;
#endif
    return bits > kPickBits ? bits - kPickBits : 0;
  }
  // After a pass with ranges of 2^shift: the range it falls in, how many of that are wanted (0: none falls there, as the ranks have
  // changed since they were counted) and how many there are.  False when the search has ended.
  KVX_BOTH bool narrow(int shift, uint32_t range, int32_t wanted, int32_t count) {
    if (wanted <= 0) return false;
    low += range << shift;
    want = wanted;
    if (shift == 0 || count == wanted) {
      rank = shift == 0 ? low : low - 1;  // low is above 0, which is no score's
      equal = shift == 0 ? want : 0;
      return false;
    }
    const uint32_t last = low + ((1u << shift) - 1);
    high = last < high ? last : high;
    return true;
  }
};

}  // namespace kvx
