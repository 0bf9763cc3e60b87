// Rules of the paged cache's kernels as functions of numbers alone, for the
// device and for the host: C++ without HIP, so that they can be checked on any
// machine.
#pragma once

#include <stdint.h>

namespace rwttt {

// ---------------------------------------------------------------------------
// select: which scores are kept
// ---------------------------------------------------------------------------

constexpr int kSelBits = 12, kSelBins = 1 << kSelBits;

// The state of a ranking of v = score - least, narrowed by the bin that the last
// kept one lies in.  Kept are all v > v0, and of those equal to v0 the first `want`.
// While bits below `top` are open, v0's are zero and `want` counts the bin's.
struct Rank {
  uint32_t v0;
  int want, top;
};

// want >= 1 of the values in [0, range].
constexpr Rank rank_begin(uint32_t range, int want) { return {0, want, range ? 32 - __builtin_clz(range) : 0}; }

constexpr int rank_bit(const Rank& r) { return r.top > kSelBits ? r.top - kSelBits : 0; }

// Whether v lies in the bin that is looked at, and its bin within.
constexpr bool rank_in(const Rank& r, uint32_t v) { return r.top == 32 || v >> r.top == r.v0 >> r.top; }
constexpr uint32_t rank_bin(const Rank& r, uint32_t v) { return (v >> rank_bit(r)) & (kSelBins - 1); }

// The last kept one lies in `bin`, which holds `count` values, with `above` in the
// bins over it.  A bin that is kept whole ends the ranking.
constexpr Rank rank_narrow(Rank r, uint32_t bin, int above, int count) {
  const int bit = rank_bit(r);
  r.v0 |= bin << bit;
  r.want -= above;
  r.top = bit;
  if (count == r.want) {
    r.top = 0;
    if (r.v0) {
      r.v0 -= 1;
      r.want = 0;
    }
  }
  return r;
}

}  // namespace rwttt
