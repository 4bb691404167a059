// Where eviction cuts the keys of a pair with up to kSmallRows rows: the steps that evict_small_kernel takes, also run by the host
// mirror omni_debug_evict_stay.
#pragma once

#include <hip/hip_runtime.h>

namespace omni {

constexpr int kRanked = 128;                   // keys of a bin that are compared with one another instead of counted by digits

// The bin that holds the need-th largest key, how many of it are wanted, and how many it holds.
struct Found {
  int bin, left, count;
};

// The keys of [base, base + span], counted in bins of 2^low: at most 2^11 of them.
struct KeyRange {
  unsigned base, span;
  int low;
  __host__ __device__ __forceinline__ bool holds(unsigned key) const { return key - base <= span; }
  __host__ __device__ __forceinline__ int bin_of(unsigned key) const { return (int)((key - base) >> low); }
  // One of its bins.  The range need not end where a bin does (narrowed, it begins and ends with a key): what the last bin would hold
  // beyond the end are keys of a range above, which the counts know as rows that stay.
  __host__ __device__ __forceinline__ void enter(int bin) {
    const unsigned from = (unsigned)bin << low, width = (1u << low) - 1;
    base += from;
    span = span - from < width ? span - from : width;
  }
  // From its smallest to its largest key.
  __host__ __device__ __forceinline__ void narrow(unsigned smallest, unsigned largest) {
    base = smallest;
    span = largest - smallest;
    const int bits = span ? 32 - __builtin_clz(span) : 0;
    low = bits > 11 ? bits - 11 : 0;
  }
};

// Where the need-th largest key lies: in a range of `count` keys, of which `need` stay, as does every key above it.
struct KeyCut {
  KeyRange range;
  int need, count;
  bool equal;                                  // many equal keys, range.base; else count == need (all stay) or at most kRanked
};

// Level by level: the keys of a range by their bins; the bin with the cut is the next range, narrowed to what it holds, until all of it
// stays, few keys are left or all are equal.  Three levels at most: 11 bits, at most 10 of the 21 left, then whole keys.
//   bins(level, range, need) -> Found; ends(level, range, smallest, largest): of the range's keys
template <typename Bins, typename Ends>
__host__ __device__ __forceinline__ KeyCut find_cut(int need, Bins bins, Ends ends) {
  KeyCut c{KeyRange{0u, ~0u, 21}, need, 0, false};
  for (int level = 0;; ++level) {
    const Found f = bins(level, c.range, c.need);
    c.range.enter(f.bin);
    c.need = f.left;
    c.count = f.count;
    if (c.count == c.need || c.count <= kRanked) return c;
    c.equal = c.range.low == 0;
    if (c.equal) return c;
    unsigned smallest, largest;
    ends(level, c.range, smallest, largest);
    c.range.narrow(smallest, largest);
    c.equal = c.range.span == 0;
    if (c.equal) return c;
  }
}

}  // namespace omni
