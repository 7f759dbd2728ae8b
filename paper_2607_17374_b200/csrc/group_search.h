// The group of a row by the groups' offsets.  Plain C++, so that it can be run on the host over as many groups as a call may have.
#pragma once

#ifndef TAURUS_HD
#ifdef __CUDACC__
#define TAURUS_HD __host__ __device__ __forceinline__
#else
#define TAURUS_HD inline
#endif
#endif

// The last of the offsets [0, groups] that is not above r; 0 where all are.  (lo + hi would pass 31 bits: there may be 2^30 groups.)
template <class Offsets>
TAURUS_HD int last_offset_not_above(const Offsets& offsets, int groups, long long r) {
  int lo = 0, hi = groups;                       // offsets[lo - 1] <= r < offsets[hi + 1], so to say
  while (lo < hi) {
    const int mid = hi - ((hi - lo) >> 1);
    if (offsets[mid] <= r) lo = mid; else hi = mid - 1;
  }
  return lo;
}
