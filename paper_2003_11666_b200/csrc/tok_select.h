// Selection of the k-th largest key by bisection; compiles for the device and for the host.
#pragma once

#ifdef __CUDACC__
#define PB_ANYWHERE __host__ __device__ __forceinline__
#else
#define PB_ANYWHERE inline
#endif

namespace pb {

// The largest t in [lo, hi] that at least k keys reach, where `reach(t)` is how many do and at least k reach `lo`;
// or any t that exactly k reach.  Halves the range in each step, so it takes 32 of them at most, and no sum here
// passes the largest unsigned number, whatever lo <= hi are (lo + hi would, and so would hi - lo + 1).
template <typename Reach>
PB_ANYWHERE unsigned highest_reached(unsigned lo, unsigned hi, int k, Reach reach) {
    while (lo < hi) {
        const unsigned mid = hi - (hi - lo) / 2;             // lo < mid <= hi
        const int c = reach(mid);
        if (c >= k) lo = mid; else hi = mid - 1;
        if (c == k) break;
    }
    return lo;
}

}  // namespace pb
