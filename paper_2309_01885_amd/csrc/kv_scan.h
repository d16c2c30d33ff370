// Sums over a workgroup of 1024 threads, for the kernels that lay out a call's work on the device.
#pragma once

#include "kv.h"

namespace qe {

constexpr int kScanThreads = 1024;

// The inclusive sum over the workgroup's threads; all: the sum of all.  part: 16 numbers of LDS, of this call alone
// until the next barrier.
__device__ inline int64_t scan_add(int64_t x, int64_t* part, int64_t& all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int64_t y = __shfl_up(x, m);
        x += lane >= m ? y : 0;
    }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int64_t before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kScanThreads / 64; ++w) {
        before += w < wave ? part[w] : 0;
        all += part[w];
    }
    return x + before;
}

// The last of n ascending numbers that is at most x (the first is).
template <class I> __device__ inline int64_t last_at_most(const I* at, int64_t n, int64_t x)
{
    int64_t lo = 0, hi = n;                              // at[lo] <= x < at[hi]
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (at[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace qe
