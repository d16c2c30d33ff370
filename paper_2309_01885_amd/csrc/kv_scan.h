// Sums over a workgroup of up to 1024 threads, for the kernels that lay out a call's work on the device.
#pragma once

#include "kv.h"

namespace qe {

constexpr int kScanThreads = 1024;

// x of the lane that the vector units' permutation CTRL names, 0 where it names none or the lane's row is not in ROWS.
template <int CTRL, int ROWS> __device__ inline int64_t moved_or_0(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)x, CTRL, ROWS, 0xf, ROWS == 0xf);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(x >> 32), CTRL, ROWS, 0xf, ROWS == 0xf);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
// The inclusive sum over 16 lanes, and over a wave.
__device__ inline int64_t row_scan(int64_t x)
{
    x += moved_or_0<0x111, 0xf>(x);                      // from the lane before, from 2, 4 and 8 before
    x += moved_or_0<0x112, 0xf>(x);
    x += moved_or_0<0x114, 0xf>(x);
    return x + moved_or_0<0x118, 0xf>(x);
}
__device__ inline int64_t wave_scan(int64_t x)
{
    x = row_scan(x);
    x += moved_or_0<0x142, 0xa>(x);                      // the last lane of rows 0 and 2 to rows 1 and 3
    return x + moved_or_0<0x143, 0xc>(x);                // lane 31 to rows 2 and 3
}
__device__ inline int64_t lane_of(int64_t x, int lane)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}

// The inclusive sums of N numbers over the workgroup's threads; all: the sums of all.  lds: of this call alone until
// the next barrier.  (Every wave sums the waves' totals by itself, a lane a wave: as a loop over them in each thread a
// sum of two numbers took 2.2 us in 16 waves.)
template <int N> struct ScanLds { int64_t part[N][kScanThreads / 64]; };
template <int N> __device__ inline void scan_add(int64_t (&x)[N], ScanLds<N>& lds, int64_t (&all)[N])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = wave_scan(x[n]);
    if (waves > 1) {
        if (lane == 63) {
#pragma unroll
            for (int n = 0; n < N; ++n) lds.part[n][wave] = x[n];
        }
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (waves == 1) {
            all[n] = lane_of(x[n], 63);
            continue;
        }
        const int64_t y = row_scan((lane & 15) < waves ? lds.part[n][lane & 15] : 0);
        all[n] = lane_of(y, 15);
        if (wave > 0) x[n] += lane_of(y, wave - 1);
    }
}

// Threads of a workgroup that has n things to do, a thread or more each.
inline int scan_threads(int64_t n) { return (int)std::min<int64_t>(kScanThreads, std::max<int64_t>(64, cdiv(n, 64) * 64)); }

// The last of n ascending numbers that is at most x (the first is).
template <class I> __device__ inline int64_t last_at_most(const I* at, int64_t n, int64_t x)
{
    int lo = 0, hi = (int)n;                             // at[lo] <= x < at[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

}  // namespace qe
