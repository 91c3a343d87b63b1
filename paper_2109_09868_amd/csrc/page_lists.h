// One workgroup's view of a cache's pages: sums over its threads, and the free pages in ascending order.
#pragma once

#include "sequences.h"

namespace approxifer {

constexpr int kThreads = 1024;                                // of the kernels that give out pages: one workgroup
constexpr int kList = 8192;                                   // free pages found at a time, in LDS

// Exclusive prefix sum over the workgroup, and the total; `sums` holds 16 of LDS.
template <class T>
__device__ __forceinline__ T block_scan(T v, T *sums, T *total) {
    const int lane = lane_id(), wave = wave_id(), waves = blockDim.x / kWave;
    T up = v;
    for (int o = 1; o < kWave; o <<= 1) {
        const T x = __shfl_up(up, o);
        if (lane >= o) up += x;
    }
    __syncthreads();                                          // the sums of the call before have been read
    if (lane == kWave - 1) sums[wave] = up;
    __syncthreads();
    if (wave == 0) {
        T x = lane < waves ? sums[lane] : 0;
        for (int o = 1; o < 16; o <<= 1) {
            const T y = __shfl_up(x, o);
            if (lane >= o) x += y;
        }
        if (lane < waves) sums[lane] = x;
    }
    __syncthreads();
    *total = sums[waves - 1];
    return up - v + (wave > 0 ? sums[wave - 1] : 0);
}

// The first `most` (at most kList) free pages from *cursor on, ascending, into list; how many there are.  Afterwards *cursor is
// where to go on once those have been taken.  By the whole workgroup of kThreads.  `ahead` holds the stretch's refs: those of the
// cursor on entry.
struct Stretch {
    int32_t refs[4];
    __device__ __forceinline__ void load(const int32_t *from, int at, int P) {
        const int p = at + 4 * static_cast<int>(threadIdx.x);
#pragma unroll
        for (int k = 0; k < 4; ++k) refs[k] = p + k < P ? from[p + k] : 1;
    }
};
__device__ __forceinline__ int find_free(const int32_t *refs, int P, int most, int *list, int *sums, int *cursor, Stretch ahead) {
    int found = 0, at = *cursor;
    while (found < most && at < P) {
        const int p0 = at + 4 * static_cast<int>(threadIdx.x);
        bool is_free[4];
        int count = 0;
        for (int k = 0; k < 4; ++k) {
            is_free[k] = ahead.refs[k] == 0;
            count += is_free[k];
        }
        ahead.load(refs, at + 4 * kThreads, P);
        int total;
        int rank = found + block_scan(count, sums, &total);
        for (int k = 0; k < 4; ++k)
            if (is_free[k]) {
                if (rank < most) list[rank] = p0 + k;
                ++rank;
            }
        found += total;
        if (found <= most) at += 4 * kThreads;                // else the rest of this stretch is for the next time
    }
    *cursor = at;
    __syncthreads();
    return min(found, most);
}

}  // namespace approxifer
