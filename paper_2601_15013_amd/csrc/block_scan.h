// Sums over a wavefront and over a workgroup of 1024 threads, for the kernels that plan a call's work in one workgroup.
#pragma once
#include "common.h"

namespace {

constexpr int PT = 1024;                // threads of such a workgroup

__device__ __forceinline__ int wave_inclusive(int v, int lane) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(v, o, 64);
        if (lane >= o) v += u;
    }
    return v;
}

// Exclusive sum of v over the workgroup (all threads call); *total is the sum over all threads.
__device__ __forceinline__ long long block_exclusive(long long v, long long* total, long long* part /* [PT / 64] in LDS */) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long u = __shfl_up(x, o, 64);
        if (lane >= o) x += u;
    }
    __syncthreads();                    // part may still be read from the call before
    if (lane == 63) part[wave] = x;
    __syncthreads();
    long long p = part[lane & 15];      // every wavefront sums the sixteen by itself
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
        const long long u = __shfl_up(p, o, 16);
        if ((lane & 15) >= o) p += u;
    }
    *total = __shfl(p, 15, 64);
    return __shfl(p, wave, 64) - __shfl(x, 63, 64) + x - v;
}

}  // namespace
