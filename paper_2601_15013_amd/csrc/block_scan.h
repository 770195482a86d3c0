// Sums over a wavefront and over a workgroup of 1024 threads, for the kernels that plan a call's work in one workgroup.
#pragma once
#include "common.h"

namespace {

constexpr int PT = 1024;                // threads of such a workgroup

// x of the lane `ctrl` says (a DPP pattern), 0 where there is none.
template <int CTRL, int ROWS> __device__ __forceinline__ int from_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS> __device__ __forceinline__ float from_lane(float x) {
    return __uint_as_float((uint32_t)from_lane<CTRL, ROWS>((int)__float_as_uint(x)));
}
// Inclusive sums over the wavefront, in registers: shifts by 1, 2, 4, 8 within rows of 16 lanes, then the last lane of a row to the next
// one, then of the lower half to the upper.  (Six shuffles through LDS take some ten times as long.)
template <typename T> __device__ __forceinline__ T wave_inclusive(T v) {
    v += from_lane<0x111, 0xf>(v);
    v += from_lane<0x112, 0xf>(v);
    v += from_lane<0x114, 0xf>(v);
    v += from_lane<0x118, 0xf>(v);
    v += from_lane<0x142, 0xa>(v);
    v += from_lane<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_inclusive(v), 63); }
__device__ __forceinline__ float wave_total(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(wave_inclusive(v)), 63));
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
