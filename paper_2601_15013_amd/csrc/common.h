// Internal helpers shared by the HIP translation units of libradixmlp.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <stddef.h>
#include "radixmlp.h"

typedef __bf16 bf16_t;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef _Float16 f16_t;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

#define RADIX_WAVE 64

#define HIP_TRY(expr)                                   \
    do {                                                \
        hipError_t _e = (expr);                         \
        if (_e != hipSuccess) return RADIX_ERR_HIP;     \
    } while (0)

static inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
__host__ __device__ static inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<bf16_t>(bf16_t v) { return (float)v; }
template <> __device__ __forceinline__ float to_f32<f16_t>(f16_t v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ f16_t from_f32<f16_t>(float v) { return (f16_t)v; }
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return (bf16_t)v; }

// 16-bit MFMA operand types: v_mfma_f32_32x32x16_{bf16,f16}.  Lane (r = lane % 32, g = lane / 32)
// supplies 8 consecutive k of row r (k-group g) for both operands; accumulator register e of the
// 32x32 result is row 8 (e / 4) + 4 g + e % 4, column r.  v_mfma_f32_16x16x32_{bf16,f16} (mfma16): lane (r = lane % 16,
// g = lane / 16) supplies 8 consecutive k of row r (k-group g); register e of the 16x16 result is row 4 g + e, column r.
template <int DT> struct Op;
template <> struct Op<RADIX_BF16> {
    typedef bf16_t T;
    typedef bf16x8 V8;
    typedef bf16x4 V4;
    static __device__ __forceinline__ f32x16 mfma(V8 a, V8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(V8 a, V8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct Op<RADIX_F16> {
    typedef f16_t T;
    typedef f16x8 V8;
    typedef f16x4 V4;
    static __device__ __forceinline__ f32x16 mfma(V8 a, V8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 mfma16(V8 a, V8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

// Device status word: first error wins.
__device__ __forceinline__ void set_status(int32_t* status, int32_t code) {
    if (status) atomicCAS(status, 0, code);
}

// The sequence that token i lies in: the smallest s with cu[s + 1] > i, searched by the whole wavefront, 64 candidates
// a step (i is the same in all lanes).  Three dependent loads for 65 000 sequences where a search by halves takes 16.
__device__ __forceinline__ int sequence_of(const int32_t* __restrict__ cu, int B, int i, int lane) {
    int lo = 0, n = B;                                      // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 63) >> 6, first = lane * step;
        const int last = first + step < n ? first + step - 1 : n - 1;       // last candidate of this lane's share
        const unsigned long long past = __ballot(cu[lo + last + 1] > i);
        const int f = past ? __ffsll((long long)past) - 1 : (n - 1) / step;
        lo += f * step;
        n = n - f * step < step ? n - f * step : step;
    }
    return lo;
}
