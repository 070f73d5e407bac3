// What the operators beside the codec share on the device: element types,
// sums and maxima over a workgroup, argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "df11_ops.h"

namespace df11ops {

struct F32 {
    using raw = float;
    static __device__ float load(raw v) { return v; }
    static __device__ raw store(float v) { return v; }
};
struct BF16 {
    using raw = uint16_t;
    static __device__ float load(raw v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
    static __device__ raw store(float v) {  // to nearest, ties to even
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    }
};
struct F16 {
    using raw = uint16_t;
    static __device__ float load(raw v) {
        return static_cast<float>(__builtin_bit_cast(_Float16, v));
    }
    static __device__ raw store(float v) {
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
    }
};

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ inline float wave_sum(float v) {
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ inline float wave_max(float v) {
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// The workgroup's sum or maximum, the same in every thread; `lds` holds a
// float per wave and is free again on return.
template <int kWavesPerWg>
__device__ inline float wg_sum(float v, float *lds) {
    v = wave_sum(v);
    if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (int w = 0; w < kWavesPerWg; ++w) s += lds[w];
    __syncthreads();
    return s;
}
template <int kWavesPerWg>
__device__ inline float wg_max(float v, float *lds) {
    v = wave_max(v);
    if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = lds[0];
    for (int w = 1; w < kWavesPerWg; ++w) s = fmaxf(s, lds[w]);
    __syncthreads();
    return s;
}

inline bool misaligned(const void *p, uintptr_t to) {
    return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0;
}
inline uint32_t elem_bytes(uint32_t dtype) { return dtype == DF11_F32 ? 4 : 2; }
inline int launched() { return hipGetLastError() == hipSuccess ? DF11_OK : DF11_E_HIP; }

}  // namespace df11ops
