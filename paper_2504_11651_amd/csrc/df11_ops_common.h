// What the operators beside the codec share on the device: element types,
// sums and maxima over a workgroup, argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "df11_ops.h"

namespace df11ops {

// An element type: `raw` as it lies in memory, `get` the e-th of the 16 bytes
// that one load brings.
struct F32 {
    using raw = float;
    static constexpr uint32_t kVec = 4;
    static constexpr uint32_t kMasked = 0xFF800000u;  // -inf
    static __device__ float load(raw v) { return v; }
    static __device__ raw store(float v) { return v; }
    static __device__ float get(const uint4 &q, uint32_t e) {
        return __uint_as_float(e == 0 ? q.x : e == 1 ? q.y : e == 2 ? q.z : q.w);
    }
};
struct BF16 {
    using raw = uint16_t;
    static constexpr uint32_t kVec = 8;
    static constexpr uint32_t kMasked = 0xFF80u;
    static __device__ float load(raw v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
    static __device__ raw store(float v) {  // to nearest, ties to even
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    }
    static __device__ float get(const uint4 &q, uint32_t e) {
        const uint32_t w = e < 2 ? q.x : e < 4 ? q.y : e < 6 ? q.z : q.w;
        return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    }
};
struct F16 {
    using raw = uint16_t;
    static constexpr uint32_t kVec = 8;
    static constexpr uint32_t kMasked = 0xFC00u;
    static __device__ float load(raw v) {
        return static_cast<float>(__builtin_bit_cast(_Float16, v));
    }
    static __device__ raw store(float v) {
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
    }
    static __device__ float get(const uint4 &q, uint32_t e) {
        const uint32_t w = e < 2 ? q.x : e < 4 ? q.y : e < 6 ? q.z : q.w;
        return load(static_cast<uint16_t>(e & 1 ? w >> 16 : w));
    }
};

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;

// 16 bytes at any address that the element type itself allows: gfx950 reads and
// writes them in one instruction whatever their alignment.
template <class R>
__device__ inline uint4 load16(const R *p) {
    uint4 q;
    __builtin_memcpy(&q, p, 16);
    return q;
}
template <class R>
__device__ inline void store16(R *p, const uint4 &q) {
    __builtin_memcpy(p, &q, 16);
}

// The wave's reduction, the same in every lane: five DPP moves inside the
// vector registers and a read of the last lane.  `none` changes nothing.
template <class Op>
__device__ inline uint32_t wave_reduce(uint32_t v, uint32_t none, Op op) {
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x111, 0xF, 0xF, false));  // row_shr 1
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x112, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x114, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x118, 0xF, 0xF, false));
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x142, 0xA, 0xF, false));  // row_bcast 15
    v = op(v, __builtin_amdgcn_update_dpp(none, v, 0x143, 0xC, 0xF, false));  // row_bcast 31
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ inline float wave_sum(float v) {
    return __uint_as_float(wave_reduce(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
__device__ inline float wave_max(float v) {
    return __uint_as_float(wave_reduce(__float_as_uint(v), 0xFF800000u, [](uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
}
__device__ inline uint32_t wave_sum(uint32_t v) {
    return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return a + b; });
}
__device__ inline uint32_t wave_max(uint32_t v) {
    return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ inline uint32_t wave_min(uint32_t v) {
    return wave_reduce(v, ~0u, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

inline bool misaligned(const void *p, uintptr_t to) {
    return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0;
}
inline uint32_t elem_bytes(uint32_t dtype) { return dtype == DF11_F32 ? 4 : 2; }
inline int launched() { return hipGetLastError() == hipSuccess ? DF11_OK : DF11_E_HIP; }

}  // namespace df11ops
