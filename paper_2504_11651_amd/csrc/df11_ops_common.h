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
    static __device__ uint32_t bits(raw v) { return __float_as_uint(v); }
    static __device__ float get(const uint4 &q, uint32_t e) {
        return __uint_as_float(word(q, e));
    }
    static __device__ uint32_t word(const uint4 &q, uint32_t e) {
        return e == 0 ? q.x : e == 1 ? q.y : e == 2 ? q.z : q.w;
    }
    // a maximum over words: v_max3 as it is (fmaxf adds an operation for each
    // operand that might be a signalling NaN; here that makes the maximum a NaN,
    // and the row has no distribution either way)
    struct Max {
        float m = -INFINITY;
        __device__ void add(uint32_t v, uint32_t w) {
            asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m) : "v"(v), "v"(w));
        }
        __device__ float value() const { return m; }
    };
    // value e >= least: `least` from at_least() for the value's place
    static __device__ float at_least(float least, uint32_t) { return least; }
    static __device__ float rough(const uint4 &q, uint32_t e) { return get(q, e); }
};
// The maximum of 16-bit floats, two to a word, without cutting them out: the
// bits of a sign and a magnitude are in order as integers where one of them is
// not negative, and in reverse where all are.
template <class T>
struct PackedMax {
    typedef short s2 __attribute__((ext_vector_type(2)));
    typedef unsigned short u2 __attribute__((ext_vector_type(2)));
    s2 high = {-32768, -32768};
    u2 low = {65535, 65535};
    __device__ void add(uint32_t v, uint32_t w) {
        high = __builtin_elementwise_max(high, __builtin_bit_cast(s2, v));
        low = __builtin_elementwise_min(low, __builtin_bit_cast(u2, v));
        high = __builtin_elementwise_max(high, __builtin_bit_cast(s2, w));
        low = __builtin_elementwise_min(low, __builtin_bit_cast(u2, w));
    }
    __device__ float value() const {
        const float a = T::load(static_cast<uint16_t>(high[0] >= 0 ? high[0] : low[0]));
        const float b = T::load(static_cast<uint16_t>(high[1] >= 0 ? high[1] : low[1]));
        return fmaxf(a, b);
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
    static __device__ uint32_t bits(raw v) { return v; }
    static __device__ float get(const uint4 &q, uint32_t e) {
        const uint32_t w = F32::word(q, e / 2);
        return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    }
    using Max = PackedMax<BF16>;
    // A word taken as a float is its upper value with the lower one's bits behind
    // its mantissa: it compares with a rounded bound as the upper value does, which
    // need not be cut out first.  (-inf becomes a NaN: not at least anything.)  The
    // bound of a negative value, and of 0 for the sake of -0, has all those bits set.
    static __device__ float at_least(float least, uint32_t e) {
        const uint32_t u = __float_as_uint(least == 0.0f ? -0.0f : least);
        return e & 1 && u & 0x80000000u ? __uint_as_float(u | 0xFFFFu) : least;
    }
    static __device__ float rough(const uint4 &q, uint32_t e) {
        const uint32_t w = F32::word(q, e / 2);
        return __uint_as_float(e & 1 ? w : w << 16);
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
    static __device__ uint32_t bits(raw v) { return v; }
    static __device__ float get(const uint4 &q, uint32_t e) {
        const uint32_t w = F32::word(q, e / 2);
        return load(static_cast<uint16_t>(e & 1 ? w >> 16 : w));
    }
    using Max = PackedMax<F16>;
    static __device__ float at_least(float least, uint32_t) { return least; }
    static __device__ float rough(const uint4 &q, uint32_t e) { return get(q, e); }
};

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;

// 16 bytes at any address that the element type itself allows: gfx950 reads and
// writes them in one instruction whatever their alignment.  `once`: they are not
// used again before much else is, and need not be kept in the caches.
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(2)));
template <class R>
__device__ inline uint4 load16(const R *p) {
    const words4 q = *reinterpret_cast<const words4 *>(p);
    return uint4{q[0], q[1], q[2], q[3]};
}
template <class R>
__device__ inline uint4 load16_once(const R *p) {
    const words4 q = __builtin_nontemporal_load(reinterpret_cast<const words4 *>(p));
    return uint4{q[0], q[1], q[2], q[3]};
}
template <class R>
__device__ inline void store16(R *p, const uint4 &q) {
    *reinterpret_cast<words4 *>(p) = words4{q.x, q.y, q.z, q.w};
}
template <class R>
__device__ inline void store16_once(R *p, const uint4 &q) {
    __builtin_nontemporal_store(words4{q.x, q.y, q.z, q.w}, reinterpret_cast<words4 *>(p));
}
// Between the two kinds of access of a branch: alike but for that, the compiler
// would make one plain access of them.
__device__ inline void keep_apart() { asm volatile("" ::: "memory"); }

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
        asm("v_max_f32 %0, %0, %1" : "+v"(a) : "v"(b));
        return a;
    }));
}
__device__ inline double wave_sum(double v) {
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
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
