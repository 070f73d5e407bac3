// Operators on rows of logits: log probabilities of given tokens with rank,
// entropy and top alternatives, distillation from a teacher's top log
// probabilities, and the gradients of both.
//
// The least they can do is to read the logits (and write the gradient).  A row is
// cut into parts of 8192 values, a workgroup takes one part and holds it in
// registers (32 values a lane, all loads issued at once), so the logits are read
// once however many statistics are wanted.  A second kernel joins the parts of a
// row:
//   - the maximum first, then sum exp2((z - max) log2e / tau) with that maximum
//     fixed, per wave; waves and parts are joined by scaling with the
//     exponential of the difference of their maxima;
//   - sum e x beside sum e gives the entropy without a second pass;
//   - the alternatives: of the 256 lanes' maxima (they are there already) a
//     value with at least `top` lanes at or above it is found by bisection over
//     the ordered bits; no value below it can be among the `top` largest, and
//     only few are above (about 1.3 top for values in any order).  They go to
//     the workspace unordered; the join orders the few that are left, by value
//     and index, which are distinct, so the order they arrived in is gone;
//   - where more than the workspace has room for are above (equal values, ordered
//     ones), a higher bound is found by bisection, and equal values are taken in
//     the order of their indices.
// Rows that start at any address are read with unaligned 16-byte loads.
//
// Kernel times, and what bounds them (4096 rows of 128,256 bf16 values are 1.05 GB:
// 215 us at the 4.9 TB/s of a device copy):
//   64 alternatives    parts 270 us, join 41 us: instruction issue, about 19
//                      vector instructions a value, a third of them for the
//                      alternatives (the threshold, and the values above it);
//   distillation       parts 202 us (5.2 TB/s), join 11, gradient 346 us (6.1
//                      TB/s, reads and writes past the caches): memory;
//   one row, fp32, 20  parts 6.6 us, join 6.9: loads and barriers after one another.
// Holding two parts, with the next one's loads under way while one is worked on,
// takes registers for half the waves and was slower (283 against 240 us); groups of
// rows whose logits stay in the memory-side cache between the two passes of the
// distillation end too many launches early (656 against 600 us at 192 MB).
#include "df11_ops_common.h"

#include <algorithm>
#include <limits>

namespace {

using namespace df11ops;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kWaves = kThreads / 64;
constexpr uint32_t kPerLane = 32;
constexpr uint32_t kPart = kThreads * kPerLane;  // values of a row in one workgroup
template <class T>
constexpr int kOccupancy = T::kVec == 4 ? 6 : 8;  // waves on a SIMD
template <class T>
constexpr uint32_t kVecs = kPerLane / T::kVec;  // 16-byte loads of a lane

// 1/tau and log2e/tau, in the forms that the kernels multiply by.
struct Tau {
    float two_over;  // 2/tau: differences of halves are multiplied by it
    float c, rest;   // log2e/tau in two parts: one would be off by |x| 2^-25 in x, the
                     // same way in every value, and so in the sum
    float two_c, two_rest;  // the same for differences of halves
    double over;     // 1/tau
    explicit Tau(float tau) : two_over(2.0f / tau), over(1.0 / tau) {
        // the first part from below, so that the second is positive and a masked
        // value stays -inf
        c = static_cast<float>(M_LOG2E / tau);
        if (c >= M_LOG2E / tau) c = std::nextafterf(c, 0.0f);
        rest = static_cast<float>(M_LOG2E / tau - c);
        // not 0 where that is below the float range (tau of 10^37 and more): 0 * -inf
        if (rest == 0.0f) rest = std::numeric_limits<float>::denorm_min();
        two_c = std::min(2.0f * c, std::numeric_limits<float>::max());  // not 0 * inf
        two_rest = 2.0f * rest;
    }
};

// (v - m) / tau, of halves so that the difference of two finite values is finite
__device__ float scaled(float v, float m, float two_over_tau) {
    return fmaf(v, 0.5f, -0.5f * m) * two_over_tau;
}

// (v - m) log2e / tau, to 2^-23 of itself and no worse however large m is
__device__ float exponent(float v, float m, const Tau &tau) {
    const float d = fmaf(v, 0.5f, -0.5f * m);
    return fmaf(d, tau.two_rest, d * tau.two_c);
}

// Bits in the order of the values: unsigned comparison.  -0 is +0.
__device__ uint32_t ordered(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ (u & 0x80000000u ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ float from_ordered(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kOrderedMasked = 0x007FFFFFu;  // of -inf

// How many lanes below this one have their bit set.
__device__ uint32_t before(uint64_t all) {
    return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(all >> 32),
                                     __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(all), 0u));
}

// The next larger float; of -inf the lowest finite one.
__device__ float above_of(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return __uint_as_float(u & 0x80000000u ? u - 1 : u + 1);
}

// A lane's values of a part: vector i of the lane holds the values from
// part + (256 i + thread) * kVec.  What lies past the row is masked.
template <class T>
struct Held {
    uint4 q[kVecs<T>];

    __device__ static uint32_t first(uint32_t part, uint32_t i) {
        return part + (kThreads * i + threadIdx.x) * T::kVec;
    }
    __device__ void load(const typename T::raw *z, uint32_t part, uint32_t vocab, bool once) {
        if (part + kPart <= vocab && once) {
            keep_apart();
#pragma unroll
            for (uint32_t i = 0; i < kVecs<T>; ++i) q[i] = load16_once(z + first(part, i));
            keep_apart();
            return;
        }
        if (part + kPart <= vocab) {
#pragma unroll
            for (uint32_t i = 0; i < kVecs<T>; ++i) q[i] = load16(z + first(part, i));
            return;
        }
        // whole vectors first, all loads under way before the first is looked at;
        // then the lane whose vector the row's end cuts takes single values
        constexpr uint32_t both = T::kVec == 8 ? T::kMasked * 0x10001u : T::kMasked;
#pragma unroll
        for (uint32_t i = 0; i < kVecs<T>; ++i) {
            const uint32_t j = first(part, i);
            q[i] = uint4{both, both, both, both};
            if (j + T::kVec <= vocab) q[i] = load16(z + j);
        }
#pragma unroll
        for (uint32_t i = 0; i < kVecs<T>; ++i) {
            const uint32_t j = first(part, i);
            if (j < vocab && j + T::kVec > vocab) q[i] = cut_vector(z + j, vocab - j);
        }
    }
    __device__ static uint4 cut_vector(const typename T::raw *z, uint32_t n) {
        constexpr uint32_t kEach = 4 / sizeof(typename T::raw);
        uint32_t w[4];
        for (uint32_t k = 0; k < 4; ++k) {
            w[k] = T::kVec == 8 ? T::kMasked * 0x10001u : T::kMasked;
            for (uint32_t e = 0; e < kEach; ++e)
                {
                    const uint32_t i = k * kEach + e, v = T::bits(z[min(i, n - 1)]);
                    const uint32_t at = 16 * e, mask = kEach == 2 ? 0xFFFFu : ~0u;
                    w[k] = i < n ? (w[k] & ~(mask << at)) | v << at : w[k];
                }
        }
        return uint4{w[0], w[1], w[2], w[3]};
    }
    // Keeps the compiler from holding the values cut out in one pass for the next:
    // cutting them out again is cheaper than the registers.
    __device__ void again() {
#pragma unroll
        for (uint32_t i = 0; i < kVecs<T>; ++i)
            asm volatile("" : "+v"(q[i].x), "+v"(q[i].y), "+v"(q[i].z), "+v"(q[i].w));
    }
    template <class F>
    __device__ void each(F f) const {  // f(value, vector, element)
#pragma unroll
        for (uint32_t i = 0; i < kVecs<T>; ++i)
#pragma unroll
            for (uint32_t e = 0; e < T::kVec; ++e) f(T::get(q[i], e), i, e);
    }
    __device__ float max() const {
        typename T::Max m;
#pragma unroll
        for (uint32_t i = 0; i < kVecs<T>; ++i) {
            m.add(q[i].x, q[i].y);
            m.add(q[i].z, q[i].w);
        }
        return m.value();
    }
};

// (v - m) / tau where a row's few results are made of it.
__device__ double scaled64(float v, float m, const Tau &tau) {
    return (static_cast<double>(v) - static_cast<double>(m)) * tau.over;
}

// What a part, or several, says about its row: maximum (at least the lowest
// finite value, so that masked values give exp(-inf)), sum e, sum e x in powers of
// two for the entropy, and how many values are above the token's.
struct PartStat {
    float m, s, t;
    uint32_t above;
};
// The same for the distillation: maximum and sum e of all values, and of those at
// places that the teacher does not name, which may be less than 32 bits hold
// beside the first.  The second maximum may be larger than the values are.
struct PairStat {
    float m, s, other_m, other_s;
};

// x = (v - m) log2e / tau for the values of a wave with the wave's maximum m, up
// to a shift that is the same for all of them: v c - m c, fused, with m c rounded.
// The shift, that rounding and (with the second part of c) m times it, goes through
// exp2 and is taken out of the sums again, so it must be small: below 1 for |m c| up
// to 2^22.  Beyond (waves of masks of -1e9 or the lowest finite value, logits of
// millions) the differences are taken first.
struct Exponent {
    float m, c, rest, mc, two_over_tau;
    bool near;
    // `most`: the wave's maximum, -inf where all is masked (then x is -inf)
    __device__ Exponent(float most, const Tau &tau)
        : m(fmaxf(most, kLowest)), c(tau.c), rest(tau.rest),
          mc(most == -INFINITY ? 0.0f : m * c), two_over_tau(tau.two_over),
          near(fabsf(mc) < 4194304.0f) {}
    // what is to be taken from x: m c, with the second part of c if x has it, is mc
    // plus this
    __device__ float shift(bool whole) const {
        if (!near || mc == 0.0f) return 0.0f;
        return whole ? fmaf(m, rest, fmaf(m, c, -mc)) : fmaf(m, c, -mc);
    }
    // Without the second part each x is short of a 2^-24th, so that sum e is short of
    // that times ln 2 sum e x, and sum e x of that times itself, to first order.
    __device__ float more() const { return near ? rest / c : 0.0f; }
    // kWhole: with the second part of c; without it the sums are corrected by more()
    template <class T, bool kWhole>
    __device__ void operator()(const uint4 &q, float *v, float *x) const {
#pragma unroll
        for (uint32_t k = 0; k < T::kVec; ++k) {
            v[k] = T::get(q, k);
            x[k] = fmaf(v[k], c, -mc);
            if constexpr (kWhole) x[k] = fmaf(v[k], rest, x[k]);
        }
        if (!near) {
            float far = two_over_tau;
            asm volatile("" : "+v"(far));  // a branch, not a selection for every value
#pragma unroll
            for (uint32_t k = 0; k < T::kVec; ++k) x[k] = scaled(v[k], m, far) * kLog2e;
        }
    }
};

// Sums with maximum m scaled to the larger maximum M: the factor, and for the
// sum of e x the shift of x.
__device__ void rescale(const PartStat &p, float M, float two_over_tau, float *s, float *t) {
    const float d = fmaxf(scaled(p.m, M, two_over_tau) * kLog2e, -300.0f);
    const float f = d <= -300.0f ? 0.0f : __builtin_amdgcn_exp2f(d);
    *s += p.s * f;
    *t += f * fmaf(d, p.s, p.t);
}
// One sum, scaled so.
__device__ float rescaled(float s, float m, float M, float two_over_tau) {
    const float d = fmaxf(scaled(m, M, two_over_tau) * kLog2e, -300.0f);
    return s * (d <= -300.0f ? 0.0f : __builtin_amdgcn_exp2f(d));
}

// The waves' statistics as one, by every thread, after a barrier.
__device__ PartStat join_waves(const PartStat *w, float two_over_tau) {
    PartStat p{w[0].m, 0.0f, 0.0f, 0};
    for (uint32_t i = 1; i < kWaves; ++i) p.m = fmaxf(p.m, w[i].m);
    for (uint32_t i = 0; i < kWaves; ++i) {
        rescale(w[i], p.m, two_over_tau, &p.s, &p.t);
        p.above += w[i].above;
    }
    return p;
}
__device__ PairStat join_two(const PairStat &a, const PairStat &b, float two_over_tau) {
    PairStat p{fmaxf(a.m, b.m), 0.0f, fmaxf(a.other_m, b.other_m), 0.0f};
    p.s = rescaled(a.s, a.m, p.m, two_over_tau) + rescaled(b.s, b.m, p.m, two_over_tau);
    p.other_s = rescaled(a.other_s, a.other_m, p.other_m, two_over_tau) +
                rescaled(b.other_s, b.other_m, p.other_m, two_over_tau);
    return p;
}
__device__ PairStat join_waves(const PairStat *w, float two_over_tau) {
    PairStat p{w[0].m, 0.0f, w[0].other_m, 0.0f};
    for (uint32_t i = 1; i < kWaves; ++i) {
        p.m = fmaxf(p.m, w[i].m);
        p.other_m = fmaxf(p.other_m, w[i].other_m);
    }
    for (uint32_t i = 0; i < kWaves; ++i) {
        p.s += rescaled(w[i].s, w[i].m, p.m, two_over_tau);
        p.other_s += rescaled(w[i].other_s, w[i].other_m, p.other_m, two_over_tau);
    }
    return p;
}

constexpr PartStat kNoStat{kLowest, 0.0f, 0.0f, 0};
constexpr PairStat kNoPair{kLowest, 0.0f, kLowest, 0.0f};

// The parts' statistics of a row as one, by a wave.  `mine`: this lane's, of the
// first 64.
__device__ PartStat join_parts(PartStat mine, const PartStat *stat, uint32_t parts,
                               float two_over_tau, uint64_t *above) {
    const uint32_t lane = threadIdx.x & 63u;
    uint64_t count = mine.above;
    for (uint32_t i = lane + 64; i < parts; i += 64) {  // past 524,288 values
        const PartStat p = stat[i];
        const float M = fmaxf(mine.m, p.m);
        PartStat both{M, 0.0f, 0.0f, 0};
        rescale(mine, M, two_over_tau, &both.s, &both.t);
        rescale(p, M, two_over_tau, &both.s, &both.t);
        count += p.above;
        mine = both;
    }
    PartStat row{wave_max(mine.m), 0.0f, 0.0f, 0};
    float s = 0.0f, t = 0.0f;
    rescale(mine, row.m, two_over_tau, &s, &t);
    row.s = wave_sum(s);
    row.t = wave_sum(t);
    *above = static_cast<uint64_t>(wave_sum(static_cast<uint32_t>(count >> 16))) * 65536u +
             wave_sum(static_cast<uint32_t>(count & 0xFFFFu));
    return row;
}
__device__ PairStat join_parts(PairStat mine, const PairStat *stat, uint32_t parts,
                               float two_over_tau) {
    for (uint32_t i = (threadIdx.x & 63u) + 64; i < parts; i += 64)
        mine = join_two(mine, stat[i], two_over_tau);
    PairStat row{wave_max(mine.m), 0.0f, wave_max(mine.other_m), 0.0f};
    row.s = wave_sum(rescaled(mine.s, mine.m, row.m, two_over_tau));
    row.other_s = wave_sum(rescaled(mine.other_s, mine.other_m, row.other_m, two_over_tau));
    return row;
}

// ------------------------------------------------------------ log probabilities
struct LogprobArgs {
    const void *logits;
    const int64_t *tokens;
    PartStat *stat;      // rows x parts
    uint32_t *count;     // rows x parts: candidates
    uint2 *candidate;    // rows x parts x room: ordered bits, index
    float *logprob, *entropy, *top_logprob, *stats;
    int64_t *rank, *top_index;
    uint64_t stride;
    uint32_t vocab, parts, top, room;
    Tau tau;
    bool once;
};

// Values above the threshold that a part may bring: twice what is wanted, and
// some, so that equal neighbours (bf16 has 8 bits of mantissa) fit.
__host__ __device__ constexpr uint32_t room_of(uint32_t top) { return top ? 2 * top + 64 : 0; }

// A workgroup's sum of a count, by every thread.
__device__ uint32_t wg_sum(uint32_t n, uint32_t *lds) {
    n = wave_sum(n);
    __syncthreads();
    if ((threadIdx.x & 63u) == 0) lds[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0;
    for (uint32_t w = 0; w < kWaves; ++w) n += lds[w];
    return n;
}

// Of 256 keys, one a lane in lane_key[], the largest that `top` of them reach,
// or one that only some more do; 0 unmasked keys below `top`: the least of all
// that are not masked.  Every wave finds the same, without a barrier.
__device__ uint32_t reached_by(const uint32_t *lane_key, uint32_t top) {
    uint32_t key[kWaves], high = 0, low = ~0u, there = 0;
    for (uint32_t i = 0; i < kWaves; ++i) {
        key[i] = lane_key[64 * i + (threadIdx.x & 63u)];
        const bool some = key[i] > kOrderedMasked;
        there += __popcll(__ballot(some));
        high = max(high, key[i]);
        low = min(low, some ? key[i] : ~0u);
    }
    if (there < top) return kOrderedMasked + 1;
    high = wave_max(high);
    uint32_t cut = wave_min(low);
    while (cut < high) {
        const uint32_t mid = high - (high - cut) / 2;
        uint32_t n = 0;
        for (uint32_t i = 0; i < kWaves; ++i) n += __popcll(__ballot(key[i] >= mid));
        if (n >= top) {
            cut = mid;
            if (n <= top + top / 4 + 2) break;
        } else {
            high = mid - 1;
        }
    }
    return cut;
}

// Where more of a part's values reach `cut` than there is room for: the least
// bound above that leaves room, by bisection over all values (the next value where
// those equal to `cut` are the many), or, where equal values are too many for any
// bound, those above them and the first of them in the order of the indices.
// Returns how many values it wrote, `top` at least.  Reads the part again: it is
// rare, and the registers it would need are not.
template <class T>
__device__ inline uint32_t trim_part(const typename T::raw *z, uint32_t part, uint32_t vocab,
                                     uint32_t cut, uint32_t top, uint32_t room, uint2 *out,
                                     uint32_t *lds) {
    const uint32_t to = min(kPart, vocab - part), wave = threadIdx.x >> 6;
    z += part;
    auto count = [&](auto f) {
        uint32_t n = 0;
#pragma unroll 4
        for (uint32_t i = threadIdx.x; i < to; i += kThreads) n += f(T::load(z[i])) ? 1u : 0u;
        return wg_sum(n, lds);
    };
    // values above `last` are taken; `larger` of them
    uint32_t lo = cut, hi = 0xFF800000u;  // ordered bits of +inf
    float last = from_ordered(lo);
    uint32_t larger = count([&](float v) { return v > last; });
    while (larger > room && lo < hi) {
        const uint32_t mid = hi - (hi - lo) / 2;
        const float at = from_ordered(mid);
        if (count([&](float v) { return v >= at; }) >= top) {
            lo = mid;
            last = at;
            larger = count([&](float v) { return v > at; });
        } else {
            hi = mid - 1;
        }
    }
    if (larger) {
        __syncthreads();
        if (threadIdx.x == 0) lds[0] = 0;
        __syncthreads();
#pragma unroll 4
        for (uint32_t i = threadIdx.x; i < to; i += kThreads) {
            const float v = T::load(z[i]);
            if (v > last) {
                const uint32_t slot = atomicAdd(&lds[0], 1u);
                if (slot < room) out[slot] = uint2{ordered(v), part + i};
            }
        }
    }
    uint32_t n = larger;
    for (uint32_t i0 = 0; i0 < to && n < top; i0 += kThreads) {
        const uint32_t i = i0 + threadIdx.x;
        const bool equal = i < to && T::load(z[min(i, to - 1)]) == last;
        const uint64_t all = __ballot(equal);
        __syncthreads();
        if ((threadIdx.x & 63u) == 0) lds[wave] = __popcll(all);
        __syncthreads();
        uint32_t slot = n + before(all), here = 0;
        for (uint32_t w = 0; w < kWaves; ++w) {
            slot += w < wave ? lds[w] : 0;
            here += lds[w];
        }
        if (equal && slot < top) out[slot] = uint2{ordered(last), part + i};
        n = min(n + here, max(top, n));
    }
    return n;
}

template <class T, bool kTop>
__device__ void logprob_part(const LogprobArgs &g) {
    __shared__ PartStat wave_stat[kWaves];
    __shared__ uint32_t lane_key[kTop ? kThreads : 1], counts[kWaves], shared_cut;
    const uint32_t wave_of = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __shared__ uint2 list[kTop ? kWaves : 1][kTop ? room_of(DF11_MAX_TOP) : 1];
    const uint32_t row_parts = g.parts;
    const uint64_t row = blockIdx.x / row_parts;
    const uint32_t part = (blockIdx.x % row_parts) * kPart;
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    Held<T> h;
    h.load(z, part, g.vocab, g.once);

    const int64_t token = g.tokens ? g.tokens[row] : -1;
    const bool asked = token >= 0 && token < g.vocab;
    const uint32_t tok = asked ? static_cast<uint32_t>(token) : 0;
    const float zt = asked ? T::load(z[tok]) : __builtin_nanf("");
    const float more = asked ? above_of(zt) : zt;

    const float lane_max = h.max();
    h.again();
    // before the token equal values count, from it on larger ones: one bound for
    // all values of a part, except in the token's own
    const bool here = asked && tok >= part && tok - part < kPart;
    const float rest = part < tok ? zt : more;
    const Exponent x_of(wave_max(lane_max), g.tau);
    float s = 0.0f, t = 0.0f;
    uint32_t above = 0;
#pragma unroll
    for (uint32_t i = 0; i < kVecs<T>; ++i) {
        float v[T::kVec], x[T::kVec], e[T::kVec], sum = 0.0f;
        x_of.operator()<T, false>(h.q[i], v, x);
#pragma unroll
        for (uint32_t k = 0; k < T::kVec; ++k) {
            e[k] = __builtin_amdgcn_exp2f(x[k]);
            s += e[k];
            sum = fmaf(e[k], x[k], sum);
        }
        if (__any(sum != sum)) {  // 0 * -inf of a masked value
            asm volatile("" : "+v"(sum));
            sum = 0.0f;
#pragma unroll
            for (uint32_t k = 0; k < T::kVec; ++k) sum = fmaf(e[k], fmaxf(x[k], -300.0f), sum);
        }
        t += sum;
        if (here) {
            const uint32_t j = h.first(part, i);
#pragma unroll
            for (uint32_t k = 0; k < T::kVec; ++k)
                above += __popcll(__ballot(v[k] >= (j + k < tok ? zt : more)));
        } else {
#pragma unroll
            for (uint32_t k = 0; k < T::kVec; ++k) above += __popcll(__ballot(v[k] >= rest));
        }
        // a vector's values at a time in registers
        asm volatile("" : "+v"(s), "+v"(t), "+s"(above));
    }
    s = wave_sum(s);
    t = wave_sum(t);
    if ((threadIdx.x & 63u) == 0) {
        const float shift = x_of.shift(false), f = __builtin_amdgcn_exp2f(-shift);
        t = fmaf(-shift, s, t);
        s = fmaf(x_of.more() * kLn2, t, s);
        t = fmaf(x_of.more(), t, t);
        wave_stat[threadIdx.x >> 6] = PartStat{x_of.m, s * f, t * f, above};
    }
    if constexpr (kTop) lane_key[threadIdx.x] = ordered(lane_max);
    __syncthreads();
    if (threadIdx.x == 0) g.stat[blockIdx.x] = join_waves(wave_stat, g.tau.two_over);
    if constexpr (kTop) {
        if (wave_of == (blockIdx.x & 3u)) {
            const uint32_t c = reached_by(lane_key, g.top);
            if ((threadIdx.x & 63u) == 0) shared_cut = c;
        }
        __syncthreads();
        const uint32_t cut = shared_cut;
        const float least = from_ordered(cut);
        const uint32_t wave = threadIdx.x >> 6;
        h.again();
        const float low = T::at_least(least, 0), high = T::at_least(least, 1);
        uint32_t n = 0;  // of this wave
#pragma unroll
        for (uint32_t i = 0; i < kVecs<T>; ++i)
#pragma unroll
            for (uint32_t e = 0; e < T::kVec; ++e) {
                const bool in = T::rough(h.q[i], e) >= (e & 1 ? high : low);
                const uint64_t all = __ballot(in);
                if (all) {
                    const uint32_t slot = n + before(all);
                    if (in && slot < g.room)
                        list[wave][slot] = uint2{__float_as_uint(T::get(h.q[i], e)),
                                                 h.first(part, i) + e};
                    n += __popcll(all);
                }
            }
        if ((threadIdx.x & 63u) == 0) counts[wave] = n;
        __syncthreads();
        uint32_t at = 0, total = 0;
        for (uint32_t w = 0; w < kWaves; ++w) {
            at += w < wave ? counts[w] : 0;
            total += counts[w];
        }
        uint2 *out = g.candidate + static_cast<uint64_t>(blockIdx.x) * g.room;
        if (total <= g.room) {
            for (uint32_t i = threadIdx.x & 63u; i < n; i += 64) {
                const uint2 v = list[wave][i];
                out[at + i] = uint2{ordered(__uint_as_float(v.x)), v.y};
            }
        } else {
            total = trim_part<T>(z, part, g.vocab, cut, g.top, g.room, out, counts);
        }
        if (threadIdx.x == 0) g.count[blockIdx.x] = total;
    }
}

template <class T>
__global__ __launch_bounds__(kThreads, kOccupancy<T>) void logprob_part_kernel(LogprobArgs g) {
    logprob_part<T, false>(g);
}
template <class T>
__global__ __launch_bounds__(kThreads, kOccupancy<T>) void logprob_top_kernel(LogprobArgs g) {
    logprob_part<T, true>(g);
}

constexpr uint32_t kSlots = 16;  // candidates that a lane of the join holds
constexpr uint32_t kList = 512;  // that are ordered by counting

// One workgroup per row: the parts' statistics, and of their candidates the
// `top` largest in order.  As in a part, a key that `top` lanes reach leaves
// few (trimmed exactly where equal ones are too many); the place of each of
// them is the number of larger ones, equal keys by their index.  Rows with more
// slots than 4096 take rounds, with what was kept so far as further candidates.
template <class T>
__global__ __launch_bounds__(kThreads) void logprob_join_kernel(LogprobArgs g) {
    __shared__ uint32_t lane_key[kThreads], counts[kWaves];
    __shared__ uint32_t list_key[kList], list_idx[kList], place[kList];
    __shared__ uint32_t best_key[DF11_MAX_TOP], best_idx[DF11_MAX_TOP];
    __shared__ double row_ln_s;
    __shared__ float row_m, row_s;
    const uint64_t row = blockIdx.x, first = row * g.parts;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t key[kSlots + 1], idx[kSlots + 1];
    const uint32_t slots = g.parts * g.room;
    // slots are `room` apart in part: which are filled, then what they hold
    const auto filled = [&](uint32_t from, bool *some) {
        uint32_t q = (from + threadIdx.x) / g.room, r = (from + threadIdx.x) % g.room;
#pragma unroll
        for (uint32_t e = 0; e < kSlots; ++e) {
            some[e] = q < g.parts && r < g.count[first + min(q, g.parts - 1)];
            q += kThreads / g.room;
            r += kThreads % g.room;
            if (r >= g.room) {
                r -= g.room;
                ++q;
            }
        }
    };
    const auto load = [&](uint32_t from, const bool *some) {
#pragma unroll
        for (uint32_t e = 0; e < kSlots; ++e) {
            const uint2 *at = g.candidate + first * g.room + from + kThreads * e + threadIdx.x;
            const uint2 v = some[e] ? *at : uint2{0u, ~0u};
            key[e] = v.x;
            idx[e] = v.y;
        }
    };
    // a row alone is all latency: what does not depend on another load goes first
    const PartStat mine = lane < g.parts ? g.stat[first + lane] : kNoStat;
    const int64_t token = g.tokens ? g.tokens[row] : -1;
    const bool asked = token >= 0 && token < g.vocab;
    if (g.top) {
        bool some[kSlots];
        filled(0, some);
        load(0, some);
    }
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    const float zt = asked ? T::load(z[token]) : 0.0f;
    if (wave == 0) {
        uint64_t above;
        const PartStat p = join_parts(mine, g.stat + first, g.parts, g.tau.two_over, &above);
        const bool broken = !(p.s >= 0.0f) || p.s == INFINITY;
        const bool empty = p.s == 0.0f;
        const float nan = __builtin_nanf("");
        // ln S is about 10, and its rounding to 32 bits would be the largest error
        const double ln_s = log(static_cast<double>(p.s));
        if (lane == 0) {
            float lp = empty ? -INFINITY : static_cast<float>(scaled64(zt, p.m, g.tau) - ln_s);
            const float h =
                broken ? nan : empty ? 0.0f : static_cast<float>(ln_s - M_LN2 * p.t / p.s);
            if (token < 0) lp = 0.0f;
            if ((token >= 0 && !asked) || broken) lp = nan;
            if (g.logprob) g.logprob[row] = lp;
            if (g.rank) g.rank[row] = asked && !broken ? static_cast<int64_t>(above) : -1;
            if (g.entropy) g.entropy[row] = h;
            if (g.stats)
                *reinterpret_cast<float4 *>(g.stats + 4 * row) =
                    float4{p.m, static_cast<float>(ln_s), h, broken ? nan : 1.0f / p.s};
            row_m = p.m;
            row_ln_s = ln_s;
            row_s = broken ? -1.0f : p.s;
        }
    }
    if (!g.top) return;

    uint32_t kept = 0;
    for (uint32_t from = 0;;) {
        key[kSlots] = threadIdx.x < kept ? best_key[threadIdx.x] : 0;
        idx[kSlots] = threadIdx.x < kept ? best_idx[threadIdx.x] : ~0u;
        uint32_t most = 0;
#pragma unroll
        for (uint32_t e = 0; e <= kSlots; ++e) most = max(most, key[e]);
        lane_key[threadIdx.x] = most;
        __syncthreads();
        uint32_t cut = reached_by(lane_key, g.top), last = ~0u, n = 0;
        const auto count = [&](auto f) {
            uint32_t c = 0;
#pragma unroll
            for (uint32_t e = 0; e <= kSlots; ++e) c += f(key[e], idx[e]) ? 1u : 0u;
            return wg_sum(c, counts);
        };
        // how many of each wave's are kept, and of all
        const auto keep = [&](uint32_t e) {
            return key[e] > cut || (key[e] == cut && idx[e] <= last);
        };
        const auto kept_by_waves = [&] {
            uint32_t c = 0;
#pragma unroll
            for (uint32_t e = 0; e <= kSlots; ++e) c += __popcll(__ballot(keep(e)));
            if (lane == 0) counts[wave] = c;
            __syncthreads();
            uint32_t all = 0;
            for (uint32_t w = 0; w < kWaves; ++w) all += counts[w];
            return all;
        };
        n = kept_by_waves();
        if (n > kList) {  // equal ones, or a few lanes with all the large ones
            __syncthreads();
            uint32_t hi = ~0u;
            while (cut < hi) {
                const uint32_t mid = hi - (hi - cut) / 2;
                const uint32_t c = count([&](uint32_t k, uint32_t) { return k >= mid; });
                if (c >= g.top) {
                    cut = mid;
                    n = c;
                    if (c <= kList) break;
                } else {
                    hi = mid - 1;
                }
            }
            uint32_t low = 0;
            while (n > kList && low < last) {
                const uint32_t mid = low + (last - low) / 2;
                const uint32_t c = count(
                    [&](uint32_t k, uint32_t i) { return k > cut || (k == cut && i <= mid); });
                if (c >= g.top) {
                    last = mid;
                    n = c;
                } else {
                    low = mid + 1;
                }
            }
            __syncthreads();
            n = kept_by_waves();
        }
        // to the list: each wave behind those below it
        uint32_t at = 0;
        for (uint32_t w = 0; w < wave; ++w) at += counts[w];
#pragma unroll
        for (uint32_t e = 0; e <= kSlots; ++e) {
            const bool in = keep(e);
            const uint64_t all = __ballot(in);
            if (in) {
                list_key[at + before(all)] = key[e];
                list_idx[at + before(all)] = idx[e];
            }
            at += __popcll(all);
        }
        for (uint32_t c = threadIdx.x; c < n; c += kThreads) place[c] = 0;
        __syncthreads();
        // each wave counts over a quarter of the list
        const uint32_t lo = wave * n / kWaves, hi = (wave + 1) * n / kWaves;
        for (uint32_t c = lane; c < n; c += 64) {
            const uint32_t k = list_key[c], i = list_idx[c];
            uint32_t larger = 0, same = c >= lo && c < hi ? ~0u : 0;
#pragma unroll 4
            for (uint32_t d = lo; d < hi; ++d) {
                larger += list_key[d] > k ? 1u : 0u;
                same += list_key[d] == k ? 1u : 0u;
            }
            if (__any(same != 0)) {  // equal keys: by their indices
#pragma unroll 4
                for (uint32_t d = lo; d < hi; ++d) {
                    const bool first = (list_key[d] == k) & (list_idx[d] < i);
                    larger += first ? 1u : 0u;
                }
            }
            atomicAdd(&place[c], larger);
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < n; c += kThreads)
            if (place[c] < g.top) {
                best_key[place[c]] = list_key[c];
                best_idx[place[c]] = list_idx[c];
            }
        __syncthreads();
        kept = min(n, g.top);
        from += kThreads * kSlots;
        if (from >= slots) break;
        bool some[kSlots];
        filled(from, some);
        load(from, some);
    }
    const bool broken = row_s < 0.0f;
    for (uint32_t k = threadIdx.x; k < g.top; k += kThreads) {
        const bool some = k < kept;
        const double x = scaled64(from_ordered(best_key[k]), row_m, g.tau);
        const float lp = static_cast<float>(x - row_ln_s);
        g.top_logprob[row * g.top + k] = broken ? __builtin_nanf("") : some ? lp : -INFINITY;
        g.top_index[row * g.top + k] = broken || !some ? -1 : static_cast<int64_t>(best_idx[k]);
    }
}

struct LogprobGradArgs {
    const void *logits;
    void *grad;
    const int64_t *tokens;
    const float *stats, *grad_logprob, *grad_entropy;
    uint64_t stride, grad_stride;
    uint32_t vocab, parts;
    Tau tau;
    bool once;
};

// Writes f(value, index) for the values of a part.
template <class T, bool kOnce, class F>
__device__ void store_values(const Held<T> &h, typename T::raw *out, uint32_t part, uint32_t vocab,
                             F f) {
#pragma unroll
    for (uint32_t i = 0; i < kVecs<T>; ++i) {
        const uint32_t j = Held<T>::first(part, i);
        typename T::raw r[T::kVec];
#pragma unroll
        for (uint32_t e = 0; e < T::kVec; ++e) r[e] = T::store(f(T::get(h.q[i], e), j + e));
        if (j + T::kVec <= vocab) {
            if constexpr (kOnce)
                store16_once(out + j, __builtin_bit_cast(uint4, r));
            else
                store16(out + j, __builtin_bit_cast(uint4, r));
        } else {
#pragma unroll
            for (uint32_t e = 0; e < T::kVec; ++e)
                if (j + e < vocab) out[j + e] = r[e];
        }
    }
}
template <class T, class F>
__device__ void store_part(const Held<T> &h, typename T::raw *out, uint32_t part, uint32_t vocab,
                           bool once, F f) {
    if (once) {
        keep_apart();
        store_values<T, true>(h, out, part, vocab, f);
        keep_apart();
    } else {
        store_values<T, false>(h, out, part, vocab, f);
    }
}

// grad = p (A + B x), p = exp2(x) / S: the formula with its factors drawn together.
// S comes as 1/S: of ln S, which is about 10, 32 bits leave 5e-7 of every p.
// The token's value, the only other one, is written by the lane that holds it.
template <class T>
__global__ __launch_bounds__(kThreads, 8) void logprob_grad_kernel(LogprobGradArgs g) {
    const uint64_t row = blockIdx.x / g.parts;
    const uint32_t part = (blockIdx.x % g.parts) * kPart;
    Held<T> h;
    h.load(static_cast<const typename T::raw *>(g.logits) + row * g.stride, part, g.vocab, g.once);
    auto *out = static_cast<typename T::raw *>(g.grad) + row * g.grad_stride;
    const int64_t token = g.tokens ? g.tokens[row] : -1;
    const float4 st = *reinterpret_cast<const float4 *>(g.stats + 4 * row);
    const float m = st.x, ln_s = st.y, entropy = st.z;
    const float over_tau = 0.5f * g.tau.two_over;
    float gl = g.grad_logprob && token >= 0 ? g.grad_logprob[row] : 0.0f;
    if (token >= static_cast<int64_t>(g.vocab)) gl = __builtin_nanf("");
    const float ge = g.grad_entropy ? g.grad_entropy[row] : 0.0f;
    const bool empty = ln_s == -INFINITY;
    const float over = over_tau * st.w;
    const float A = -over * fmaf(ge, entropy - ln_s, gl), B = -over * ge * kLn2;
    const float hit = over_tau * gl;
    const uint32_t tok = token >= 0 && token < g.vocab ? static_cast<uint32_t>(token) : ~0u;
    store_part(h, out, part, g.vocab, g.once, [&](float v, uint32_t j) {
        const float x = exponent(v, m, g.tau);
        const float d = __builtin_amdgcn_exp2f(x) * fmaf(B, fmaxf(x, -300.0f), A);
        return empty ? 0.0f : j == tok ? d + hit : d;
    });
}

// ---------------------------------------------------------------- distillation
struct DistillArgs {
    const void *logits;
    void *grad;
    const int64_t *index;
    const float *teacher, *weight;
    PairStat *stat;
    float *loss, *stats;
    uint64_t stride, grad_stride;
    uint32_t vocab, parts, top, tail;
    Tau tau;
    bool once;
};

// Whether the teacher's entry is there, and whether it is out of range.
__device__ bool named(int64_t place) { return place >= 0; }
__device__ bool bad_entry(int64_t place, float logprob, uint32_t vocab) {
    return place >= 0 && (place >= static_cast<int64_t>(vocab) || !(logprob < INFINITY));
}

// sum e and the sum over the places that the teacher does not name: these are
// a bit for each value of the part in LDS (1 KB), a lane reads its vector's.
// The second sum is kept beside the first, not taken from it by subtraction:
// where the named places have nearly all the probability nothing would be left.
// Where they have more than that, it is taken relative to its own maximum.
template <class T>
__global__ __launch_bounds__(kThreads, 8) void distill_part_kernel(DistillArgs g) {
    __shared__ PairStat wave_stat[kWaves];
    __shared__ uint32_t bits[kPart / 32];
    const uint64_t row = blockIdx.x / g.parts;
    const uint32_t part = (blockIdx.x % g.parts) * kPart;
    Held<T> h;
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    h.load(z, part, g.vocab, g.once);
    static_assert(kPart / 32 == kThreads, "a word a thread");
    bits[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < g.top; k += kThreads) {
        const int64_t i = g.index[row * g.top + k];
        if (i >= part && i < int64_t{part} + kPart)
            atomicOr(&bits[(i - part) >> 5], 1u << ((i - part) & 31));
    }
    __syncthreads();
    const Exponent x_of(wave_max(h.max()), g.tau);
    h.again();
    // a vector at a time: few of them have a named place in any lane
    float s = 0.0f, t = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < kVecs<T>; ++i) {
        float v[T::kVec], e[T::kVec], sum = 0.0f;
        x_of.operator()<T, true>(h.q[i], v, e);
#pragma unroll
        for (uint32_t k = 0; k < T::kVec; ++k) {
            e[k] = __builtin_amdgcn_exp2f(e[k]);
            sum += e[k];
        }
        const uint32_t at = h.first(0, i);
        uint32_t mask = bits[at >> 5] >> (at & 31u) & ((1u << T::kVec) - 1);
        s += sum;
        if (__any(mask != 0)) {
            asm volatile("" : "+v"(mask));  // a branch, not a selection for every vector
            sum = 0.0f;
#pragma unroll
            for (uint32_t k = 0; k < T::kVec; ++k) sum += mask >> k & 1u ? 0.0f : e[k];
        }
        t += sum;
    }
    s = wave_sum(s);
    t = wave_sum(t);
    const float f = __builtin_amdgcn_exp2f(-x_of.shift(true));
    PairStat mine{x_of.m, s * f, x_of.m, t * f};
    if (t < s * 0x1p-64f) {
        // next to nothing beside the named places: from its own maximum.  The values
        // are read again: it is rare, and the registers it would need are not
        const auto each_other = [&](auto use) {
#pragma unroll 1
            for (uint32_t i = 0; i < kVecs<T>; ++i)
#pragma unroll 1
                for (uint32_t k = 0; k < T::kVec; ++k) {
                    const uint32_t j = h.first(0, i) + k;
                    if (part + j < g.vocab && !(bits[j >> 5] >> (j & 31u) & 1u))
                        use(T::load(z[part + j]));
                }
        };
        float most = kLowest, sum = 0.0f;
        each_other([&](float v) { most = fmaxf(most, v); });
        mine.other_m = wave_max(most);
        each_other([&](float v) {
            sum += __builtin_amdgcn_exp2f(scaled(v, mine.other_m, g.tau.two_over) * kLog2e);
        });
        mine.other_s = wave_sum(sum);
    }
    if ((threadIdx.x & 63u) == 0) wave_stat[threadIdx.x >> 6] = mine;
    __syncthreads();
    if (threadIdx.x == 0) g.stat[blockIdx.x] = join_waves(wave_stat, g.tau.two_over);
}

// One wave per row: the loss from the parts and the student's values at the
// named places, and what the gradient needs: m, 1/S (0: no gradient) and, with
// the tail, the maximum and the factor of the exponentials where no place is named,
// without it what scales the teacher's probabilities exp(lt - top) / sum.  They are
// taken relative to the largest, so that their sum to divide by is between 1 and
// `top` however little the teacher gives the named places.
template <class T>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillArgs g) {
    const uint64_t row = blockIdx.x;
    const uint32_t lane = threadIdx.x;
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    const PairStat first = lane < g.parts ? g.stat[row * g.parts + lane] : kNoPair;
    constexpr uint32_t kMost = DF11_MAX_TOP / 64;
    float lt[kMost], v[kMost], top = -INFINITY;
    double p[kMost], mass = 0.0;
    bool some = false, bad = false;
#pragma unroll
    for (uint32_t e = 0; e < kMost; ++e) {
        const uint32_t k = 64 * e + lane;
        const int64_t at = k < g.top ? g.index[row * g.top + k] : -1;
        lt[e] = k < g.top ? g.teacher[row * g.top + k] : 0.0f;
        some |= named(at);
        bad |= bad_entry(at, lt[e], g.vocab);
        if (!named(at)) lt[e] = -INFINITY;
        v[e] = named(at) && at < g.vocab ? T::load(z[at]) : 0.0f;
        top = fmaxf(top, lt[e]);
    }
    top = g.tail ? 0.0f : wave_max(top);
#pragma unroll
    for (uint32_t e = 0; e < kMost; ++e) {
        p[e] = lt[e] > -INFINITY ? exp(static_cast<double>(lt[e]) - top) : 0.0;
        mass += p[e];
    }
    some = __any(some);
    bad = __any(bad);
    mass = wave_sum(mass);
    const PairStat st = join_parts(first, g.stat + row * g.parts, g.parts, g.tau.two_over);
    // a row's few terms in 64 bits: the loss is a difference of larger ones
    const double ln_s = log(static_cast<double>(st.s));
    const double scale = g.tail ? 1.0 : 1.0 / mass, ln_mass = g.tail ? 0.0 : top + log(mass);
    double sum = 0.0;
#pragma unroll
    for (uint32_t e = 0; e < kMost; ++e)
        if (p[e] > 0.0)
            sum += p[e] * scale * (lt[e] - ln_mass - (scaled64(v[e], st.m, g.tau) - ln_s));
    sum = wave_sum(sum);
    if (lane) return;
    // what is left to the others, by the teacher and (its logarithm) by the student
    double r = fmax(0.0, 1.0 - mass);
    // 32-bit logarithms, each right to 2^-21 (1 + |lt|), leave sum p (1 + |lt|) 2^-21 of 1,
    // 2.8e-6 for 128 places: no probability where there is no place to have it
    if (st.other_s == 0.0f && r <= 0x1p-18) r = 0.0;
    const double ln_left = scaled64(st.other_m, st.m, g.tau) + log(double{st.other_s}) - ln_s;
    const float nan = __builtin_nanf("");
    float over_s = 1.0f / st.s;
    if (g.tail && r > 0.0) sum += r * (log(r) - ln_left);
    // q (1 - r/Q) of a place is exp((z - other_m) / tau) times this
    float other = st.other_s > 0.0f ? static_cast<float>((exp(ln_left) - r) / st.other_s) : 0.0f;
    float loss = static_cast<float>(sum);
    if (st.s == 0.0f) {
        over_s = 0.0f;
        loss = INFINITY;
    }
    if (!(st.s >= 0.0f) || st.s == INFINITY) loss = over_s = other = nan;
    if (!some || (!g.tail && mass == 0.0)) {
        loss = over_s = 0.0f;
    }
    if (bad) loss = over_s = other = nan;
    g.loss[row] = loss;
    *reinterpret_cast<float4 *>(g.stats + 4 * row) =
        float4{st.m, over_s, g.tail ? st.other_m : top,
               g.tail ? other : static_cast<float>(scale)};
}

// An exponential times its factor everywhere, then the few named places of the part
// once more, q minus the teacher's probability.  Their logits are read before the
// first store, so that the gradient may replace the logits.
template <class T>
__global__ __launch_bounds__(kThreads, 8) void distill_grad_kernel(DistillArgs g) {
    __shared__ uint32_t place[DF11_MAX_TOP], many;
    const uint64_t row = blockIdx.x / g.parts;
    const uint32_t part = (blockIdx.x % g.parts) * kPart;
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    auto *out = static_cast<typename T::raw *>(g.grad) + row * g.grad_stride;
    Held<T> h;
    h.load(z, part, g.vocab, g.once);
    const float4 st = *reinterpret_cast<const float4 *>(g.stats + 4 * row);
    const float m = st.x, over_s = st.y, other_m = g.tail ? st.z : m;
    const float top = g.tail ? 0.0f : st.z, scale = g.tail ? 1.0f : st.w;
    const float w = (g.weight ? g.weight[row] : 1.0f) * (0.5f * g.tau.two_over);
    const bool none = over_s == 0.0f;
    const float every = (g.tail ? st.w : over_s) * w;

    // a thread an entry; the places of this part go to LDS, so that an entry
    // sees whether its place is named again
    static_assert(DF11_MAX_TOP <= kThreads, "a thread an entry");
    if (threadIdx.x == 0) many = 0;
    __syncthreads();
    const int64_t at = threadIdx.x < g.top ? g.index[row * g.top + threadIdx.x] : -1;
    const bool mine = at >= part && at < min(int64_t{part} + kPart, int64_t{g.vocab});
    if (mine) place[atomicAdd(&many, 1u)] = static_cast<uint32_t>(at);
    __syncthreads();
    float value = 0.0f, target = 0.0f;
    if (mine) {
        value = T::load(z[at]);
        target = expf(g.teacher[row * g.top + threadIdx.x] - top);
        uint32_t same = 0;
        for (uint32_t k = 0; k < many; ++k) same += place[k] == at ? 1u : 0u;
        if (same > 1) {  // all its entries, in their order: each of them writes the same
            target = 0.0f;
            for (uint32_t k = 0; k < g.top; ++k)
                if (g.index[row * g.top + k] == at) target += expf(g.teacher[row * g.top + k] - top);
        }
    }
    __syncthreads();
    store_part(h, out, part, g.vocab, g.once, [&](float v, uint32_t) {
        const float x = exponent(v, other_m, g.tau);
        return none ? 0.0f : __builtin_amdgcn_exp2f(x) * every;
    });
    __syncthreads();
    if (mine && !none) {
        const float q = __builtin_amdgcn_exp2f(exponent(value, m, g.tau)) * over_s;
        out[at] = T::store((q - target * scale) * w);
    }
}

// ---- host side
constexpr uint64_t kMostParts = 1ull << 23;

uint32_t parts_of(uint32_t vocab) {
    return (vocab - 1) / kPart + 1;
}

int check_logits(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                 uint64_t stride) {
    if (dtype > DF11_F16 || vocab == 0 || vocab > 0x7FFFFFFFu) return DF11_E_INVALID_ARG;
    if (rows && rows * parts_of(vocab) / rows != parts_of(vocab)) return DF11_E_UNSUPPORTED;
    if (rows * parts_of(vocab) > kMostParts) return DF11_E_UNSUPPORTED;
    if (rows && (!logits || misaligned(logits, elem_bytes(dtype)))) return DF11_E_INVALID_ARG;
    if (rows > 1 && (stride < vocab || stride > (1ull << 40))) return DF11_E_INVALID_ARG;
    return DF11_OK;
}

int check_temperature(float t) {
    return t > 0.0f && std::isfinite(t) && std::isfinite(2.0f / t) ? DF11_OK : DF11_E_INVALID_ARG;
}

int check_grad(const void *logits, const void *grad, uint32_t dtype, uint64_t rows, uint32_t vocab,
               uint64_t stride, uint64_t grad_stride) {
    if (!rows) return DF11_OK;
    if (!grad || misaligned(grad, elem_bytes(dtype))) return DF11_E_INVALID_ARG;
    if (rows > 1 && (grad_stride < vocab || grad_stride > (1ull << 40))) return DF11_E_INVALID_ARG;
    // in place only as a whole: a part that is written must be the part that is read
    if (grad == logits && rows > 1 && grad_stride != stride) return DF11_E_INVALID_ARG;
    return DF11_OK;
}

int check_workspace(const void *ws, uint64_t have, uint64_t need) {
    if (have < need) return DF11_E_BUFFER_TOO_SMALL;
    return need && (!ws || misaligned(ws, 16)) ? DF11_E_INVALID_ARG : DF11_OK;
}

// Whether the logits pass the caches by: from 256 MB, what the memory-side cache
// holds, a gradient would not find there what the forward pass read.  4096 x
// 128,256 bf16, distillation with its gradient: 608 us through the caches, 560
// past them; 1023 x 32,001 (65 MB), log probabilities with theirs: 46.8 and 49.0.
bool streams(uint32_t dtype, uint64_t rows, uint32_t vocab) {
    return rows * vocab * elem_bytes(dtype) >= (256ull << 20);
}

// The workspace of `all` parts: their statistics, counts and candidates.
struct Space {
    uint64_t count, candidate, bytes;
};
Space logprob_space(uint64_t all, uint32_t top) {
    Space s{sizeof(PartStat) * all, 0, 0};
    s.candidate = s.count + (top ? (4 * all + 15) / 16 * 16 : 0);
    s.bytes = s.candidate + sizeof(uint2) * room_of(top) * all;
    return s;
}

#define DF11_BY_DTYPE(dtype, kernel, grid, block, stream, args)                            \
    do {                                                                                   \
        if ((dtype) == DF11_F32)                                                           \
            hipLaunchKernelGGL(kernel<F32>, dim3(grid), dim3(block), 0, stream, args);     \
        else if ((dtype) == DF11_BF16)                                                     \
            hipLaunchKernelGGL(kernel<BF16>, dim3(grid), dim3(block), 0, stream, args);    \
        else                                                                               \
            hipLaunchKernelGGL(kernel<F16>, dim3(grid), dim3(block), 0, stream, args);     \
    } while (0)

}  // namespace

extern "C" {

int df11_logprobs_workspace_bytes(uint32_t dtype, uint64_t rows, uint32_t vocab, uint32_t top,
                                  uint64_t *bytes) {
    if (!bytes || top > DF11_MAX_TOP || top > vocab) return DF11_E_INVALID_ARG;
    static const float some = 0.0f;
    const int rc = check_logits(&some, dtype, rows, vocab, vocab);
    if (rc) return rc;
    *bytes = logprob_space(rows * parts_of(vocab), top).bytes;
    return DF11_OK;
}

int df11_logprobs(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                  uint64_t row_stride, const int64_t *tokens, uint32_t top, float temperature,
                  float *logprob, int64_t *rank, float *entropy, float *top_logprob,
                  int64_t *top_index, float *stats, void *workspace, uint64_t workspace_bytes,
                  hipStream_t stream) {
    int rc = check_logits(logits, dtype, rows, vocab, row_stride);
    if (!rc) rc = check_temperature(temperature);
    if (rc) return rc;
    if (top > DF11_MAX_TOP || top > vocab) return DF11_E_INVALID_ARG;
    if (!rows) return DF11_OK;
    if (top ? !top_logprob || !top_index : false) return DF11_E_INVALID_ARG;
    if (!tokens && (logprob || rank)) return DF11_E_INVALID_ARG;
    if (misaligned(tokens, 8) || misaligned(rank, 8) || misaligned(top_index, 8) ||
        misaligned(logprob, 4) || misaligned(entropy, 4) || misaligned(top_logprob, 4) ||
        misaligned(stats, 16))
        return DF11_E_INVALID_ARG;
    const uint32_t parts = parts_of(vocab);
    const Space s = logprob_space(rows * parts, top);
    if ((rc = check_workspace(workspace, workspace_bytes, s.bytes))) return rc;
    char *ws = static_cast<char *>(workspace);
    LogprobArgs g{logits, tokens, reinterpret_cast<PartStat *>(ws),
                  reinterpret_cast<uint32_t *>(ws + s.count),
                  reinterpret_cast<uint2 *>(ws + s.candidate), logprob, entropy, top_logprob, stats,
                  rank, top_index, row_stride, vocab, parts, top, room_of(top), Tau(temperature),
                  top || streams(dtype, rows, vocab)};
    if (top)
        DF11_BY_DTYPE(dtype, logprob_top_kernel, rows * parts, kThreads, stream, g);
    else
        DF11_BY_DTYPE(dtype, logprob_part_kernel, rows * parts, kThreads, stream, g);
    if ((rc = launched())) return rc;
    DF11_BY_DTYPE(dtype, logprob_join_kernel, rows, kThreads, stream, g);
    return launched();
}

int df11_logprobs_backward(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                           uint64_t row_stride, const int64_t *tokens, const float *stats,
                           const float *grad_logprob, const float *grad_entropy,
                           float temperature, void *grad, uint64_t grad_stride,
                           hipStream_t stream) {
    int rc = check_logits(logits, dtype, rows, vocab, row_stride);
    if (!rc) rc = check_temperature(temperature);
    if (!rc) rc = check_grad(logits, grad, dtype, rows, vocab, row_stride, grad_stride);
    if (rc) return rc;
    if (!rows) return DF11_OK;
    if (!stats || (!grad_logprob && !grad_entropy) || (grad_logprob && !tokens))
        return DF11_E_INVALID_ARG;
    if (misaligned(tokens, 8) || misaligned(stats, 16) || misaligned(grad_logprob, 4) ||
        misaligned(grad_entropy, 4))
        return DF11_E_INVALID_ARG;
    LogprobGradArgs g{logits, grad, tokens, stats, grad_logprob, grad_entropy, row_stride,
                      grad_stride, vocab, parts_of(vocab), Tau(temperature),
                      streams(dtype, rows, vocab)};
    DF11_BY_DTYPE(dtype, logprob_grad_kernel, rows * g.parts, kThreads, stream, g);
    return launched();
}

int df11_distill_workspace_bytes(uint32_t dtype, uint64_t rows, uint32_t vocab, uint64_t *bytes) {
    if (!bytes) return DF11_E_INVALID_ARG;
    static const float some = 0.0f;
    const int rc = check_logits(&some, dtype, rows, vocab, vocab);
    if (rc) return rc;
    *bytes = sizeof(PairStat) * rows * parts_of(vocab);
    return DF11_OK;
}

int df11_distill(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                 uint64_t row_stride, const int64_t *teacher_index, const float *teacher_logprob,
                 uint32_t top, uint32_t tail, float temperature, const float *weight, float *loss,
                 float *stats, void *grad, uint64_t grad_stride, void *workspace,
                 uint64_t workspace_bytes, hipStream_t stream) {
    int rc = check_logits(logits, dtype, rows, vocab, row_stride);
    if (!rc) rc = check_temperature(temperature);
    if (!rc && grad) rc = check_grad(logits, grad, dtype, rows, vocab, row_stride, grad_stride);
    if (rc) return rc;
    if (top == 0 || top > DF11_MAX_TOP) return DF11_E_INVALID_ARG;
    if (!rows) return DF11_OK;
    if (!teacher_index || !teacher_logprob || !loss || !stats) return DF11_E_INVALID_ARG;
    if (misaligned(teacher_index, 8) || misaligned(teacher_logprob, 4) || misaligned(weight, 4) ||
        misaligned(loss, 4) || misaligned(stats, 16))
        return DF11_E_INVALID_ARG;
    const uint32_t parts = parts_of(vocab);
    rc = check_workspace(workspace, workspace_bytes, sizeof(PairStat) * rows * parts);
    if (rc) return rc;
    DistillArgs g{logits, grad, teacher_index, teacher_logprob, weight,
                  static_cast<PairStat *>(workspace), loss, stats, row_stride, grad_stride, vocab,
                  parts, top, tail, Tau(temperature), streams(dtype, rows, vocab)};
    DF11_BY_DTYPE(dtype, distill_part_kernel, rows * parts, kThreads, stream, g);
    if ((rc = launched())) return rc;
    DF11_BY_DTYPE(dtype, distill_join_kernel, rows, 64, stream, g);
    if ((rc = launched()) || !grad) return rc;
    DF11_BY_DTYPE(dtype, distill_grad_kernel, rows * parts, kThreads, stream, g);
    return launched();
}

int df11_distill_backward(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                          uint64_t row_stride, const int64_t *teacher_index,
                          const float *teacher_logprob, uint32_t top, uint32_t tail,
                          float temperature, const float *stats, const float *grad_loss,
                          void *grad, uint64_t grad_stride, hipStream_t stream) {
    int rc = check_logits(logits, dtype, rows, vocab, row_stride);
    if (!rc) rc = check_temperature(temperature);
    if (!rc) rc = check_grad(logits, grad, dtype, rows, vocab, row_stride, grad_stride);
    if (rc) return rc;
    if (top == 0 || top > DF11_MAX_TOP) return DF11_E_INVALID_ARG;
    if (!rows) return DF11_OK;
    if (!teacher_index || !teacher_logprob || !stats) return DF11_E_INVALID_ARG;
    if (misaligned(teacher_index, 8) || misaligned(teacher_logprob, 4) ||
        misaligned(grad_loss, 4) || misaligned(stats, 16))
        return DF11_E_INVALID_ARG;
    DistillArgs g{logits, grad, teacher_index, teacher_logprob, grad_loss, nullptr, nullptr,
                  const_cast<float *>(stats), row_stride, grad_stride, vocab, parts_of(vocab), top,
                  tail, Tau(temperature), streams(dtype, rows, vocab)};
    DF11_BY_DTYPE(dtype, distill_grad_kernel, rows * g.parts, kThreads, stream, g);
    return launched();
}

}  // extern "C"
