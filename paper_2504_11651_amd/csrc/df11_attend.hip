// Attention of a batch to a prefix that its sequences share and to their own
// tokens, over a paged cache.
//
// One pass over keys and values: scores s of 64 tokens at a time, p = 2^(c (s - m))
// with m a running bound of the row's s (c = scale log2 e), l += p, O += p v, and
// l and O taken down by 2^(c (m - m')) where the bound rises.  Parts of a row that
// different workgroups took are joined with 2^(c (m_i - m)).
//
// A tile is kRows rows of q (tokens x query heads that share a head of the cache)
// against 64 tokens.  S^T = K Q^T on v_mfma_f32_32x32x16: a lane then holds 16
// scores of ONE row of q, so that the softmax is in-lane but for one exchange with
// lane + 32, and P^T is the next product's operand where it lies: O^T = V^T P^T sums
// over the tokens in the order that the scores have in the registers, and V is read
// transposed from LDS (ds_read_tr16) in that same order.
//
// K and V go from memory to LDS without passing registers, a tile ahead of the
// products.  A direct load fills LDS in the lanes' order, so the rows cannot be
// padded; instead the 16-byte pieces of token t lie at piece ^ swizzle(t), which
// each lane takes into account in the address it loads from.
//
// Two workgroups of four waves a CU (66 KB of LDS and 256 registers a lane each).  Few
// rows are bound by memory: 31 sequences of up to 30,001 tokens, 1.7 GB of keys and
// values, take 292 us (5.9 TB/s); 8 rows behind 131,072 shared tokens 112 to 123 us.
// Many are bound by what a SIMD issues: a prompt of 8192 tokens, 32 heads over 8, runs at
// 950 to 1,010 TFLOP/s (by the card) with the matrix cores busy 47% of the time and the
// softmax' 139 vector operations a tile of 32 x 64 most of the rest (without its
// exponentials it would take 6% less, without any of its operations but the maximum 12%,
// without the reads of V from LDS 7%).

#include "df11_kv_common.h"

#include <algorithm>
#include <type_traits>

namespace {

using namespace df11ops;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kTile = 64;   // tokens of a tile
constexpr uint32_t kRows = 128;  // rows of a tile: 32 a wave
constexpr uint32_t kMaxParts = 256;  // of the prefix, and of a sequence's own tokens
// How far c s may rise above c m before O is taken down: what is summed in 32 bits loses
// nothing by it.
constexpr float kSlack = 8.0f;
// From c m of this size on p is taken from s - m, which is exact where it counts, by an
// operation more for each score (a prompt of 8192 tokens 549 -> 553 us).  Below, c m is off
// by half a step, 2^-15 at most, and so is the weight of all that was summed under one
// bound: a 23rd of fp16's half step.
constexpr float kLarge = 1024.0f;
constexpr float kMaxSlack = 1.0e38f;  // of s, whatever c is: -inf and it are -inf

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

template <class C>
struct Mat;
template <>
struct Mat<BF16> {
    static constexpr uint32_t kInf = 0x7F80;  // the least that is not finite, without sign
    static constexpr float kLift = 0.0f;      // p = 2^(c (s - m) + kLift)
    static __device__ acc16 product(s8 a, s8 b, acc16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a),
                                                       __builtin_bit_cast(b8, b), c, 0, 0, 0);
    }
};
template <>
struct Mat<F16> {
    static constexpr uint32_t kInf = 0x7C00;
    // p from 2^7 for the largest on, below 2^(7 + kSlack) = half the largest fp16.  Its
    // steps end at 2^-24, which is 2^-31 of the largest then: thousands of tokens far below
    // it still weigh what l counts of them.  (8192 tokens 15 powers of e below one: from 1
    // on 2.6% of their share was lost, at 17.5 powers all of it.)
    static constexpr float kLift = 7.0f;
    static __device__ acc16 product(s8 a, s8 b, acc16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a),
                                                      __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
};

struct AttendArgs {
    const uint16_t *q;
    const uint16_t *k, *v;
    uint16_t *out;
    float *lse;
    float *part_o;   // parts x tokens x heads x dim
    float2 *part_ml; // parts x tokens x heads: m, l
    uint64_t q_stride, out_stride, page_k, page_v;
    Batch batch;
    float c;      // scale log2 e
    float slack;  // kSlack / c
    uint32_t pages, page_shift, heads, kv_heads, group;
    uint32_t own_tiles, own_groups;  // `whole`: tile numbers; groups of them that share an XCD
    // `shares`: tiles of rows and of tokens of the prefix, most parts of a row's prefix and
    // of its own tokens, and for the join the share's size, where own tokens begin, their
    // units, and those in front of every sequence
    uint32_t row_tiles, front_tiles, front_parts, own_parts;
    uint32_t *sums;
};

// Tokens that a table row has pages for: what lies beyond is not read, and rows that
// see it have no result.
__device__ inline uint32_t room(const Batch &b, uint32_t page_shift) {
    return min(uint64_t{b.width} << page_shift, uint64_t{INT32_MAX});
}
// A sequence's rows, in tiles of kRows, and the tokens of its own that they see.
struct Sequence {
    uint32_t from, to;  // rows of the call
    int32_t before;     // a row r sees before + r
    __device__ uint32_t tiles(const AttendArgs &a) const {
        return to > from ? ((to - from) * a.group + kRows - 1) / kRows : 0;
    }
    __device__ uint32_t first_row(const AttendArgs &a, uint32_t i) const {
        return from * a.group + i * kRows;
    }
    __device__ uint32_t rows(const AttendArgs &a, uint32_t i) const {
        return min(kRows, to * a.group - first_row(a, i));
    }
    // what the first and the last row of a tile see
    __device__ int32_t least(const AttendArgs &a, uint32_t i) const {
        return before + static_cast<int32_t>(first_row(a, i) / a.group);
    }
    __device__ uint32_t end(const AttendArgs &a, uint32_t i) const {
        const uint32_t last = first_row(a, i) + rows(a, i) - 1;
        return min(static_cast<uint32_t>(max(before + static_cast<int32_t>(last / a.group), 0)),
                   room(a.batch, a.page_shift));
    }
    __device__ uint32_t token_tiles(const AttendArgs &a, uint32_t i) const {
        return (end(a, i) + kTile - 1) / kTile;
    }
};
__device__ inline Sequence sequence(const Batch &b, uint32_t s) {
    const uint32_t to = b.first(s + 1);
    return {b.first(s), to, max(b.length[s], 0) - static_cast<int32_t>(to) + 1};
}

// Four neighbouring tokens 64 bytes apart, which the transposed reads take at once, and
// each four 16 bytes further: no two lanes meet at a bank (counted: none; with the tokens
// 16 or 32 bytes apart a third to a half of LDS' cycles are conflicts).
template <uint32_t D>
__device__ inline uint32_t swizzle(uint32_t t) {
    return D == 64 ? (t & 2) * 2 | ((t >> 2) & 3) : (t & 3) * 4 | ((t >> 2) & 3);
}

typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void mem_void;
typedef __attribute__((address_space(3))) s4 lds_s4;

// What a workgroup has to attend to: tokens [begin, end) of one table.
struct Range {
    const int32_t *table;
    uint32_t width, begin, end;
};

// Where a wave reads and writes LDS: fixed for the kernel.
template <uint32_t D>
struct Places {
    static constexpr uint32_t kRowBytes = 2 * D;
    static constexpr uint32_t kSteps = D / 16;   // of K Q^T
    static constexpr uint32_t kBlocks = D / 32;  // of O
    uint32_t k[kSteps], v[kBlocks][2];
    // `first`: of the tile's tokens that the wave looks at
    __device__ Places(uint32_t lane, uint32_t first) {
        const uint32_t half = lane >> 5, t = lane & 31;
        for (uint32_t s = 0; s < kSteps; s++)
            k[s] = (first + t) * kRowBytes + (((2 * s + half) ^ swizzle<D>(t & 15)) << 4);
        // groups of 16 lanes read 4 tokens x 16 values: lane i the 8 bytes i % 4 of token i / 4
        const uint32_t i = lane & 15, tok = 4 * half + (i >> 2);
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; b++)
#pragma unroll
            for (uint32_t e = 0; e < 2; e++) {
                const uint32_t piece = 4 * b + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
                const uint32_t t = tok + 8 * e;
                v[b][e] = (first + t) * kRowBytes + ((piece ^ swizzle<D>(t)) << 4) + (i & 1) * 8;
            }
    }
};

template <class C, uint32_t D>
struct Worker {
    using P = Places<D>;
    static constexpr uint32_t kLoads = 2 * D / 64;     // 1 KB each: 16 tokens
    static constexpr uint32_t kEach = 16 / kLoads;     // tokens of one

    const AttendArgs &a;
    const P at;
    const uint32_t lane, wave, kvh;
    uint64_t head_off;
    uint32_t from[kLoads];  // a lane's bytes from its 16 tokens' first
    s8 q[P::kSteps];
    acc16 o[P::kBlocks];
    float m = -INFINITY, l = 0.0f;
    float base = 0.0f;   // c m - kLift where m is a number
    bool large = false;  // in some lane of the wave

    __device__ Worker(const AttendArgs &args, uint32_t thread, uint32_t kvh_, bool split)
        : a(args), at(thread & 63, split ? thread >> 1 & 32 : 0), lane(thread & 63),
          wave(__builtin_amdgcn_readfirstlane(thread >> 6)), kvh(kvh_) {
        head_off = (uint64_t{kvh} * D) << a.page_shift;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; i++) {
            constexpr uint32_t kLanes = 64 / kEach;  // of a token
            const uint32_t t = i * kEach + lane / kLanes;
            from[i] = t * 2 * D + (((lane % kLanes) ^ swizzle<D>(t)) << 4);
        }
#pragma unroll
        for (auto &x : o)
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) x[e] = 0.0f;
    }

    // The page numbers of a tile's tokens, asked for a tile ahead of its loads: lanes
    // 4 i + j have that of tokens 16 j.. (16 tokens lie on one page, also at the end).
    __device__ uint32_t pages(const Range &r, uint32_t tile) const {
        const uint32_t at = min(tile + 16 * (lane & 3), r.end - 1) >> a.page_shift;
        return at < r.width ? static_cast<uint32_t>(r.table[at]) : ~0u;
    }
    // Loads this wave's 16 tokens of a tile into LDS, past the registers.  Bit i: tokens
    // 16 i.. of the tile lie on no page of the cache; another's are loaded in their place.
    __device__ uint32_t load(const Range &r, uint32_t tile, uint32_t numbers, uint8_t *k,
                         uint8_t *v) const {
        uint32_t page = __builtin_amdgcn_readlane(numbers, wave);
        if (page >= a.pages) page = 0;
        const uint32_t t = min(tile + 16 * wave, (r.end - 1) & ~15u);  // behind: of no effect
        const uint64_t in = (uint64_t{t & ((1u << a.page_shift) - 1)} * D + head_off) * 2;
        const auto *kp = reinterpret_cast<const uint8_t *>(a.k + page * a.page_k) + in;
        const auto *vp = reinterpret_cast<const uint8_t *>(a.v + page * a.page_v) + in;
        k += 16 * wave * P::kRowBytes;
        v += 16 * wave * P::kRowBytes;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; i++) {
            // 32 bits beside a base in scalar registers; widened before the loop it would be
            // an addition of 64 bits a load
            uint32_t off = from[i];
            asm volatile("" : "+v"(off));
            __builtin_amdgcn_global_load_lds((mem_void *)(kp + off), (lds_void *)(k + i * 1024), 16,
                                             0, 0);
            __builtin_amdgcn_global_load_lds((mem_void *)(vp + off), (lds_void *)(v + i * 1024), 16,
                                             0, 0);
        }
        return __ballot(numbers >= a.pages) & 15;
    }
    __device__ static void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
    // Clears the values of this wave's tokens behind the range: they meet a p of 0, and
    // what memory holds there may be an infinity.
    __device__ void clear(const Range &r, uint32_t tile, uint8_t *v) const {
#pragma nounroll
        for (uint32_t i = 0; i < kLoads; i++) {
            constexpr uint32_t kLanes = 64 / kEach;
            if (tile + 16 * wave + i * kEach + lane / kLanes >= r.end)
                *reinterpret_cast<uint4 *>(v + 16 * wave * P::kRowBytes + i * 1024 + lane * 16) =
                    uint4{0, 0, 0, 0};
        }
    }

    __device__ static s8 read_v(const uint8_t *v, uint32_t lo, uint32_t hi) {
        const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(v + lo));
        const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)(v + hi));
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }

    // Scores of tokens `first` .. first + 32 kCount of a tile.
    template <uint32_t kCount>
    __device__ void scores(const uint8_t *k, acc16 (&s)[kCount]) const {
#pragma unroll
        for (uint32_t b = 0; b < kCount; b++)
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) s[b][e] = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < P::kSteps; i++)
#pragma unroll
            for (uint32_t b = 0; b < kCount; b++)
                s[b] = Mat<C>::product(
                    *reinterpret_cast<const s8 *>(k + at.k[i] + b * 32 * P::kRowBytes), q[i], s[b]);
    }
    // The softmax' step: p of them, in the order in which they meet the values.  l sums
    // them in 32 bits; the matrix cores take them in the cache's type.  That rounding, half
    // a step of each p to either side, and the result's own are the only ones to fewer bits
    // (relative error of a result 0.0022 against 0.0017 for the result's rounding alone, in
    // BF16); P in two terms would take a second product with V for each.
    template <uint32_t kCount>
    __device__ void weigh(acc16 (&s)[kCount], s8 (&p)[2 * kCount]) {
        float top = s[0][0];
#pragma unroll
        for (uint32_t b = 0; b < kCount; b++)
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) top = fmaxf(top, s[b][e]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top),
                                                           __float_as_uint(top), false, false);
        top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
        if (__builtin_expect(__any(top > m + a.slack), 0)) {
            const float rise = fmaxf(m, top), at = rise == -INFINITY ? 0.0f : rise;
            const float down = __builtin_amdgcn_exp2f((m - at) * a.c);
            m = rise;
            base = fmaf(at, a.c, -Mat<C>::kLift);
            large = __any(fabsf(base) >= kLarge);
            l *= down;
#pragma unroll
            for (auto &x : o)
#pragma unroll
                for (uint32_t e = 0; e < 16; e++) x[e] *= down;
        }
        float shift = base;
        if (__builtin_expect(large, 0)) {
            const float at = m == -INFINITY ? 0.0f : m;
            shift = -Mat<C>::kLift;
#pragma unroll
            for (uint32_t b = 0; b < kCount; b++)
#pragma unroll
                for (uint32_t e = 0; e < 16; e++) s[b][e] -= at;
        }
#pragma unroll
        for (uint32_t b = 0; b < kCount; b++)
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[b][e], a.c, -shift));
                l += x;
                p[2 * b + e / 8][e % 8] = static_cast<short>(C::store(x));
            }
    }

    // Tokens of a tile that every row sees.
    template <uint32_t kCount>
    __device__ void tokens(const uint8_t *k, const uint8_t *v) {
        acc16 s[kCount];
        s8 p[2 * kCount];
        // (in front of the wave of the other workgroup, which is at its softmax then: 558 ->
        // 545 us for a prompt of 8192 tokens)
        __builtin_amdgcn_s_setprio(1);
        scores<kCount>(k, s);
        __builtin_amdgcn_s_setprio(0);
        weigh<kCount>(s, p);
        products<kCount>(v, p);
    }

    // 32 tokens of which the lane's row sees the first `seen`; bit i of `lost`: tokens 16 i..
    // are of no page of the cache.  A value that is an infinity or a NaN must not meet the
    // p of 0 of a row that does not see it: those are left out, and true comes back if there
    // are any.
    __device__ bool tokens_of_some(const uint8_t *k, const uint8_t *v, int32_t seen,
                                   uint32_t lost) {
        acc16 s[1];
        s8 p[2];
        scores<1>(k, s);
        seen -= 4 * static_cast<int32_t>(lane >> 5);
#pragma unroll
        for (uint32_t e = 0; e < 16; e++) {
            const int32_t t = 8 * (e / 4) + e % 4;
            s[0][e] = t >= seen ? -INFINITY : lost >> (e / 8) & 1 ? NAN : s[0][e];
        }
        weigh<1>(s, p);
        u4 bad = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t i = 0; i < 2; i++)
#pragma unroll
            for (uint32_t b = 0; b < P::kBlocks; b++) {
                const s8 x = read_v(v + i * 16 * P::kRowBytes, at.v[b][0], at.v[b][1]);
                const u4 out = not_finite(x);
                bad |= out;
                // 0 for 1, all bits for 0
                const us8 keep = __builtin_bit_cast(us8, out) - static_cast<unsigned short>(1);
                o[b] = Mat<C>::product(x & __builtin_bit_cast(s8, keep), p[i], o[b]);
            }
        return __any((bad[0] | bad[1] | bad[2] | bad[3]) != 0);
    }

    // Of each half of a word: 1 if it holds an infinity or a NaN.
    typedef unsigned short us8 __attribute__((ext_vector_type(8)));
    __device__ static u4 not_finite(s8 x) {
        const us8 t = __builtin_bit_cast(us8, x) & static_cast<unsigned short>(0x7FFF);
        constexpr unsigned short kCarry = 0x8000 - Mat<C>::kInf;
        return __builtin_bit_cast(u4, (t + kCarry) >> 15);
    }
    template <uint32_t kCount>
    __device__ void products(const uint8_t *v, const s8 (&p)[2 * kCount]) {
#pragma unroll
        for (uint32_t i = 0; i < 2 * kCount; i++)
#pragma unroll
            for (uint32_t b = 0; b < P::kBlocks; b++)
                o[b] = Mat<C>::product(
                    read_v(v + i * 16 * P::kRowBytes, at.v[b][0], at.v[b][1]), p[i], o[b]);
    }
};

// Adds to x the infinities and NaN among eight values of the tokens [from, to) of a
// range: what tokens_of_some left out.
template <class C, uint32_t D>
__device__ void add_left_out(const AttendArgs &a, const Range &r, uint32_t from, uint32_t to,
                             uint32_t kvh, uint32_t piece, float (&x)[8]) {
    for (uint32_t t = from; t < to; t++) {
        const uint32_t i = t >> a.page_shift;
        if (i >= r.width) return;  // the row has no result
        const uint32_t page = r.table[i];
        if (page >= a.pages) return;
        const uint64_t in =
            (uint64_t{kvh * D} << a.page_shift) + (t & ((1u << a.page_shift) - 1)) * D;
        const uint4 y = load16(a.v + page * a.page_v + in + 8 * piece);
        for (uint32_t e = 0; e < 8; e++) {
            const float z = C::get(y, e);
            if (!(fabsf(z) < INFINITY)) x[e] += z;
        }
    }
}

// A tile of rows against a part of the prefix or of own tokens, or both after one
// another.  `places`: own tokens that the first row sees.
template <class C, uint32_t D, bool kWhole>
__device__ __forceinline__ void attend(const AttendArgs &a, uint32_t kvh, uint32_t row0,
                                       uint32_t rows, uint32_t part, const Range &front,
                                       const Range &own, int32_t places, uint8_t *k0, uint8_t *v0,
                                       uint8_t *k1, uint8_t *v1, float2 *stats,
                                       uint32_t *left_out) {
    using W = Worker<C, D>;
    using P = Places<D>;
    // up to 64 rows: waves 2 i and 2 i + 1 take rows 32 i.. and share the tokens of a tile
    const bool split = rows <= 64;
    // (its places are made anew for each tile of rows: kept over a loop around this they
    // are spilled, and a spilled register is a round trip to memory)
    uint32_t thread = threadIdx.x;
    asm volatile("" : "+v"(thread));
    W w(a, thread, kvh, split);
    const uint32_t half = w.lane >> 5, n = w.lane & 31;
    const uint32_t mine = 32 * (split ? w.wave >> 1 : w.wave);
    const bool busy = mine < rows;
    const uint32_t row = row0 + min(mine + n, rows - 1);
    const uint32_t token = row / a.group;
    const uint32_t head = kvh * a.group + row % a.group;
    const int32_t later = static_cast<int32_t>(token - row0 / a.group);
    if (busy) {
        const uint16_t *p = a.q + token * a.q_stride + uint64_t{head} * D + 8 * half;
#pragma unroll
        for (uint32_t i = 0; i < P::kSteps; i++)
            w.q[i] = __builtin_bit_cast(s8, load16(p + 16 * i));
    }
    bool lost = false;  // a page outside the cache, among tokens that all rows see
    for (uint32_t i = 0; i < 2; i++) {
        const Range r = i ? own : front;
        if (r.begin >= r.end) continue;
        // what every row sees, and the lane's row
        const int32_t end = static_cast<int32_t>(r.end);
        const uint32_t least = i ? max(min(places, end), 0) : end;
        const int32_t sees = i ? min(places + later, end) : end;
        const uint32_t plain = least & ~(kTile - 1);  // tiles before it: no row is masked
        // (page numbers behind the last tile: its own once more)
        uint32_t none = w.load(r, r.begin, w.pages(r, r.begin), k0, v0);
        bool odd = false;
        uint32_t next = w.pages(r, r.begin + kTile), t = r.begin;
        w.landed();
        __syncthreads();
        // One tile is looked at while the next one is loaded.  (A loop for each kind of wave:
        // where they meet in one, O is copied around in every turn.)
        const auto loop = [&](auto count) {
            constexpr uint32_t kCount = decltype(count)::value;
            const auto step = [&](uint8_t *k, uint8_t *v, uint8_t *to_k, uint8_t *to_v) {
                lost = lost || none;
                const bool more = t + kTile < r.end;
                if (more) none = w.load(r, t + kTile, next, to_k, to_v);
                next = w.pages(r, t + 2 * kTile);
                if constexpr (kCount) w.template tokens<kCount>(k, v);
                t += kTile;
                odd = !odd;
                w.landed();
                __syncthreads();
            };
            while (t < plain) {
                step(k0, v0, k1, v1);
                if (t >= plain) break;
                step(k1, v1, k0, v0);
            }
        };
        if (!busy)
            loop(std::integral_constant<uint32_t, 0>{});
        else if (split)
            loop(std::integral_constant<uint32_t, 1>{});
        else
            loop(std::integral_constant<uint32_t, 2>{});
        while (t < r.end) {
            uint8_t *k = odd ? k1 : k0, *v = odd ? v1 : v0;
            if (t + kTile > r.end) {
                w.clear(r, t, v);
                __syncthreads();
            }
            if (busy) {
                const uint32_t first = split ? w.wave & 1 : 0;
#pragma nounroll
                for (uint32_t j = 0; j < (split ? 1 : 2); j++)
                    if (w.tokens_of_some(k + 32 * j * P::kRowBytes, v + 32 * j * P::kRowBytes,
                                         sees - static_cast<int32_t>(t + 32 * (first + j)),
                                         none >> 2 * (first + j)))
                        *left_out = 1;
            }
            t += kTile;
            __syncthreads();
            if (t >= r.end) break;
            none = w.load(r, t, next, k0, v0);
            next = w.pages(r, t + kTile);
            w.landed();
            __syncthreads();
            odd = false;
        }
    }
    // Rows through LDS: a wave's 32 x D floats in a buffer, 16-byte pieces of row n at
    // piece ^ n.  Waves that shared tokens bring theirs to the larger bound first.
    float l = w.l + __shfl_xor(w.l, 32), m = w.m;
    if (lost || (kWhole && places + later > static_cast<int32_t>(room(a.batch, a.page_shift))))
        l = NAN;  // (of a share's rows the join knows: a row may have no share of own tokens)
    float *slice =
        reinterpret_cast<float *>(w.wave == 0 ? k0 : w.wave == 1 ? v0 : w.wave == 2 ? k1 : v1);
    if (split) {
        if (half == 0) stats[w.wave * 32 + n] = float2{m, l};
        __syncthreads();
        const float2 other = stats[(w.wave ^ 1) * 32 + n];
        const float both = fmaxf(m, other.x), base = both == -INFINITY ? 0.0f : both;
        const float down = __builtin_amdgcn_exp2f((m - base) * a.c);
        l = l * down + other.y * __builtin_amdgcn_exp2f((other.x - base) * a.c);
        m = both;
#pragma unroll
        for (auto &x : w.o)
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) x[e] *= down;
        __syncthreads();
    }
    if (half == 0) stats[w.wave * 32 + n] = float2{m, l};
#pragma unroll
    for (uint32_t b = 0; b < P::kBlocks; b++)
#pragma unroll
        for (uint32_t e = 0; e < 4; e++) {
            const uint32_t piece = 8 * b + 2 * e + half;
            *reinterpret_cast<float4 *>(slice + n * D + ((piece ^ (n & (D / 4 - 1))) << 2)) =
                float4{w.o[b][4 * e], w.o[b][4 * e + 1], w.o[b][4 * e + 2], w.o[b][4 * e + 3]};
        }
    __syncthreads();
    constexpr uint32_t kPieces = D / 8;  // of a row: 8 values each
#pragma nounroll
    for (uint32_t i = thread; i < rows * kPieces; i += kThreads) {
        const uint32_t r = i / kPieces, piece = i % kPieces;
        const uint32_t src = split ? 2 * (r / 32) : r / 32, nn = r % 32;
        const float2 ml = stats[src * 32 + nn];
        float x[8] = {};
#pragma nounroll
        for (uint32_t from = src; from < src + (split ? 2 : 1); from++) {
            const float *p = reinterpret_cast<const float *>(
                                 from == 0 ? k0 : from == 1 ? v0 : from == 2 ? k1 : v1) + nn * D;
#pragma unroll
            for (uint32_t e = 0; e < 2; e++) {
                const float4 y = *reinterpret_cast<const float4 *>(
                    p + (((2 * piece + e) ^ (nn & (D / 4 - 1))) << 2));
                x[4 * e] += y.x, x[4 * e + 1] += y.y, x[4 * e + 2] += y.z, x[4 * e + 3] += y.w;
            }
        }
        const uint32_t at = row0 + r, tok = at / a.group, hd = kvh * a.group + at % a.group;
        if (*left_out) {
            // the tiles that not all rows see to their end
            const int32_t sees = places + static_cast<int32_t>(tok - row0 / a.group);
            for (uint32_t j = 0; j < 2; j++) {
                const Range y = j ? own : front;
                const uint32_t least = j ? max(places, 0) : y.end;
                if (y.begin < y.end)
                    add_left_out<C, D>(a, y, max(y.begin, least & ~(kTile - 1)),
                                       j ? min(y.end, static_cast<uint32_t>(max(sees, 0))) : y.end,
                                       kvh, piece, x);
            }
        }
        if constexpr (kWhole) {
            const float inv = ml.y == 0.0f ? 0.0f : 1.0f / ml.y;
            uint32_t word[4];
#pragma unroll
            for (uint32_t e = 0; e < 4; e++)
                word[e] = C::store(x[2 * e] * inv) |
                          static_cast<uint32_t>(C::store(x[2 * e + 1] * inv)) << 16;
            store16(a.out + tok * a.out_stride + uint64_t{hd} * D + 8 * piece,
                    uint4{word[0], word[1], word[2], word[3]});
            if (a.lse && piece == 0)
                a.lse[uint64_t{tok} * a.heads + hd] =
                    ml.y == 0.0f ? -INFINITY
                                 : fmaf(ml.x, a.c, log2f(ml.y) - Mat<C>::kLift) * kLn2;
        } else {
            const uint64_t slot = (uint64_t{part} * a.batch.rows + tok) * a.heads + hd;
            float *p = a.part_o + slot * D + 8 * piece;
            *reinterpret_cast<float4 *>(p) = float4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<float4 *>(p + 4) = float4{x[4], x[5], x[6], x[7]};
            if (piece == 0) a.part_ml[slot] = ml;
        }
    }
}

#define DF11_ATTEND_LDS                                                                       \
    constexpr uint32_t kBytes = kTile * 2 * D;                                                \
    __shared__ __attribute__((aligned(1024))) uint8_t k0[kBytes], v0[kBytes], k1[kBytes],     \
        v1[kBytes];                                                                           \
    __shared__ float2 stats[4 * 32];                                                          \
    __shared__ uint32_t left_out

// A workgroup reads the prefix and all own tokens of a tile of a sequence's rows.
template <class C, uint32_t D>
__global__ __launch_bounds__(kThreads, 2) void attend_whole_kernel(AttendArgs a) {
    DF11_ATTEND_LDS;
    const Batch &b = a.batch;
    // tile numbers ascend over the sequences, and the last, which see the most, come first;
    // an XCD takes whole heads or every own_groups-th tile of one, so that its L2 holds
    // their keys and values
    const uint32_t x = blockIdx.x & 7, z = blockIdx.x >> 3;
    const uint32_t per = (a.own_tiles + a.own_groups - 1) / a.own_groups;
    const uint32_t combo = z / per * 8 + x, kvh = combo / a.own_groups;
    const uint32_t number = z % per * a.own_groups + combo % a.own_groups;
    if (kvh >= a.kv_heads || number >= a.own_tiles) return;
    const uint32_t id = a.own_tiles - 1 - number;
    // sequence s has the numbers from (its first row) / kRows + s on: never fewer than its
    // tiles
    const auto base = [&](uint32_t s) { return b.first(s) * a.group / kRows + s; };
    const uint32_t s = __builtin_amdgcn_readfirstlane(wave_search(b.sequences, id, base));
    if (s == ~0u) return;
    const Sequence q = sequence(b, s);
    const uint32_t i = id - base(s);
    if (i >= q.tiles(a)) return;
    if (threadIdx.x == 0) left_out = 0;  // (barriers follow before it is set or read)
    const Range front{b.prefix_table, b.prefix_pages, 0, b.prefix_len};
    const Range own{b.table + s * b.table_stride, b.width, 0, q.end(a, i)};
    const uint32_t row0 = q.first_row(a, i), rows = q.rows(a, i);
    attend<C, D, true>(a, kvh, row0, rows, 0, front, own, q.least(a, i), k0, v0, k1, v1, stats,
                       &left_out);
}

// All the work in a row, cut into equal shares: the prefix' tokens for each head and tile
// of rows, then every sequence's own tokens for each head and tile of its rows.  The unit
// is a tile of kTile tokens; kStart units before an item's tiles stand for what it costs to
// begin and end one: loads after one another, and code that is run once.  (Units of 2, 4 and
// 6: 16 rows behind 4,099 shared tokens 24.7, 22.2 and 22.4 us, 64 behind 32,768 109, 108
// and 112.)
constexpr uint32_t kStart = 4;
__device__ inline uint32_t cost(uint32_t tiles) { return tiles ? kStart + tiles : 0; }
__device__ inline uint32_t pieces(uint32_t n, uint32_t of) { return (n + of - 1) / of; }
// Where a few tiles of rows read the prefix, a share of it is taken by as many workgroups,
// one for each tile, on one XCD: its L2 reads the keys and values once for all.  (Behind
// 32,768 shared tokens: two tiles of 128 rows 533 -> 399 MB from memory and 84 -> 81 us, 8 tiles
// 208 -> 203, 16 379 -> 373; 32 and 64 tiles are bound by their products, and no faster.)
constexpr uint32_t kMaxTogether = 16;
__host__ __device__ inline uint32_t together(uint32_t row_tiles) {
    return row_tiles <= kMaxTogether ? row_tiles : 1;
}
struct Shares {
    uint32_t size;         // units of a share
    uint32_t front;        // units of the prefix for `copies` tiles of rows
    uint32_t copies, runs; // shares of the prefix: of `runs` each is there `copies` times
    uint32_t own_at, own;  // own tokens: where they begin, units for a head
};
// The prefix' place in the row for a head and tile of rows.
__device__ inline uint32_t front_at(const AttendArgs &a, uint32_t kvh, uint32_t tile) {
    const uint32_t tiles = together(a.row_tiles) == a.row_tiles ? 1 : a.row_tiles;
    return (kvh * tiles + (tiles == 1 ? 0 : tile)) * cost(a.front_tiles);
}

// 64 sequences, one a lane: their rows, units, and the units of all sequences before.
struct Lane {
    Sequence q;
    uint32_t units, before, most;  // most: tiles of the row that sees the most
};
__device__ inline Lane lane_of(const AttendArgs &a, uint32_t s0) {
    const uint32_t s = s0 + (threadIdx.x & 63);
    Lane y{};
    if (s < a.batch.sequences) {
        y.q = sequence(a.batch, s);
        for (uint32_t i = 0; i < y.q.tiles(a); i++) {
            y.most = y.q.token_tiles(a, i);  // later rows see more
            y.units += cost(y.most);
        }
    }
    return y;
}
// Calls f(first sequence, Lane) for 64 sequences after the other until it returns true.
// All units, where it never does.
template <class F>
__device__ inline uint64_t each_64(const AttendArgs &a, F f) {
    uint64_t all = 0;
    for (uint32_t s0 = 0; s0 < a.batch.sequences; s0 += 64) {
        Lane y = lane_of(a, s0);
        uint32_t sum = y.units;  // of the lanes up to this one
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xF, 0xF, false);  // row_shr 1
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xF, 0xF, false);
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xF, 0xF, false);
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xF, 0xF, false);
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x142, 0xA, 0xF, false);  // row_bcast 15
        sum += __builtin_amdgcn_update_dpp(0, sum, 0x143, 0xC, 0xF, false);  // row_bcast 31
        y.before = static_cast<uint32_t>(all) + sum - y.units;
        if (f(s0, y)) break;
        all += __builtin_amdgcn_readlane(sum, 63);
    }
    return all;
}
// The lane's sequence that holds unit `to` of all, in every lane.
struct Found {
    uint32_t s, unit;
    Sequence q;
};
__device__ inline bool find(uint32_t s0, const Lane &y, uint32_t to, Found *found) {
    const uint64_t here = __ballot(y.before <= to && to < y.before + y.units);
    if (!here) return false;
    const uint32_t at = __builtin_ctzll(here);
    found->s = s0 + at;
    found->unit = to - __builtin_amdgcn_readlane(y.before, at);
    found->q.from = __builtin_amdgcn_readlane(y.q.from, at);
    found->q.to = __builtin_amdgcn_readlane(y.q.to, at);
    found->q.before = __builtin_amdgcn_readlane(y.q.before, at);
    return true;
}

// A workgroup takes one share.  It holds as many tiles as any other whatever the
// sequences' lengths are; a row's parts are the shares that its tiles lie in.
template <class C, uint32_t D>
__global__ __launch_bounds__(kThreads, 2) void attend_shares_kernel(AttendArgs a) {
    DF11_ATTEND_LDS;
    const Batch &b = a.batch;
    const uint32_t lane = threadIdx.x & 63;
    // the units of all sequences, and the most tiles of a row
    Shares w{};
    w.copies = together(a.row_tiles);
    w.front = a.kv_heads * (a.row_tiles / w.copies) * cost(a.front_tiles);
    uint32_t most = 0;
    Lane y{};  // of up to 64 sequences: all of them
    const uint64_t own_units = each_64(a, [&](uint32_t s0, const Lane &z) {
        y = z;
        most = max(most, z.most);
        if (blockIdx.x == 0 && threadIdx.x < 64 && s0 + lane < b.sequences)
            a.sums[3 + s0 + lane] = z.before;
        return false;
    });
    most = wave_max(most);
    // (more than 31 bits only where the sequences' starts do not ascend: no result)
    w.own = (w.front * w.copies + a.kv_heads * own_units) >> 31 ? 0 : own_units;
    // no row has more parts than there is room for, and no more shares are than workgroups
    w.size = pieces(w.front * w.copies + a.kv_heads * w.own,
                    gridDim.x - (w.copies > 1 ? w.copies + 1 : 0));
    if (a.front_parts > 1) w.size = max(w.size, pieces(a.front_tiles - 1, a.front_parts - 1));
    if (a.own_parts > 1) w.size = max(w.size, pieces(most - min(most, 1u), a.own_parts - 1));
    w.size = max(w.size, 1u);
    w.runs = pieces(w.front, w.size);
    // (one copy: a share may have the prefix' last units and the first of own tokens)
    w.own_at = w.copies > 1 ? w.runs * w.copies * w.size : w.front;
    if (blockIdx.x == 0 && threadIdx.x == 0)
        a.sums[0] = w.size, a.sums[1] = w.own_at, a.sums[2] = w.own;
    // A CU has the workgroups i and i + 256: one takes its share from the front of the row
    // (the prefix, which the matrix cores bound), the other from its end (own tokens, which
    // memory bounds).
    const uint32_t half = gridDim.x / 2;
    const uint32_t share = blockIdx.x < half ? blockIdx.x : gridDim.x - 1 - (blockIdx.x - half);
    uint32_t at = share * w.size, end = min(at + w.size, w.own_at + a.kv_heads * w.own);
    uint32_t run = share, copy = 0;
    if (w.copies > 1 && share < w.runs * w.copies) {
        // eight runs' copies after one another: the copies of a run are eight apart, on the
        // same XCD
        const uint32_t eight = share / (8 * w.copies), n = min(8u, w.runs - 8 * eight);
        const uint32_t in = share - 8 * eight * w.copies;
        run = 8 * eight + in % n;
        copy = in / n;
        at = run * w.size;
        end = min(at + w.size, w.front);
    }
    if (at >= end) return;
    uint32_t s = ~0u, i = 0, own_unit = 0, kvh = 0;  // own tokens: where `at` is
    Sequence q{};
    // own tokens from unit `to` of a head's on
    const auto go = [&](uint32_t to, bool known) {
        Found found{~0u, 0, {}};
        if (known)
            find(0, y, to, &found);
        else
            each_64(a, [&](uint32_t s0, const Lane &z) { return find(s0, z, to, &found); });
        s = __builtin_amdgcn_readfirstlane(found.s);
        q = found.q;
        own_unit = found.unit;
        for (i = 0; s != ~0u && own_unit >= cost(q.token_tiles(a, i)); i++)
            own_unit -= cost(q.token_tiles(a, i));
    };
    // (known before the first tile of rows: not kept beyond it)
    if (end > w.own_at && b.sequences <= 64) {
        const uint32_t from = max(at, w.own_at) - w.own_at;
        kvh = from / w.own;
        go(from % w.own, true);
    }
    while (at < end) {
        uint32_t row0, rows, part, head, n, tiles, unit;
        int32_t least = INT32_MIN / 2;  // own tokens that the first row sees: none
        Range front{}, own{};
        if (at < w.front) {
            tiles = a.front_tiles;
            const uint32_t item = at / cost(tiles), of_head = a.row_tiles / w.copies;
            unit = at % cost(tiles);
            head = item / of_head;
            row0 = (item % of_head + copy) * kRows;
            const uint32_t all = b.first(b.sequences) * a.group;
            rows = row0 < all ? min(kRows, all - row0) : 0;
        } else {
            if (s == ~0u) {
                kvh = (at - w.own_at) / w.own;
                go((at - w.own_at) % w.own, false);
                if (s == ~0u) return;
            }
            unit = own_unit;
            tiles = q.token_tiles(a, i);
            head = kvh;
            row0 = q.first_row(a, i);
            rows = q.rows(a, i);
            least = q.least(a, i);
        }
        n = min(cost(tiles) - unit, end - at);
        const uint32_t first = max(unit, kStart) - kStart, last = max(unit + n, kStart) - kStart;
        part = (at < w.front ? run : share) - (at - unit + kStart) / w.size;
        if (at < w.front) {
            front = {b.prefix_table, b.prefix_pages, first * kTile,
                     min(b.prefix_len, last * kTile)};
        } else {
            part += a.front_parts;
            own = {b.table + s * b.table_stride, b.width, first * kTile,
                   min(q.end(a, i), last * kTile)};
        }
        if (first == last) rows = 0;
        if (rows) {
            __syncthreads();  // LDS is read
            if (threadIdx.x == 0) left_out = 0;
            attend<C, D, false>(a, head, row0, rows, part, front, own, least, k0, v0, k1, v1,
                                stats, &left_out);
        }
        at += n;
        if (at <= w.own_at || at >= end) continue;
        // on to the next tile of rows that sees something
        own_unit = 0;
        do i++;
        while (i < q.tiles(a) && !q.token_tiles(a, i));
        if (i < q.tiles(a)) continue;
        i = 0;
        for (uint32_t from = s + 1;; from += 64) {
            if (from >= b.sequences) from = 0, kvh++;
            const uint32_t next = from + lane;
            bool some = false;
            if (next < b.sequences) {
                const Sequence y = sequence(b, next);
                some = y.tiles(a) && y.token_tiles(a, y.tiles(a) - 1);
            }
            if (const uint64_t here = __ballot(some)) {
                s = __builtin_amdgcn_readfirstlane(from + __builtin_ctzll(here));
                break;
            }
        }
        q = sequence(b, s);
        while (!q.token_tiles(a, i)) i++;
    }
}

// A row's sequence, and the parts of the prefix and of own tokens that a head of it has:
// those of the prefix are 0.., of own tokens front_parts...  past: it sees places past the
// table's width, whose tokens are in no part.
struct Parts {
    uint32_t front, own;
    bool past;
};
__device__ inline bool parts_of(const AttendArgs &a, uint32_t token, uint32_t head, Parts *p) {
    const uint32_t kvh = head / a.group, row = token * a.group + head % a.group;
    const uint32_t size = a.sums[0], own_at = a.sums[1], all = a.sums[2];
    uint32_t before;
    Sequence q;
    if (a.batch.sequences <= 64) {
        // one round of loads for all that is asked
        const uint32_t lane = threadIdx.x & 63, s = min(lane, a.batch.sequences - 1);
        const Sequence y = sequence(a.batch, s);
        const uint32_t sum = a.sums[3 + s];
        const uint64_t here = __ballot(lane == s && y.from <= token && token < y.to);
        if (!here) return false;
        const uint32_t at = __builtin_ctzll(here);
        q.from = __builtin_amdgcn_readlane(y.from, at);
        q.to = __builtin_amdgcn_readlane(y.to, at);
        q.before = __builtin_amdgcn_readlane(y.before, at);
        before = __builtin_amdgcn_readlane(sum, at);
    } else {
        const Owner o = owner(a.batch, token);
        if (o.s == ~0u) return false;
        q = sequence(a.batch, o.s);
        before = a.sums[3 + o.s];
    }
    *p = {0, 0,
          q.before + static_cast<int32_t>(token) >
              static_cast<int32_t>(room(a.batch, a.page_shift))};
    if (a.front_tiles) {
        const uint32_t at = front_at(a, kvh, row / kRows) + kStart;
        p->front = min((at + a.front_tiles - 1) / size - at / size + 1, a.front_parts);
    }
    const uint32_t i = (row - q.from * a.group) / kRows, n = q.token_tiles(a, i);
    if (n) {
        uint32_t at = own_at + kvh * all + before + kStart;
        for (uint32_t j = 0; j < i; j++) at += cost(q.token_tiles(a, j));
        p->own = min((at + n - 1) / size - at / size + 1, a.own_parts);
    }
    return true;
}

// Joins the parts of a row and head: kWaves waves for each, several parts at a time.
template <class C, uint32_t D, uint32_t kWaves>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a) {
    constexpr uint32_t kLanes = D / 4, kAtOnce = 64 / kLanes;  // lanes of a part
    __shared__ float2 stats[4 / kWaves][2 * kMaxParts];
    __shared__ float weights[4 / kWaves][2 * kMaxParts];
    __shared__ float4 sums[4][kLanes];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, mine = wave / kWaves;
    const uint32_t at = __builtin_amdgcn_readfirstlane(blockIdx.x * (4 / kWaves) + mine);
    const uint32_t token = at / a.heads, head = at % a.heads;
    Parts n;
    if (token >= a.batch.rows || !parts_of(a, token, head, &n)) return;  // (kWaves = 4: all waves)
    const uint32_t parts = n.front + n.own, skip = a.front_parts - n.front;
    const uint64_t each = uint64_t{a.batch.rows} * a.heads;
    const auto slot = [&](uint32_t i) { return (i < n.front ? i : i + skip) * each + at; };
    const uint32_t sub = wave % kWaves * kAtOnce + lane / kLanes, col = lane % kLanes * 4;
    constexpr uint32_t kStep = kWaves * kAtOnce;
    const auto value = [&](uint32_t i) {
        return *reinterpret_cast<const float4 *>(a.part_o + slot(i) * D + col);
    };
    // The first values are asked for with the bounds and sums.  (Loops that are not
    // unrolled: a kernel begins with no code in the instruction cache, and what it runs once
    // costs about a microsecond a kilobyte.)
    const float4 none = {0.0f, 0.0f, 0.0f, 0.0f}, first = sub < parts ? value(sub) : none;
    float m = -INFINITY, l = n.past ? NAN : 0.0f;
#pragma nounroll
    for (uint32_t i = lane; i < parts; i += 64) {
        const float2 ml = a.part_ml[slot(i)];
        stats[mine][i] = ml;  // kWaves = 4: each wave writes the same
        m = fmaxf(m, ml.x);
    }
    m = wave_max(m);
    const float base = m == -INFINITY ? 0.0f : m;
#pragma nounroll
    for (uint32_t i = lane; i < parts; i += 64) {  // (its own)
        const float w = __builtin_amdgcn_exp2f((stats[mine][i].x - base) * a.c);
        l += w * stats[mine][i].y;
        weights[mine][i] = w;
    }
    l = wave_sum(l);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    float4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    const auto add = [&](float w, const float4 &y) {
        x.x += w * y.x, x.y += w * y.y, x.z += w * y.z, x.w += w * y.w;
    };
    if (sub < parts) add(weights[mine][sub], first);
    uint32_t i = sub + kStep;
    for (; i + 3 * kStep < parts; i += 4 * kStep) {
        float4 y[4];
        for (uint32_t e = 0; e < 4; e++) y[e] = value(i + e * kStep);
        for (uint32_t e = 0; e < 4; e++) add(weights[mine][i + e * kStep], y[e]);
    }
#pragma nounroll
    for (; i < parts; i += kStep) add(weights[mine][i], value(i));
    for (uint32_t d = kLanes; d < 64; d *= 2) {
        x.x += __shfl_xor(x.x, d), x.y += __shfl_xor(x.y, d);
        x.z += __shfl_xor(x.z, d), x.w += __shfl_xor(x.w, d);
    }
    if constexpr (kWaves == 4) {
        if (lane < kLanes) sums[wave][lane] = x;
        __syncthreads();
        if (wave) return;
        for (uint32_t j = 1; j < 4; j++) add(1.0f, sums[j][lane % kLanes]);
    }
    if (lane < kLanes) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        *reinterpret_cast<uint2 *>(a.out + token * a.out_stride + uint64_t{head} * D + col) =
            uint2{C::store(x.x * inv) | static_cast<uint32_t>(C::store(x.y * inv)) << 16,
                  C::store(x.z * inv) | static_cast<uint32_t>(C::store(x.w * inv)) << 16};
    }
    if (a.lse && lane == 0)
        a.lse[at] = l == 0.0f ? -INFINITY : fmaf(m, a.c, log2f(l) - Mat<C>::kLift) * kLn2;
}

constexpr uint32_t kSlots = 512;  // workgroups that the GPU holds at once: two a CU
// Up to so many rows and heads four waves join one (32 of them 17.9 us a call against 18.7
// with one wave each, 512 24.1 against 25.4), beyond one wave does (4096 50.6 us against
// 54.2 with four, 16,384 159 against 178).
constexpr uint32_t kFewJoins = 1024;

struct Plan {
    uint32_t own_tiles, own_groups, row_tiles, front_tiles, front_parts, own_parts;
    bool whole;
    uint64_t grid, joins, bytes;
};

uint64_t up(uint64_t n, uint64_t of) { return (n + of - 1) / of; }

int plan_of(uint64_t tokens, uint32_t heads, const df11_kv_cache &c, const df11_kv_batch &b,
            Plan *p) {
    *p = {};
    if (!heads || heads >> 20 || heads % c.heads || tokens > kMaxSequences || tokens * heads >> 31)
        return DF11_E_INVALID_ARG;
    if (!tokens || !b.sequences) return DF11_OK;
    const uint64_t rows = tokens * (heads / c.heads), tiles = up(rows, kRows);
    const uint64_t own_tiles = rows / kRows + b.sequences;
    const uint64_t space = std::min<uint64_t>(uint64_t{b.width} * c.page_size, INT32_MAX);
    const uint64_t own = std::max<uint64_t>(1, up(space, kTile)), front = up(b.prefix_len, kTile);
    // Rows that fill tiles by themselves, enough of them to fill half the GPU: the prefix
    // is read with the own tokens, and nothing has to be joined (32 heads over 8 behind 6,000
    // tokens: 250 rows, 64 tiles, 157 us against 64 in shares, 750 169 against 152, 1000,
    // 256 tiles, 176 against 193, 2000 256 against 429).  So it is, too, where a workgroup
    // has little to read (single tokens of 250 9.2 us against 13.0, 64 of up to 1000 27.5
    // against 33.8, a prompt of 512 21.9 against 41.3; at 32 tiles 59 against 56).  Lengths
    // are not known here: the tables' width stands for them, and the mean of the rows for
    // each sequence's.
    const uint64_t each = rows / std::min<uint64_t>(tokens, b.sequences), read = front + own;
    p->whole = read <= 8 || (!front && read <= 16 && own_tiles * c.heads >= kSlots) ||
               (each >= 64 && (read <= 24 || tiles * c.heads >= kSlots / 2));
    if (p->whole) {
        p->own_tiles = own_tiles;
        p->own_groups = 8 / std::__gcd(c.heads, 8u);
        p->grid = 8 * up(uint64_t{c.heads} * p->own_groups, 8) * up(own_tiles, p->own_groups);
        return p->grid < kMaxGrid ? DF11_OK : DF11_E_UNSUPPORTED;
    }
    // Shares: at least so many parts that items as long as each other can fill the GPU,
    // and for own tokens, whose lengths differ, up to 64 while they take no more than 64 MB
    // (8 sequences of up to 30,001 tokens 87 us against 96 without, 2 37 against 41; with up
    // to 256 the same).
    const auto parts = [](uint64_t n, uint64_t items, uint64_t least) {
        return std::min<uint64_t>({n, kMaxParts, std::max<uint64_t>(least, kSlots / items + 2)});
    };
    const uint64_t part_bytes = tokens * heads * (4ull * c.dim + 8);
    p->row_tiles = tiles;
    p->front_tiles = front;
    p->front_parts = parts(p->front_tiles, tiles * c.heads, 1);
    p->own_parts =
        parts(own, own_tiles * c.heads, std::min<uint64_t>(64, (64u << 20) / part_bytes));
    const uint64_t all = c.heads * (tiles * (p->front_tiles + kStart) + own_tiles * (own + kStart));
    p->grid = std::min<uint64_t>(kSlots, up(all + together(tiles) + 1, 2) * 2);
    p->joins = tokens * heads;
    if (all >> 31 || up(p->joins, 4) >= kMaxGrid) return DF11_E_UNSUPPORTED;
    p->bytes = (p->front_parts + p->own_parts) * part_bytes + 4 * up(3 + b.sequences, 4) * 4;
    return DF11_OK;
}

template <class C, uint32_t D>
int launch(const AttendArgs &a, const Plan &p, hipStream_t stream) {
    const dim3 grid(p.grid), block(kThreads);
    if (p.whole) {
        hipLaunchKernelGGL((attend_whole_kernel<C, D>), grid, block, 0, stream, a);
        return launched();
    }
    hipLaunchKernelGGL((attend_shares_kernel<C, D>), grid, block, 0, stream, a);
    if (const int rc = launched()) return rc;
    if (p.joins <= kFewJoins)
        hipLaunchKernelGGL((attend_join_kernel<C, D, 4>), dim3(p.joins), block, 0, stream, a);
    else
        hipLaunchKernelGGL((attend_join_kernel<C, D, 1>), dim3(up(p.joins, 4)), block, 0, stream,
                           a);
    return launched();
}

int check_sizes(const df11_kv_cache *cache, const df11_kv_batch *batch) {
    const int rc = check_cache_sizes(cache);
    return rc ? rc : check_batch_sizes(batch);
}

}  // namespace

extern "C" {

int df11_prefix_attention_workspace_bytes(uint64_t tokens, uint32_t heads,
                                          const df11_kv_cache *cache, const df11_kv_batch *batch,
                                          uint64_t *bytes) {
    if (!bytes) return DF11_E_INVALID_ARG;
    Plan p;
    int rc = check_sizes(cache, batch);
    if (!rc) rc = plan_of(tokens, heads, *cache, *batch, &p);
    if (!rc) *bytes = p.bytes;
    return rc;
}

int df11_prefix_attention(const void *q, uint64_t q_stride, uint64_t tokens, uint32_t heads,
                          float scale, const df11_kv_cache *cache, const df11_kv_batch *batch,
                          void *out, uint64_t out_stride, float *lse, void *workspace,
                          uint64_t workspace_bytes, hipStream_t stream) {
    Plan p;
    int rc = check_cache(cache);
    if (!rc) rc = check_batch(batch);
    if (!rc) rc = plan_of(tokens, heads, *cache, *batch, &p);
    if (rc) return rc;
    // (a c below the normal numbers would be taken for 0)
    if (!(scale >= 1.17549435e-38f) || !(scale * kLog2e < INFINITY)) return DF11_E_INVALID_ARG;
    if (!tokens || !batch->sequences) return DF11_OK;
    if (batch->prefix_len &&
        (!batch->prefix_table || misaligned(batch->prefix_table, 4) ||
         uint64_t{batch->prefix_pages} * cache->page_size < batch->prefix_len))
        return DF11_E_INVALID_ARG;
    const uint64_t cols = uint64_t{heads} * cache->dim;
    rc = check_strided(q, q_stride, cols, tokens, 2);
    if (!rc) rc = check_strided(out, out_stride, cols, tokens, 2);
    if (!rc && (misaligned(lse, 4) || (q == out && tokens > 1 && q_stride != out_stride)))
        rc = DF11_E_INVALID_ARG;
    if (!rc && p.bytes && (!workspace || misaligned(workspace, 16))) rc = DF11_E_INVALID_ARG;
    if (!rc && workspace_bytes < p.bytes) rc = DF11_E_BUFFER_TOO_SMALL;
    if (rc) return rc;
    const uint64_t parts = p.front_parts + p.own_parts;
    auto *part_o = static_cast<float *>(workspace);
    auto *part_ml = reinterpret_cast<float2 *>(part_o + parts * tokens * cols);
    const AttendArgs a{static_cast<const uint16_t *>(q), static_cast<const uint16_t *>(cache->k),
                       static_cast<const uint16_t *>(cache->v), static_cast<uint16_t *>(out), lse,
                       part_o, part_ml, q_stride, out_stride, cache->k_stride, cache->v_stride,
                       device_batch(*batch, tokens), scale * kLog2e,
                       std::min(kSlack / (scale * kLog2e), kMaxSlack), cache->pages,
                       static_cast<uint32_t>(__builtin_ctz(cache->page_size)), heads, cache->heads,
                       heads / cache->heads, p.own_tiles, p.own_groups, p.row_tiles, p.front_tiles,
                       p.front_parts, p.own_parts,
                       reinterpret_cast<uint32_t *>(part_ml + parts * tokens * heads)};
    if (cache->dtype == DF11_BF16)
        return cache->dim == 128 ? launch<BF16, 128>(a, p, stream) : launch<BF16, 64>(a, p, stream);
    return cache->dim == 128 ? launch<F16, 128>(a, p, stream) : launch<F16, 64>(a, p, stream);
}

}  // extern "C"
