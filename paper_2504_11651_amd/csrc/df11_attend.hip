// Attention of a batch to a prefix that its sequences share and to their own
// tokens, over a paged cache.
//
// One pass over keys and values: scores s of 64 tokens at a time, p = 2^(c s - m)
// with m a running bound of the row's c s (c = scale log2 e), l += p, O += p v, and
// l and O taken down by 2^(m - m') where the bound rises.  Parts of a row that
// different workgroups took are joined with 2^(m_i - m).
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

#include "df11_kv_common.h"

#include <algorithm>

namespace {

using namespace df11ops;

constexpr uint32_t kThreads = 256;
constexpr uint32_t kTile = 64;   // tokens of a tile
constexpr uint32_t kRows = 128;  // rows of a tile: 32 a wave
// How far c s may rise above m before O is taken down: p stays below 2^8, far from
// the largest fp16, and what is summed in 32 bits loses nothing.
constexpr float kSlack = 8.0f;

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
    static __device__ acc16 product(s8 a, s8 b, acc16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a),
                                                       __builtin_bit_cast(b8, b), c, 0, 0, 0);
    }
};
template <>
struct Mat<F16> {
    static constexpr uint32_t kInf = 0x7C00;
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
    float c;  // scale log2 e
    uint32_t pages, page_shift, heads, kv_heads, group;
    // the prefix: row tiles, parts and their tokens, workgroups; none if it is read
    // with a sequence's own tokens
    uint32_t front_tiles, front_parts, front_step, front_grid;
    // the own tokens: tile numbers, most parts, groups of tiles that share an XCD
    uint32_t own_tiles, own_parts, own_groups;
    uint32_t whole;  // a workgroup reads the prefix and all own tokens of its rows
};

// Parts that a sequence's `length` own tokens are cut into, and their tokens: at
// least four tiles each, and no more parts than there is room for.
struct Cut {
    uint32_t parts, step;
};
__device__ inline Cut cut(uint32_t length, uint32_t most) {
    const uint32_t tiles = (length + kTile - 1) / kTile;
    const uint32_t step = max(4u, (tiles + most - 1) / most);
    return {(tiles + step - 1) / step, step * kTile};
}

__device__ inline uint32_t swizzle64(uint32_t t) { return 2 * ((t >> 1) & 3) | ((t >> 3) & 1); }
__device__ inline uint32_t swizzle128(uint32_t t) { return 2 * (t & 7) | ((t >> 3) & 1); }
template <uint32_t D>
__device__ inline uint32_t swizzle(uint32_t t) {
    return D == 64 ? swizzle64(t) : swizzle128(t);
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
    __device__ Places(uint32_t lane) {
        const uint32_t half = lane >> 5, t = lane & 31;
        for (uint32_t s = 0; s < kSteps; s++)
            k[s] = t * kRowBytes + (((2 * s + half) ^ swizzle<D>(t & 15)) << 4);
        // groups of 16 lanes read 4 tokens x 16 values: lane i the 8 bytes i % 4 of token i / 4
        const uint32_t i = lane & 15, tok = 4 * half + (i >> 2);
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; b++)
#pragma unroll
            for (uint32_t e = 0; e < 2; e++) {
                const uint32_t piece = 4 * b + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
                v[b][e] = (tok + 8 * e) * kRowBytes + ((piece ^ swizzle<D>(tok + 8 * e)) << 4) +
                          (i & 1) * 8;
            }
    }
};

template <class C, uint32_t D>
struct Worker {
    using P = Places<D>;
    static constexpr uint32_t kBytes = kTile * 2 * D;  // of a tile of K or V
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

    __device__ Worker(const AttendArgs &args, uint32_t kvh_)
        : a(args), at(threadIdx.x & 63), lane(threadIdx.x & 63),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), kvh(kvh_) {
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

    // Loads this wave's 16 tokens of a tile into LDS, past the registers.  True: the
    // tile's tokens lie on pages of the cache; where they do not, those of another page
    // are loaded in their place.
    __device__ bool load(const Range &r, uint32_t tile, uint8_t *k, uint8_t *v) const {
        uint32_t page = 0;
        bool fine = true;
        // (16 tokens lie on one page, and 64 do from that page size on)
        for (uint32_t i = 0; i < (a.page_shift >= 6 ? 1u : 4u); i++) {
            const uint32_t at = min(tile + 16 * i, r.end - 1) >> a.page_shift;
            uint32_t p = ~0u;
            if (at < r.width) p = __builtin_amdgcn_readfirstlane(r.table[at]);
            fine = fine && p < a.pages;
            if (i == wave || a.page_shift >= 6) page = p;
        }
        if (page >= a.pages) page = 0;
        const uint32_t t = min(tile + 16 * wave, (r.end - 1) & ~15u);  // behind: of no effect
        const uint64_t in = (uint64_t{t & ((1u << a.page_shift) - 1)} * D + head_off) * 2;
        const auto *kp = reinterpret_cast<const uint8_t *>(a.k + page * a.page_k) + in;
        const auto *vp = reinterpret_cast<const uint8_t *>(a.v + page * a.page_v) + in;
        k += 16 * wave * P::kRowBytes;
        v += 16 * wave * P::kRowBytes;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; i++) {
            __builtin_amdgcn_global_load_lds((mem_void *)(kp + from[i]), (lds_void *)(k + i * 1024),
                                             16, 0, 0);
            __builtin_amdgcn_global_load_lds((mem_void *)(vp + from[i]), (lds_void *)(v + i * 1024),
                                             16, 0, 0);
        }
        return fine;
    }
    // Waits for them, and clears the values of tokens behind the range: they meet a
    // p of 0, and what memory holds there may be an infinity.
    __device__ void landed(const Range &r, uint32_t tile, uint8_t *v) const {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (tile + kTile <= r.end) return;
#pragma unroll
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

    // Tokens 32 kFirst .. 32 (kFirst + kCount) of a tile.  `end`: the tokens that the
    // lane's row sees, from the tile's first; `masked`: not all rows see all.
    template <uint32_t kCount>
    __device__ void tokens(const uint8_t *k, const uint8_t *v, uint32_t first, bool masked,
                           int32_t end, bool lost, bool uneven) {
        k += first * P::kRowBytes;
        v += first * P::kRowBytes;
        acc16 s[kCount];
#pragma unroll
        for (uint32_t b = 0; b < kCount; b++) {
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) s[b][e] = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < P::kSteps; i++)
                s[b] = Mat<C>::product(
                    *reinterpret_cast<const s8 *>(k + at.k[i] + b * 32 * P::kRowBytes), q[i], s[b]);
        }
        if (lost)  // a page outside the cache
#pragma unroll
            for (auto &x : s)
#pragma unroll
                for (uint32_t e = 0; e < 16; e++) x[e] = NAN;
        const int32_t seen = end - static_cast<int32_t>(first + 4 * (lane >> 5));
        if (masked)
#pragma unroll
            for (uint32_t b = 0; b < kCount; b++)
#pragma unroll
                for (uint32_t e = 0; e < 16; e++)
                    if (static_cast<int32_t>(32 * b + 8 * (e / 4) + e % 4) >= seen)
                        s[b][e] = -INFINITY;
        float top = s[0][0];
#pragma unroll
        for (uint32_t b = 0; b < kCount; b++)
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) top = fmaxf(top, s[b][e]);
        top = fmaxf(top, __shfl_xor(top, 32)) * a.c;
        if (__any(top > m + kSlack)) {
            const float rise = fmaxf(m, top);
            const float down = __builtin_amdgcn_exp2f(m - (rise == -INFINITY ? 0.0f : rise));
            m = rise;
            l *= down;
#pragma unroll
            for (auto &x : o)
#pragma unroll
                for (uint32_t e = 0; e < 16; e++) x[e] *= down;
        }
        const float base = m == -INFINITY ? 0.0f : m;
        s8 p[2 * kCount];
#pragma unroll
        for (uint32_t b = 0; b < kCount; b++)
#pragma unroll
            for (uint32_t e = 0; e < 16; e++) {
                const float x = __builtin_amdgcn_exp2f(fmaf(s[b][e], a.c, -base));
                l += x;
                p[2 * b + e / 8][e % 8] = static_cast<short>(C::store(x));
            }
        if (uneven) {
            // rows see different tokens: a value that is an infinity or a NaN must not
            // meet the p of 0 of a row that does not see it
            u4 worst = {0, 0, 0, 0};
#pragma unroll
            for (uint32_t i = 0; i < 2 * kCount; i++)
#pragma unroll
                for (uint32_t b = 0; b < P::kBlocks; b++)
                    worst |= not_finite(read_v(v + i * 16 * P::kRowBytes, at.v[b][0], at.v[b][1]));
            if (__any((worst[0] | worst[1] | worst[2] | worst[3]) != 0)) {
                products<kCount, true>(v, p);
                add_not_finite<kCount>(v, end - static_cast<int32_t>(first));
                return;
            }
        }
        products<kCount, false>(v, p);
    }

    // Of each half of a word: 1 if it holds an infinity or a NaN.
    typedef unsigned short us8 __attribute__((ext_vector_type(8)));
    __device__ static u4 not_finite(s8 x) {
        const us8 t = __builtin_bit_cast(us8, x) & static_cast<unsigned short>(0x7FFF);
        return __builtin_bit_cast(u4, (t + static_cast<unsigned short>(0x8000 - Mat<C>::kInf)) >> 15);
    }
    template <uint32_t kCount, bool kFinite>
    __device__ void products(const uint8_t *v, const s8 (&p)[2 * kCount]) {
#pragma unroll
        for (uint32_t i = 0; i < 2 * kCount; i++)
#pragma unroll
            for (uint32_t b = 0; b < P::kBlocks; b++) {
                s8 x = read_v(v + i * 16 * P::kRowBytes, at.v[b][0], at.v[b][1]);
                if constexpr (kFinite)  // the others as 0
                    x &= __builtin_bit_cast(s8, __builtin_bit_cast(us8, not_finite(x)) -
                                                    static_cast<unsigned short>(1));
                o[b] = Mat<C>::product(x, p[i], o[b]);
            }
    }
    // What the products left out, token after token: the sum becomes the infinity or the
    // NaN of every value that the lane's row sees.
    template <uint32_t kCount>
    __device__ void add_not_finite(const uint8_t *v, int32_t seen) {
        typedef unsigned short us4 __attribute__((ext_vector_type(4)));
#pragma nounroll
        for (uint32_t t = 0; t < 32 * kCount; t++) {
            const uint32_t sees = static_cast<int32_t>(t) < seen ? ~0u : 0u;
#pragma unroll
            for (uint32_t b = 0; b < P::kBlocks; b++)
#pragma unroll
                for (uint32_t e = 0; e < 4; e++) {
                    const us4 x = *reinterpret_cast<const us4 *>(
                        v + t * P::kRowBytes + (((4 * b + e) ^ swizzle<D>(t & 15)) << 4) +
                        8 * (lane >> 5));
                    const us4 bad = ((x & static_cast<unsigned short>(0x7FFF)) +
                                     static_cast<unsigned short>(0x8000 - Mat<C>::kInf)) >> 15;
                    const us4 y = x & -bad & static_cast<unsigned short>(sees);
#pragma unroll
                    for (uint32_t j = 0; j < 4; j++) o[b][4 * e + j] += C::load(y[j]);
                }
        }
    }

    // One tile of a range.  `sees`: tokens of the range that the lane's row sees (every
    // row of the workgroup at least `least`, at most r.end).
    template <bool kSplit>
    __device__ void tile(const Range &r, uint32_t tile, const uint8_t *k, const uint8_t *v,
                         int32_t sees, int32_t least, bool fine) {
        const int32_t at = static_cast<int32_t>(tile);
        const bool masked = at + static_cast<int32_t>(kTile) > least;
        const bool uneven = masked && least < static_cast<int32_t>(r.end);
        if constexpr (kSplit)
            tokens<1>(k, v, 32 * (wave & 1), masked, sees - at, !fine, uneven);
        else
            tokens<2>(k, v, 0, masked, sees - at, !fine, uneven);
    }
};

// kSplit: the rows are at most 64, waves 2 i and 2 i + 1 take rows 32 i.. and share
// the tokens of a tile.
template <class C, uint32_t D, bool kSplit>
__device__ __forceinline__ void attend(const AttendArgs &a, uint32_t kvh, uint32_t row0,
                                       uint32_t rows, uint32_t part, const Range &front,
                                       const Range &own, int32_t places, uint8_t *k0, uint8_t *v0,
                                       uint8_t *k1, uint8_t *v1, float2 *stats) {
    using W = Worker<C, D>;
    using P = Places<D>;
    W w(a, kvh);
    const uint32_t half = w.lane >> 5, n = w.lane & 31;
    const uint32_t mine = 32 * (kSplit ? w.wave >> 1 : w.wave);
    const bool busy = mine < rows;
    const uint32_t row = row0 + min(mine + n, rows - 1);
    const uint32_t token = row / a.group;
    const uint32_t head = kvh * a.group + row % a.group;
    if (busy) {
        const uint16_t *p = a.q + token * a.q_stride + uint64_t{head} * D + 8 * half;
#pragma unroll
        for (uint32_t i = 0; i < P::kSteps; i++)
            w.q[i] = __builtin_bit_cast(s8, load16(p + 16 * i));
    }
    for (uint32_t i = 0; i < 2; i++) {
        const Range r = i ? own : front;
        if (r.begin >= r.end) continue;
        // own tokens that the rows see: `places` the workgroup's first row
        const int32_t end = static_cast<int32_t>(r.end);
        const int32_t least = i ? min(places, end) : end;
        const int32_t sees =
            i ? min(places + static_cast<int32_t>(token - row0 / a.group), end) : end;
        bool fine0 = w.load(r, r.begin, k0, v0), fine1 = true;
        w.landed(r, r.begin, v0);
        __syncthreads();
        for (uint32_t t = r.begin;; t += 2 * kTile) {
            const bool more = t + kTile < r.end;
            if (more) fine1 = w.load(r, t + kTile, k1, v1);
            if (busy) w.template tile<kSplit>(r, t, k0, v0, sees, least, fine0);
            if (!more) break;
            w.landed(r, t + kTile, v1);
            __syncthreads();
            const bool again = t + 2 * kTile < r.end;
            if (again) fine0 = w.load(r, t + 2 * kTile, k0, v0);
            if (busy) w.template tile<kSplit>(r, t + kTile, k1, v1, sees, least, fine1);
            if (!again) break;
            w.landed(r, t + 2 * kTile, v0);
            __syncthreads();
        }
        __syncthreads();
    }
    // Rows through LDS: a wave's 32 x D floats in a buffer, 16-byte pieces of row n at
    // piece ^ n.  Waves that shared tokens bring theirs to the larger bound first.
    float l = w.l + __shfl_xor(w.l, 32), m = w.m;
    float *slice = reinterpret_cast<float *>(w.wave == 0 ? k0 : w.wave == 1 ? v0 : w.wave == 2 ? k1 : v1);
    if constexpr (kSplit) {
        if (half == 0) stats[w.wave * 32 + n] = float2{m, l};
        __syncthreads();
        const float2 other = stats[(w.wave ^ 1) * 32 + n];
        const float both = fmaxf(m, other.x), base = both == -INFINITY ? 0.0f : both;
        const float down = __builtin_amdgcn_exp2f(m - base);
        l = l * down + other.y * __builtin_amdgcn_exp2f(other.x - base);
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
    for (uint32_t i = threadIdx.x; i < rows * kPieces; i += kThreads) {
        const uint32_t r = i / kPieces, piece = i % kPieces;
        const uint32_t src = kSplit ? 2 * (r / 32) : r / 32, nn = r % 32;
        const float2 ml = stats[src * 32 + nn];
        float x[8];
        for (uint32_t s = 0; s < (kSplit ? 2 : 1); s++) {
            const uint32_t from = src + s;
            const float *p = reinterpret_cast<const float *>(
                                 from == 0 ? k0 : from == 1 ? v0 : from == 2 ? k1 : v1) + nn * D;
#pragma unroll
            for (uint32_t e = 0; e < 2; e++) {
                const float4 y = *reinterpret_cast<const float4 *>(
                    p + (((2 * piece + e) ^ (nn & (D / 4 - 1))) << 2));
                const float z[4] = {y.x, y.y, y.z, y.w};
                for (uint32_t j = 0; j < 4; j++) x[4 * e + j] = s ? x[4 * e + j] + z[j] : z[j];
            }
        }
        const uint32_t at = row0 + r, tok = at / a.group, hd = kvh * a.group + at % a.group;
        if (a.whole) {
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
                    ml.y == 0.0f ? -INFINITY : (ml.x + log2f(ml.y)) * kLn2;
        } else {
            const uint64_t slot = (uint64_t{part} * a.batch.rows + tok) * a.heads + hd;
            float *p = a.part_o + slot * D + 8 * piece;
            *reinterpret_cast<float4 *>(p) = float4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<float4 *>(p + 4) = float4{x[4], x[5], x[6], x[7]};
            if (piece == 0) a.part_ml[slot] = ml;
        }
    }
}

template <class C, uint32_t D>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendArgs a) {
    constexpr uint32_t kBytes = kTile * 2 * D;
    __shared__ __attribute__((aligned(1024))) uint8_t k0[kBytes], v0[kBytes], k1[kBytes], v1[kBytes];
    __shared__ float2 stats[4 * 32];
    const uint32_t x = blockIdx.x & 7;
    const Batch &b = a.batch;
    Range front{}, own{};
    uint32_t kvh, row0, rows, part;
    int32_t first = 0;
    if (blockIdx.x < a.front_grid) {
        // a part of the prefix for rows of all sequences; the tiles of a part and head
        // have numbers that one XCD takes, whose L2 then holds its K and V
        const uint32_t y = blockIdx.x >> 3, pair = y / a.front_tiles * 8 + x;
        kvh = pair % a.kv_heads;
        part = pair / a.kv_heads;
        if (part >= a.front_parts) return;
        const uint32_t all = b.first(b.sequences) * a.group;
        row0 = y % a.front_tiles * kRows;
        if (row0 >= all) return;
        rows = min(kRows, all - row0);
        const uint32_t begin = part * a.front_step;
        front = {b.prefix_table, b.prefix_pages, begin, min(b.prefix_len, begin + a.front_step)};
    } else {
        // a sequence's rows: tile numbers ascend over the sequences, and the last, which
        // see the most, come first; an XCD takes whole heads or every own_groups-th tile
        const uint32_t z = (blockIdx.x - a.front_grid) >> 3;
        const uint32_t per = (a.own_tiles + a.own_groups - 1) / a.own_groups * a.own_parts;
        const uint32_t combo = z / per * 8 + x, rest = z % per;
        kvh = combo / a.own_groups;
        if (kvh >= a.kv_heads) return;
        const uint32_t cut_part = rest % a.own_parts;
        const uint32_t number = rest / a.own_parts * a.own_groups + combo % a.own_groups;
        if (number >= a.own_tiles) return;
        const uint32_t id = a.own_tiles - 1 - number;
        // sequence s has the numbers from (its first row) / kRows + s on: never fewer
        // than its tiles
        const auto base = [&](uint32_t s) { return b.first(s) * a.group / kRows + s; };
        const uint32_t s = __builtin_amdgcn_readfirstlane(wave_search(b.sequences, id, base));
        if (s == ~0u) return;
        const uint32_t from = b.first(s), to = b.first(s + 1);
        row0 = from * a.group + (id - base(s)) * kRows;
        if (to <= from || row0 >= to * a.group) return;
        rows = min(kRows, to * a.group - row0);
        // tokens that the tile's first and last rows see
        const int32_t length = max(b.length[s], 0);
        const int32_t before = length - static_cast<int32_t>(to) + 1;
        first = before + static_cast<int32_t>(row0 / a.group);
        const int32_t last = before + static_cast<int32_t>((row0 + rows - 1) / a.group);
        const uint32_t end = max(last, 0);
        const int32_t *table = b.table + s * b.table_stride;
        if (a.whole) {
            part = 0;
            front = {b.prefix_table, b.prefix_pages, 0, b.prefix_len};
            own = {table, b.width, 0, end};
        } else {
            const Cut c = cut(length, a.own_parts);
            if (cut_part >= c.parts) return;
            part = a.front_parts + cut_part;
            own = {table, b.width, cut_part * c.step, min(end, (cut_part + 1) * c.step)};
        }
    }
    if (rows <= 64)
        attend<C, D, true>(a, kvh, row0, rows, part, front, own, first, k0, v0, k1, v1, stats);
    else
        attend<C, D, false>(a, kvh, row0, rows, part, front, own, first, k0, v0, k1, v1, stats);
}

// Joins the parts of a row and head: a wave for each.  A lane has one part's bound
// and sum, then D / 64 of the values.
template <class C, uint32_t D>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t at = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const uint32_t token = at / a.heads, head = at % a.heads;
    if (token >= a.batch.rows) return;
    const Owner o = owner(a.batch, token);
    if (o.s == ~0u) return;
    const uint32_t parts = a.front_parts + cut(max(a.batch.length[o.s], 0), a.own_parts).parts;
    const uint64_t each = uint64_t{a.batch.rows} * a.heads;
    const float2 ml = lane < parts ? a.part_ml[lane * each + at] : float2{-INFINITY, 0.0f};
    const float m = wave_max(ml.x), base = m == -INFINITY ? 0.0f : m;
    const float part = __builtin_amdgcn_exp2f(ml.x - base);
    const float l = wave_sum(part * ml.y);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    constexpr uint32_t kEach = D / 64;
    float x[kEach] = {};
    const float *p = a.part_o + uint64_t{at} * D + lane * kEach;
    for (uint32_t i = 0; i < parts; i++) {
        const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(part), i));
        for (uint32_t e = 0; e < kEach; e++) x[e] += f * p[i * each * D + e];
    }
    uint16_t *out = a.out + token * a.out_stride + uint64_t{head} * D + lane * kEach;
    if constexpr (kEach == 2)
        *reinterpret_cast<uint32_t *>(out) =
            C::store(x[0] * inv) | static_cast<uint32_t>(C::store(x[1] * inv)) << 16;
    else
        *out = C::store(x[0] * inv);
    if (a.lse && lane == 0) a.lse[at] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

constexpr uint32_t kMaxParts = 32;  // of the prefix, and of a sequence's own tokens
constexpr uint32_t kSlots = 512;    // workgroups that the GPU holds at once: two a CU

struct Plan {
    uint32_t front_tiles, front_parts, front_step, own_tiles, own_parts, own_groups, whole;
    uint64_t front_grid, own_grid, bytes;
};

uint64_t up(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }

int plan_of(uint64_t tokens, uint32_t heads, const df11_kv_cache &c, const df11_kv_batch &b,
            Plan *p) {
    *p = {};
    if (!heads || heads >> 20 || heads % c.heads || tokens > kMaxSequences || tokens * heads >> 31)
        return DF11_E_INVALID_ARG;
    if (!tokens || !b.sequences) return DF11_OK;
    const uint64_t group = heads / c.heads, rows = tokens * group;
    const uint64_t tiles = (rows + kRows - 1) / kRows;
    const uint64_t own_tiles = rows / kRows + b.sequences;
    const uint64_t capacity = uint64_t{b.width} * c.page_size;
    p->own_tiles = own_tiles;
    p->own_groups = 8 / std::__gcd(c.heads, 8u);
    p->own_parts = 1;
    // Rows that fill tiles by themselves, enough of them to fill the GPU: the prefix is
    // read with the own tokens, and nothing has to be joined.
    const uint64_t each = rows / std::min<uint64_t>(tokens, b.sequences);
    p->whole = each >= 64 && tiles * c.heads >= kSlots / 2;
    if (!p->whole) {
        if (b.prefix_len) {
            const uint64_t parts = std::max<uint64_t>(
                1, std::min<uint64_t>(kMaxParts, kSlots / (tiles * c.heads)));
            p->front_tiles = tiles;
            p->front_step = std::max<uint64_t>(4 * kTile, up((b.prefix_len + parts - 1) / parts, kTile));
            p->front_parts = (b.prefix_len + p->front_step - 1) / p->front_step;
            p->front_grid = 8 * tiles * up(uint64_t{c.heads} * p->front_parts, 8) / 8;
        }
        p->own_parts = std::max<uint64_t>(
            1, std::min<uint64_t>({kMaxParts, (capacity + 4 * kTile - 1) / (4 * kTile),
                                   4 * kSlots / (own_tiles * c.heads)}));
        p->bytes = (p->front_parts + p->own_parts) * tokens * heads * (4ull * c.dim + 8);
    }
    p->own_grid = up(uint64_t{c.heads} * p->own_groups, 8) *
                  ((own_tiles + p->own_groups - 1) / p->own_groups) * p->own_parts;
    const uint64_t joins = p->whole ? 0 : (tokens * heads + 3) / 4;
    return std::max(p->front_grid + p->own_grid, joins) < kMaxGrid ? DF11_OK : DF11_E_UNSUPPORTED;
}

template <class C, uint32_t D>
int launch(const AttendArgs &a, uint64_t grid, hipStream_t stream) {
    hipLaunchKernelGGL((attend_kernel<C, D>), dim3(grid), dim3(kThreads), 0, stream, a);
    if (const int rc = launched()) return rc;
    if (a.whole) return DF11_OK;
    const uint32_t wgs = (a.batch.rows * a.heads + 3) / 4;
    hipLaunchKernelGGL((attend_join_kernel<C, D>), dim3(wgs), dim3(kThreads), 0, stream, a);
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
    if (!(scale > 0.0f) || !(scale * kLog2e < INFINITY)) return DF11_E_INVALID_ARG;
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
    const uint64_t values = (p.front_parts + p.own_parts) * tokens * cols;
    const AttendArgs a{static_cast<const uint16_t *>(q), static_cast<const uint16_t *>(cache->k),
                       static_cast<const uint16_t *>(cache->v), static_cast<uint16_t *>(out), lse,
                       static_cast<float *>(workspace),
                       reinterpret_cast<float2 *>(static_cast<float *>(workspace) + values),
                       q_stride, out_stride, cache->k_stride, cache->v_stride,
                       device_batch(*batch, tokens), scale * kLog2e, cache->pages,
                       static_cast<uint32_t>(__builtin_ctz(cache->page_size)), heads, cache->heads,
                       heads / cache->heads, p.front_tiles, p.front_parts, p.front_step,
                       static_cast<uint32_t>(p.front_grid), p.own_tiles, p.own_parts, p.own_groups,
                       p.whole};
    const uint64_t grid = p.front_grid + p.own_grid;
    if (cache->dtype == DF11_BF16)
        return cache->dim == 128 ? launch<BF16, 128>(a, grid, stream)
                                 : launch<BF16, 64>(a, grid, stream);
    return cache->dim == 128 ? launch<F16, 128>(a, grid, stream) : launch<F16, 64>(a, grid, stream);
}

}  // extern "C"
