// Low-rank adapters of many requests beside a shared projection, and their
// gradients.  With v[t] = A_i x[t] and u[t] = s_i B_i^T dy[t], i the adapter of t:
//   out = base + s_i B_i v      dx = dx_base + A_i^T u
//   dA_i = sum u x^T            dB_i = s_i sum dy v^T
//
// A rank of 8 to 128 against thousands of columns: everything is bound by
// reading x, base and dy and writing out and dx once; the products are small and
// go to the matrix cores (v_mfma_f32_16x16x32_bf16) so that nothing else gets in
// the way.  The kernels:
//   shrink  u and v: 16 tokens by all ranks, the columns over the waves of a
//           workgroup and over workgroups (partial sums; `expand` and `prepare`
//           add them in order), so that one token alone still has many loads
//           under way;
//   prepare u and v, their parts added, as the terms that the others multiply;
//   expand  out and dx: 64 columns by 16 tokens a wave, through LDS so that base
//           and out are read and written in whole rows; few tokens one by one;
//   outer   dA and dB: 64 columns a wave over a chunk of tokens, partial sums
//           for several chunks, then `join`.
// u and v are sums in 32 bits; where they meet the matrix cores they are cut into
// three BF16 terms, which lose nothing, and so is an fp32 dy.  x, A, B and a BF16
// dy are BF16 as they are.  A tile of tokens may hold several adapters: a kernel goes
// through the distinct ones, each for its own tokens' rows; up to kFewTokens
// tokens they are spread over workgroups instead.  A workgroup reads which
// adapters its tokens have from `adapter`: nothing is sorted or prepared.
//
// Kernel times, and what bounds them:
//   1 token, 4096 -> 4096, rank 16: shrink 3.4 us, expand 3.0: loads after one another;
//   64 tokens of 32 adapters, 4096 -> 14336, fp32: 5.5 and 6.7 (22 MB of adapters, base
//     and out): the same, and the adapters' rows from the L2 cache;
//   6001 tokens, 4096 -> 14336, bf16: shrink 19.7, prepare 4.8, expand 73 (344 MB: 4.7
//     TB/s; 70 with two of the three terms): memory;
//   gradients, 8192 tokens, 4096 x 4096, rank 64: transpose 5, shrink 62, prepare 8,
//     expand 51 (44 with two terms), outer 61, join 13 for 67 MB each of dy, x, dx_base
//     and dx: the loads of A, B and of the terms, which at this rank are as many as those
//     of the tokens;
//   of an LM head of 128,256 rows, 1024 tokens, fp32 dy (525 MB): shrink 111, outer 104:
//     memory (4.8 and 5.1 TB/s), dy is read twice.
#include "df11_ops_common.h"

#include <algorithm>
#include <type_traits>

namespace {

using namespace df11ops;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kThreads = 256;
constexpr uint32_t kWaves = kThreads / 64;
constexpr uint32_t kTile = 16;        // tokens of a matrix product
constexpr uint32_t kFewTokens = 256;  // up to these, a workgroup an adapter of a tile
constexpr uint32_t kManyTiles = 4;    // tiles that a workgroup of `expand` takes above them
constexpr uint32_t kFewValues = 1024; // tokens x rank up to which `expand` takes single tokens

__device__ f32x4 mfma(const uint4 &a, const uint4 &b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight floats as the sums of three BF16 terms each, exactly: 24 bits of mantissa
// cut into 8, 8 and 8, each remainder a difference without rounding.  An infinity
// is all in the first term, and so is a NaN.
constexpr uint32_t kTerms = 3;
__device__ void split8(const float *v, uint4 *terms) {
    uint32_t first[8], second[8], third[8];
    float most = 0.0f;
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
        first[e] = __float_as_uint(v[e]) & 0xFFFF0000u;
        const float rest = v[e] - __uint_as_float(first[e]);
        second[e] = __float_as_uint(rest) & 0xFFFF0000u;
        third[e] = __float_as_uint(rest - __uint_as_float(second[e]));
        most += fabsf(rest);
    }
    if (__any(!(most < INFINITY))) {  // inf - inf
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            if (!(fabsf(v[e]) < INFINITY)) {
                // the quiet bit: cutting must not leave an infinity of a NaN
                first[e] |= v[e] != v[e] ? 0x00400000u : 0u;
                second[e] = third[e] = 0;
            }
    }
    const auto pack = [](const uint32_t *w) {  // the upper halves
        return uint4{__builtin_amdgcn_perm(w[1], w[0], 0x07060302u),
                     __builtin_amdgcn_perm(w[3], w[2], 0x07060302u),
                     __builtin_amdgcn_perm(w[5], w[4], 0x07060302u),
                     __builtin_amdgcn_perm(w[7], w[6], 0x07060302u)};
    };
    terms[0] = pack(first);
    terms[1] = pack(second);
    terms[2] = pack(third);
}

__device__ uint4 zero4() { return uint4{0, 0, 0, 0}; }

// The adapter of a token, -1 for none; -2 past the last token.
__device__ int32_t adapter_of(const int32_t *adapter, uint64_t t, uint64_t tokens, uint32_t n) {
    if (t >= tokens) return -2;
    const int32_t i = adapter[t];
    return i >= 0 && static_cast<uint32_t>(i) < n ? i : -1;
}

// Calls f(adapter, its tokens' bits) for the distinct adapters from `least` on of
// the first kTokens lanes' `id`.  Workgroup z of gridDim.z takes every
// gridDim.z-th of them.
template <uint32_t kTokens, class F>
__device__ void each_adapter(int32_t id, int32_t least, F f) {
    constexpr uint64_t kAll = kTokens == 64 ? ~0ull : (1ull << kTokens) - 1;
    uint64_t left = __ballot(id >= least) & kAll;
    uint32_t turn = 0;
    while (left) {
        const int32_t a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const uint64_t mine = __ballot(id == a) & kAll;
        left &= ~mine;
        if (turn++ % gridDim.z == blockIdx.z) f(a, mine);
    }
}

// ---------------------------------------------------------------------- shrink
// part[split][t][r] = sum over the split's columns of x[t][c] w[i][r][c]; rows of
// tokens without an adapter are not written (nor read later).
struct ShrinkJob {
    const void *x;
    const uint16_t *w;  // n_adapters x rank x len
    float *part;
    uint64_t stride;
    uint32_t len, per, splits;  // columns, columns of a split (a multiple of 256)
};
struct ShrinkArgs {
    ShrinkJob job[2];  // splits of the first, then of the second, along gridDim.y
    const int32_t *adapter;
    uint64_t tokens;
    uint32_t rank, n_adapters;
};

// 64 columns of kSub tiles of 16 tokens and of the ranks: lane group q takes 16 of
// the columns, in both operands, so that every load brings whole 128-byte lines.
template <class T, uint32_t kRanks, uint32_t kSub>
struct Columns {
    uint4 x[kSub][T::kVec == 4 ? 4 : 2], w[kRanks][2];
    __device__ void load(const typename T::raw *const *row, const uint16_t *w0, uint32_t k,
                         uint32_t len, uint32_t rank, uint32_t c, bool in) {
#pragma unroll
        for (uint32_t s = 0; s < kSub; ++s)
#pragma unroll
            for (uint32_t e = 0; e < sizeof(x[0]) / 16; ++e)
                x[s][e] = in ? *reinterpret_cast<const uint4 *>(row[s] + k + T::kVec * e) : zero4();
#pragma unroll
        for (uint32_t r = 0; r < kRanks; ++r) {
            const uint16_t *wr = w0 + static_cast<uint64_t>(min(16 * r + c, rank - 1)) * len + k;
#pragma unroll
            for (uint32_t e = 0; e < 2; ++e)
                w[r][e] = in ? *reinterpret_cast<const uint4 *>(wr + 8 * e) : zero4();
        }
    }
    __device__ void add(f32x4 (*acc)[kRanks]) const {
#pragma unroll
        for (uint32_t s = 0; s < kSub; ++s)
#pragma unroll
            for (uint32_t e = 0; e < 2; ++e) {
                constexpr uint32_t kParts = T::kVec == 4 ? kTerms : 1;
                uint4 t[kParts];
                if constexpr (T::kVec == 4) {
                    float v[8];
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) v[i] = F32::get(x[s][2 * e + i / 4], i % 4);
                    split8(v, t);
                } else {
                    t[0] = x[s][e];
                }
#pragma unroll
                for (uint32_t r = 0; r < kRanks; ++r)
#pragma unroll
                    for (uint32_t i = 0; i < kParts; ++i)
                        acc[s][r] = mfma(t[i], w[r][e], acc[s][r]);
            }
    }
};

// Tiles of 16 tokens that a wave of the wide kernel takes.  From 32 ranks the loads
// of w are more than those of x, and tiles share them (8192 tokens, rank 64: one
// tile 92 us, two 72, four 61), with an fp32 x at any rank (1024 tokens x 128,256,
// rank 16: one 124 us, two 110); else more tiles only lower the number of waves
// (6001 tokens, rank 16: one 18.1 us, two 21.6).  Above 64 ranks four do not fit the
// registers.
constexpr uint32_t wide_tiles(uint32_t rank, bool f32) {
    return !f32 && rank > 32 && rank <= 64 ? 4 : rank > 16 || f32 ? 2 : 1;
}
constexpr uint32_t wide_tokens(uint32_t rank, bool f32) {
    return kTile * kWaves * wide_tiles(rank, f32);
}

// kWide: each wave takes tiles of its own, over all the columns of the split (the
// waves' loads of w meet in the L1 cache, and each serves two tiles); else the
// waves share one tile's columns and add their sums through LDS, so that a single
// tile has four times the loads under way.
template <class T, uint32_t kRanks, bool kWide, uint32_t kWideTiles>
__device__ void shrink(const ShrinkArgs &g, const ShrinkJob &j, uint32_t split, float *red) {
    constexpr uint32_t kSub = kWide ? kWideTiles : 1, kTokens = kSub * kTile;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, q = lane >> 4;
    const uint64_t t0 =
        (uint64_t{blockIdx.x} * (kWide ? kWaves : 1) + (kWide ? wave : 0)) * kTokens;
    if (t0 >= g.tokens) return;  // a whole workgroup, or a wave that meets no barrier
    const int32_t id = adapter_of(g.adapter, t0 + (lane & (kTokens - 1)), g.tokens, g.n_adapters);
    const typename T::raw *x[kSub];
#pragma unroll
    for (uint32_t s = 0; s < kSub; ++s)
        x[s] = static_cast<const typename T::raw *>(j.x) +
               std::min(t0 + kTile * s + c, g.tokens - 1) * j.stride;
    const uint32_t from = split * j.per, to = min(j.len, from + j.per);
    constexpr uint32_t kStep = 64 * (kWide ? 1 : kWaves);
    each_adapter<kTokens>(id, 0, [&](int32_t a, uint64_t mine) {
        const uint16_t *w = j.w + static_cast<uint64_t>(a) * g.rank * j.len;
        f32x4 acc[kSub][kRanks];
#pragma unroll
        for (uint32_t s = 0; s < kSub; ++s)
#pragma unroll
            for (uint32_t r = 0; r < kRanks; ++r) acc[s][r] = f32x4{0, 0, 0, 0};
        // the next step's loads are under way; lengths are multiples of 16
        Columns<T, kRanks, kSub> one, two;
        uint32_t k = from + (kWide ? 0 : 64 * wave) + 16 * q;
        one.load(x, w, k, j.len, g.rank, c, k < to);
        for (; k - 16 * q < to; k += 2 * kStep) {
            two.load(x, w, k + kStep, j.len, g.rank, c, k + kStep < to);
            one.add(acc);
            one.load(x, w, k + 2 * kStep, j.len, g.rank, c, k + 2 * kStep < to);
            two.add(acc);
        }
        // token 4q + e of a tile, rank 16r + c
        if constexpr (kWide) {
#pragma unroll
            for (uint32_t s = 0; s < kSub; ++s)
#pragma unroll
                for (uint32_t r = 0; r < kRanks; ++r)
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) {
                        const uint32_t row = kTile * s + 4 * q + e;
                        if (mine >> row & 1u && 16 * r + c < g.rank)
                            j.part[(split * g.tokens + t0 + row) * g.rank + 16 * r + c] =
                                acc[s][r][e];
                    }
        } else {
            __syncthreads();
#pragma unroll
            for (uint32_t r = 0; r < kRanks; ++r)
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                    red[(wave * kTile + 4 * q + e) * (16 * kRanks) + 16 * r + c] = acc[0][r][e];
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < kTile * 16 * kRanks; i += kThreads) {
                const uint32_t row = i / (16 * kRanks), r = i % (16 * kRanks);
                if (!(mine >> row & 1u) || r >= g.rank) continue;
                float s = 0.0f;
                for (uint32_t v = 0; v < kWaves; ++v) s += red[v * kTile * 16 * kRanks + i];
                j.part[(split * g.tokens + t0 + row) * g.rank + r] = s;
            }
        }
    });
}

template <class T, uint32_t kRanks, bool kWide>
__global__ __launch_bounds__(kThreads) void lora_shrink_kernel(ShrinkArgs g) {
    __shared__ float red[kWide ? 1 : kWaves * kTile * 16 * kRanks];
    constexpr uint32_t kTiles = wide_tiles(16 * kRanks, T::kVec == 4);
    if (blockIdx.y < g.job[0].splits)
        shrink<T, kRanks, kWide, kTiles>(g, g.job[0], blockIdx.y, red);
    else
        shrink<BF16, kRanks, kWide, kTiles>(g, g.job[1], blockIdx.y - g.job[0].splits, red);
}

// ---------------------------------------------------------------------- expand
// out[t][c] = base[t][c] + sum_r low[t][r] w[i][c][r], low the sum of the parts
// times scale[i].
struct ExpandArgs {
    const float *part;
    const float *scale;
    const uint16_t *terms;  // low as three terms, tokens x rank each
    const uint16_t *w;      // n_adapters x len x rank
    const int32_t *adapter;
    const void *base;
    void *out;
    uint64_t tokens, base_stride, out_stride;
    uint32_t len, rank, n_adapters, splits, blocks;  // blocks: of 256 columns
};

__device__ void wave_lds_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// kSteps products of 32 ranks a term; 0: up to 16 ranks, where one product holds two
// terms.  A BF16 out takes all three too: where base and the adapter's part cancel,
// its own rounding hides nothing.
template <class T, uint32_t kSteps, uint32_t kTiles>
__global__ __launch_bounds__(kThreads) void lora_expand_kernel(ExpandArgs g) {
    constexpr uint32_t kFrags = kSteps ? kSteps : 1, kCols = 64, kRow = kCols + 4;
    constexpr uint32_t kLanes = kCols / T::kVec;  // lanes that share a row of base and out
    constexpr uint32_t kTrips = kTile * kLanes / 64;
    __shared__ float tile[kWaves][kTile * kRow];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, q = lane >> 4;
    float *const mytile = tile[wave];
    const uint32_t n0 = (blockIdx.x % g.blocks * kWaves + wave) * kCols;
    const uint64_t group = blockIdx.x / g.blocks;
    if (n0 >= g.len) return;  // no barrier of the workgroup below
    const uint32_t col = n0 + T::kVec * (lane % kLanes);
    const auto *base = static_cast<const typename T::raw *>(g.base);
    auto *out = static_cast<typename T::raw *>(g.out);
    int32_t loaded = -1;
    uint4 w[4][kFrags];
    static_assert(kTiles * kTile <= 64, "a lane a token");
    const int32_t ids =
        adapter_of(g.adapter, group * kTiles * kTile + lane, g.tokens, g.n_adapters);
#pragma unroll 1
    for (uint32_t s = 0; s < kTiles; ++s) {
        const uint64_t t0 = (group * kTiles + s) * kTile;
        if (t0 >= g.tokens) return;
        const int32_t id = __shfl(ids, kTile * s + c);
        each_adapter<kTile>(id, -1, [&](int32_t a, uint64_t mine) {
            uint4 held[kTrips];
#pragma unroll
            for (uint32_t i = 0; i < kTrips; ++i) {
                const uint32_t row = i * (64 / kLanes) + lane / kLanes;
                held[i] = zero4();
                if (base && (mine >> row & 1u) && col < g.len)
                    held[i] =
                        *reinterpret_cast<const uint4 *>(base + (t0 + row) * g.base_stride + col);
            }
            if (a >= 0) {
                if (a != loaded) {
                    loaded = a;
                    const uint16_t *wa = g.w + static_cast<uint64_t>(a) * g.len * g.rank;
#pragma unroll
                    for (uint32_t f = 0; f < 4; ++f)
#pragma unroll
                        for (uint32_t k = 0; k < kFrags; ++k) {
                            const uint32_t r = kSteps ? 32 * k + 8 * q : 8 * (q & 1u);
                            const uint32_t n = min(n0 + 16 * f + c, g.len - 1);
                            w[f][k] = r < g.rank ? *reinterpret_cast<const uint4 *>(
                                                       wa + static_cast<uint64_t>(n) * g.rank + r)
                                                 : zero4();
                        }
                }
                constexpr uint32_t kProducts = kSteps ? kTerms : 2;
                uint4 t[kProducts][kFrags];
#pragma unroll
                for (uint32_t k = 0; k < kFrags; ++k)
#pragma unroll
                    for (uint32_t i = 0; i < kProducts; ++i) {
                        const uint32_t r = kSteps ? 32 * k + 8 * q : 8 * (q & 1u);
                        // up to 16 ranks lane groups 2 and 3 hold the next term
                        const uint32_t term = kSteps ? i : 2 * i + q / 2;
                        const bool in = r < g.rank && (mine >> c & 1u) && term < kTerms;
                        t[i][k] = in ? *reinterpret_cast<const uint4 *>(
                                           g.terms + (term * g.tokens + t0 + c) * g.rank + r)
                                     : zero4();
                    }
                // column 16f + 4q + e of token c
#pragma unroll
                for (uint32_t f = 0; f < 4; ++f) {
                    f32x4 acc{0, 0, 0, 0};
#pragma unroll
                    for (uint32_t k = 0; k < kFrags; ++k)
#pragma unroll
                        for (uint32_t i = 0; i < kProducts; ++i)
                            acc = mfma(w[f][k], t[i][k], acc);
                    *reinterpret_cast<f32x4 *>(mytile + c * kRow + 16 * f + 4 * q) = acc;
                }
                wave_lds_sync();
            }
#pragma unroll
            for (uint32_t i = 0; i < kTrips; ++i) {
                const uint32_t row = i * (64 / kLanes) + lane / kLanes;
                typename T::raw o[T::kVec];
                const float *d = mytile + row * kRow + T::kVec * (lane % kLanes);
#pragma unroll
                for (uint32_t e = 0; e < T::kVec; e += 4) {
                    const f32x4 v =
                        a >= 0 ? *reinterpret_cast<const f32x4 *>(d + e) : f32x4{0, 0, 0, 0};
#pragma unroll
                    for (uint32_t k = 0; k < 4; ++k)
                        o[e + k] = T::store(T::get(held[i], e + k) + v[k]);
                }
                if ((mine >> row & 1u) && col < g.len)
                    *reinterpret_cast<uint4 *>(out + (t0 + row) * g.out_stride + col) =
                        a >= 0 ? __builtin_bit_cast(uint4, o) : held[i];
            }
            wave_lds_sync();
        });
    }
}

// The same for few tokens, a thread a column of one token: no tile to fill, no
// terms to prepare, and no more than two loads after one another.
template <class T>
__global__ __launch_bounds__(kThreads) void lora_expand_few_kernel(ExpandArgs g) {
    __shared__ float low[DF11_MAX_RANK];
    const uint64_t t = blockIdx.y;
    const int32_t a = adapter_of(g.adapter, t, g.tokens, g.n_adapters);
    const uint32_t col = blockIdx.x * kThreads + threadIdx.x;
    const bool in = col < g.len;
    float v = 0.0f;
    if (in && g.base)
        v = T::load(static_cast<const typename T::raw *>(g.base)[t * g.base_stride + col]);
    if (a >= 0) {
        if (threadIdx.x < g.rank) {
            float s = 0.0f;
#pragma unroll 4
            for (uint32_t p = 0; p < g.splits; ++p)
                s += g.part[(p * g.tokens + t) * g.rank + threadIdx.x];
            low[threadIdx.x] = s * (g.scale ? g.scale[a] : 1.0f);
        }
        __syncthreads();
        if (in) {
            const uint16_t *w = g.w + (static_cast<uint64_t>(a) * g.len + col) * g.rank;
            float d = 0.0f;
#pragma unroll 2
            for (uint32_t r = 0; r < g.rank; r += 8) {
                const uint4 q = *reinterpret_cast<const uint4 *>(w + r);
#pragma unroll
                for (uint32_t e = 0; e < 8; ++e) d = fmaf(low[r + e], BF16::get(q, e), d);
            }
            v += d;
        }
    }
    if (in) static_cast<typename T::raw *>(g.out)[t * g.out_stride + col] = T::store(v);
}

// --------------------------------------------------------------- the gradients
// to[i][r][c] = from[i][c][r], 64 c a workgroup; two matrices, along gridDim.y.
struct TransposeJob {
    const uint16_t *from;
    uint16_t *to;
    uint32_t rows, cols;  // of `from`
};
struct TransposeArgs {
    TransposeJob job[2];
};

__global__ __launch_bounds__(kThreads) void lora_transpose_kernel(TransposeArgs g) {
    constexpr uint32_t kSide = 64, kRow = kSide + 2;
    __shared__ uint16_t tile[kSide * kRow];
    const TransposeJob j = g.job[blockIdx.y];
    const uint32_t across = (j.cols + kSide - 1) / kSide, down = (j.rows + kSide - 1) / kSide;
    if (blockIdx.x >= across * down) return;
    const uint32_t r0 = blockIdx.x / across * kSide, c0 = blockIdx.x % across * kSide;
    const uint64_t at = uint64_t{blockIdx.z} * j.rows * j.cols;
    // eight values a load and a store: both sides are multiples of 8
    uint4 v[2];
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t r = threadIdx.x / 8 + 32 * i, c = threadIdx.x % 8 * 8;
        if (r0 + r < j.rows && c0 + c < j.cols)
            v[i] = *reinterpret_cast<const uint4 *>(
                j.from + at + static_cast<uint64_t>(r0 + r) * j.cols + c0 + c);
    }
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t r = threadIdx.x / 8 + 32 * i, c = threadIdx.x % 8 * 8;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            tile[(c + e) * kRow + r] =
                static_cast<uint16_t>(F32::word(v[i], e / 2) >> 16 * (e & 1u));
    }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t c = threadIdx.x / 8 + 32 * i, r = threadIdx.x % 8 * 8;
        uint32_t w[4];
        for (uint32_t e = 0; e < 4; ++e)
            w[e] = tile[c * kRow + r + 2 * e] |
                   static_cast<uint32_t>(tile[c * kRow + r + 2 * e + 1]) << 16;
        if (r0 + r < j.rows && c0 + c < j.cols)
            *reinterpret_cast<uint4 *>(j.to + at + static_cast<uint64_t>(c0 + c) * j.rows + r0 +
                                       r) = uint4{w[0], w[1], w[2], w[3]};
    }
}

// u and v, their parts added, times the scale, as three BF16 terms each: tokens x
// rank for the expand kernel, and rank x `padded` tokens for the gradients (0 for
// tokens without an adapter and past the last one).
struct PrepareJob {
    const float *part;
    uint16_t *rows, *ranks;  // the first terms, the others behind them; either may be null
    uint32_t splits;
};
struct PrepareArgs {
    PrepareJob job[2];
    const float *scale;
    const int32_t *adapter;
    uint64_t tokens, padded;
    uint32_t rank, n_adapters;
};

// Writes the terms of four values, `apart` values from each other.
__device__ void put4(float4 v, uint16_t *to, uint64_t apart) {
    const float x[8] = {v.x, v.y, v.z, v.w, 0, 0, 0, 0};
    uint4 t[kTerms];
    split8(x, t);
#pragma unroll
    for (uint32_t i = 0; i < kTerms; ++i)
        *reinterpret_cast<uint2 *>(to + i * apart) = uint2{t[i].x, t[i].y};
}

__global__ __launch_bounds__(kThreads) void lora_prepare_kernel(PrepareArgs g) {
    constexpr uint32_t kTokens = 32;
    __shared__ float tile[kTokens][DF11_MAX_RANK + 1];
    const uint64_t t0 = uint64_t{blockIdx.x} * kTokens;
    const PrepareJob j = g.job[blockIdx.y];
    const uint32_t quads = g.rank / 4;
    for (uint32_t i = threadIdx.x; i < kTokens * quads; i += kThreads) {
        const uint32_t row = i / quads, r = i % quads * 4;
        const int32_t a = adapter_of(g.adapter, t0 + row, g.tokens, g.n_adapters);
        float4 s{0, 0, 0, 0};
        if (a >= 0) {
            const float scale = g.scale ? g.scale[a] : 1.0f;
#pragma unroll 4
            for (uint32_t p = 0; p < j.splits; ++p) {
                const float4 v = *reinterpret_cast<const float4 *>(
                    j.part + (p * g.tokens + t0 + row) * g.rank + r);
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
            s.x *= scale, s.y *= scale, s.z *= scale, s.w *= scale;
        }
        if (j.rows && a >= -1) put4(s, j.rows + (t0 + row) * g.rank + r, g.tokens * g.rank);
        tile[row][r] = s.x, tile[row][r + 1] = s.y, tile[row][r + 2] = s.z, tile[row][r + 3] = s.w;
    }
    if (!j.ranks) return;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kTokens / 4 * g.rank; i += kThreads) {
        const uint32_t r = i / (kTokens / 4), row = i % (kTokens / 4) * 4;
        put4(float4{tile[row][r], tile[row + 1][r], tile[row + 2][r], tile[row + 3][r]},
             j.ranks + r * g.padded + t0 + row, g.rank * g.padded);
    }
}

// d[i][...] = sum over the chunk's tokens t of i: m[t][c] w[t][r]
struct OuterJob {
    const void *m;
    const uint16_t *terms;  // three terms of w, each rank x padded
    float *d;               // n_adapters x len x rank, or rank x len: a chunk's
    uint64_t stride, chunk_floats;
    uint32_t len, blocks;
    bool rank_rows;  // d is rank x len
};
struct OuterArgs {
    OuterJob job[2];
    const int32_t *adapter;
    uint32_t *present;  // chunks x n_adapters; null: one chunk, straight into d
    uint64_t tokens, padded, per;  // per: tokens of a chunk, a multiple of 32
    uint32_t rank, n_adapters;
};

constexpr uint32_t kScan = 4096;  // tokens whose adapters are looked at together

// The terms of some tokens in LDS, a row per rank: 8 values more keep the 16 lanes
// that read 16 bytes of 16 rows apart.  128 tokens up to rank 64, 52 KB, so that
// three workgroups of rank 64 fit a CU.
template <uint32_t kRanks>
constexpr uint32_t kPiece = kRanks > 4 ? 64 : 128;
template <uint32_t kRanks>
constexpr uint32_t kPieceRow = kPiece<kRanks> + 8;

template <class T, uint32_t kRanks>
__device__ void outer(const OuterArgs &g, const OuterJob &j, uint32_t block, uint32_t *member,
                      uint16_t *terms) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, c = lane & 15u, q = lane >> 4;
    const int32_t a = blockIdx.z;
    const uint32_t c0 = (block * kWaves + wave) * 64;
    // lane group q takes tokens 8q..8q+7 of a step, lane c of it columns 4c..4c+3
    const uint32_t col = min(c0 + 4 * c, j.len - 4);
    const auto *m = static_cast<const typename T::raw *>(j.m);
    const uint64_t from = uint64_t{blockIdx.y} * g.per, to = std::min(g.tokens, from + g.per);
    constexpr uint32_t kPieceSteps = kPiece<kRanks> / 32;
    constexpr uint32_t kTermSize = 16 * kRanks * kPieceRow<kRanks>;
    f32x4 acc[4][kRanks];
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e)
#pragma unroll
        for (uint32_t r = 0; r < kRanks; ++r) acc[e][r] = f32x4{0, 0, 0, 0};
    bool some = false;
    for (uint64_t s0 = from; s0 < to; s0 += kScan) {
        // a bit for each token: is it this adapter's
        __syncthreads();
        const uint32_t scan = static_cast<uint32_t>(std::min<uint64_t>(kScan, to - s0));
        for (uint32_t i = threadIdx.x; i - lane < scan; i += kThreads) {
            const uint64_t all = __ballot(i < scan && g.adapter[s0 + min(i, scan - 1)] == a);
            if (lane < 2) member[i / 64 * 2 + lane] = static_cast<uint32_t>(all >> (32 * lane));
        }
        __syncthreads();
        const uint32_t steps = (scan + 31) / 32;
        using Row = typename std::conditional<T::kVec == 4, uint4, uint2>::type;
        // the steps that hold tokens of this adapter, with the next one's rows under way
        const auto from_step = [&](uint32_t s) {
            while (s < steps && !__builtin_amdgcn_readfirstlane(member[s])) ++s;
            return s;
        };
        const auto load = [&](uint32_t s, Row *row) {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const uint64_t t = std::min(s0 + 32 * s + 8 * q + i, g.tokens - 1);
                row[i] = *reinterpret_cast<const Row *>(m + t * j.stride + col);
            }
        };
        uint32_t s = from_step(0), piece = ~0u;
        Row ahead[8];
        if (s < steps) load(s, ahead);
        while (s < steps) {
            const uint32_t bits = __builtin_amdgcn_readfirstlane(member[s]), now = s;
            some = true;
            const uint32_t ours = bits >> (8 * q) & 0xFFu;
            // the terms of the step's piece: every wave comes here for the same steps
            if (now / kPieceSteps != piece) {
                piece = now / kPieceSteps;
                const uint64_t p0 = s0 + piece * kPiece<kRanks>;
                __syncthreads();
                constexpr uint32_t kEach = kPiece<kRanks> / 8;  // loads of a row
                constexpr uint32_t kLoads = kTerms * 16 * kRanks * kEach / kThreads, kBatch = 6;
                static_assert(kLoads % kBatch == 0 || kLoads < kBatch, "whole batches");
                // a batch of loads under way at a time; rows past the rank repeat the last
                // one, which is never multiplied into a rank that is kept
#pragma unroll
                for (uint32_t b = 0; b < kLoads; b += kBatch) {
                    uint4 v[kBatch];
#pragma unroll
                    for (uint32_t k = 0; k < kBatch && b + k < kLoads; ++k) {
                        const uint32_t i = (b + k) * kThreads + threadIdx.x, row = i / kEach;
                        const uint32_t term = row / (16 * kRanks), r = row % (16 * kRanks);
                        const uint64_t at = std::min<uint64_t>(p0 + i % kEach * 8, g.padded - 8);
                        v[k] = *reinterpret_cast<const uint4 *>(
                            j.terms + (term * g.rank + min(r, g.rank - 1)) * g.padded + at);
                    }
#pragma unroll
                    for (uint32_t k = 0; k < kBatch && b + k < kLoads; ++k) {
                        const uint32_t i = (b + k) * kThreads + threadIdx.x, row = i / kEach;
                        *reinterpret_cast<uint4 *>(terms + row * kPieceRow<kRanks> +
                                                   i % kEach * 8) = v[k];
                    }
                }
                __syncthreads();
            }
            Row row[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) row[i] = ahead[i];
            s = from_step(now + 1);
            if (s < steps) load(s, ahead);
            uint32_t keep[4] = {~0u, ~0u, ~0u, ~0u};
            if (bits != ~0u) {
                // other adapters' tokens: whatever they hold must not count
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (!(ours >> i & 1u)) row[i] = Row{};
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    keep[i] = (ours >> (2 * i) & 1u ? 0xFFFFu : 0u) |
                              (ours >> (2 * i + 1) & 1u ? 0xFFFF0000u : 0u);
            }
            // column 4c + e of the lane's eight tokens
            const auto w_term = [&](uint32_t r, uint32_t i) {
                const uint32_t at =
                    (16 * r + c) * kPieceRow<kRanks> + now % kPieceSteps * 32 + 8 * q;
                uint4 w = *reinterpret_cast<const uint4 *>(terms + i * kTermSize + at);
                w.x &= keep[0], w.y &= keep[1], w.z &= keep[2], w.w &= keep[3];
                return w;
            };
            if constexpr (T::kVec == 4) {
                // a column's terms at a time: four columns' do not fit the registers
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) {
                    float v[8];
                    uint4 t[kTerms];
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) v[i] = F32::get(row[i], e);
                    split8(v, t);
#pragma unroll
                    for (uint32_t r = 0; r < kRanks; ++r)
#pragma unroll
                        for (uint32_t i = 0; i < kTerms; ++i) {
                            const uint4 w = w_term(r, i);
                            // products of 2^-24 and less of the whole are left out
#pragma unroll
                            for (uint32_t p = 0; p + i < kTerms; ++p)
                                acc[e][r] = mfma(t[p], w, acc[e][r]);
                        }
                }
            } else {
                uint4 t[4];
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e) {
                    uint32_t p[4];
                    const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        const uint32_t x = e < 2 ? row[2 * i].x : row[2 * i].y;
                        const uint32_t y = e < 2 ? row[2 * i + 1].x : row[2 * i + 1].y;
                        p[i] = __builtin_amdgcn_perm(y, x, pick);
                    }
                    t[e] = uint4{p[0], p[1], p[2], p[3]};
                }
#pragma unroll
                for (uint32_t r = 0; r < kRanks; ++r)
#pragma unroll
                    for (uint32_t i = 0; i < kTerms; ++i) {
                        const uint4 w = w_term(r, i);
#pragma unroll
                        for (uint32_t e = 0; e < 4; ++e) acc[e][r] = mfma(t[e], w, acc[e][r]);
                    }
            }
        }
    }
    if (g.present) {
        if (blockIdx.x == 0 && threadIdx.x == 0)
            g.present[blockIdx.y * g.n_adapters + a] = some ? 1u : 0u;
        if (!some) return;
    }
    // acc[e][r][k]: column 4 (4q + k) + e, rank 16r + c
    float *d = j.d + blockIdx.y * j.chunk_floats + static_cast<uint64_t>(a) * j.len * g.rank;
#pragma unroll
    for (uint32_t r = 0; r < kRanks; ++r) {
        const uint32_t rank = 16 * r + c;
        if (rank >= g.rank) continue;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t n = c0 + 16 * q + 4 * k;
            if (n >= j.len) continue;
            if (j.rank_rows) {
                *reinterpret_cast<f32x4 *>(d + static_cast<uint64_t>(rank) * j.len + n) =
                    f32x4{acc[0][r][k], acc[1][r][k], acc[2][r][k], acc[3][r][k]};
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                    d[static_cast<uint64_t>(n + e) * g.rank + rank] = acc[e][r][k];
            }
        }
    }
}

// Waves on a SIMD: as many as the registers hold without spilling.
template <class T>
constexpr int outer_waves(uint32_t ranks) {
    if (T::kVec == 4) return ranks == 1 ? 3 : ranks == 2 ? 2 : 1;
    return ranks <= 2 ? 3 : ranks <= 4 ? 2 : 1;
}

template <class T, uint32_t kRanks>
__global__ __launch_bounds__(kThreads, outer_waves<T>(kRanks)) void lora_outer_kernel(OuterArgs g) {
    __shared__ uint32_t member[kScan / 32];
    __shared__ __align__(16) uint16_t terms[kTerms * 16 * kRanks * kPieceRow<kRanks>];
    if (blockIdx.x < g.job[0].blocks)
        outer<T, kRanks>(g, g.job[0], blockIdx.x, member, terms);
    else
        outer<BF16, kRanks>(g, g.job[1], blockIdx.x - g.job[0].blocks, member, terms);
}

// d = the chunks' sums in order; 0 for an adapter without tokens.
struct JoinArgs {
    const float *from[2];
    float *to[2];
    const uint32_t *present;
    uint64_t each[2], all[2];  // floats of an adapter, of all of them
    uint32_t chunks, n_adapters;
};

__global__ __launch_bounds__(kThreads) void lora_join_kernel(JoinArgs g) {
    const uint32_t job = blockIdx.y;
    for (uint64_t i = (uint64_t{blockIdx.x} * kThreads + threadIdx.x) * 4; i < g.all[job];
         i += uint64_t{gridDim.x} * kThreads * 4) {
        const uint32_t a = static_cast<uint32_t>(i / g.each[job]);
        f32x4 s{0, 0, 0, 0};
        for (uint32_t k = 0; k < g.chunks; ++k)
            if (g.present[k * g.n_adapters + a])
                s += *reinterpret_cast<const f32x4 *>(g.from[job] + k * g.all[job] + i);
        *reinterpret_cast<f32x4 *>(g.to[job] + i) = s;
    }
}

// Zeros, where there are no tokens: a kernel, which a graph may record.
__global__ __launch_bounds__(kThreads) void lora_zero_kernel(float *p, uint64_t n) {
    for (uint64_t i = uint64_t{blockIdx.x} * kThreads + threadIdx.x; i < n;
         i += uint64_t{gridDim.x} * kThreads)
        p[i] = 0.0f;
}

// ---- host side
uint64_t up(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }

int check_shapes(uint64_t tokens, uint32_t cols, uint32_t rows, uint32_t rank,
                 uint32_t n_adapters) {
    if (!cols || !rows || !rank || !n_adapters) return DF11_E_INVALID_ARG;
    if (cols % 64 || rows % 16 || rank % 8 || rank > DF11_MAX_RANK || tokens > (1ull << 24) ||
        n_adapters > 65535u || cols > (1u << 23) || rows > (1u << 23))
        return DF11_E_UNSUPPORTED;
    // `expand` over out or dx: a launch holds 2^32 threads
    const uint64_t blocks = (std::max(rows, cols) + 255) / 256;
    const uint64_t groups = (tokens + kTile * kManyTiles - 1) / (kTile * kManyTiles);
    return groups * blocks > 0xFFFFFFFFull / kThreads ? DF11_E_UNSUPPORTED : DF11_OK;
}

int check_rows(const void *p, uint64_t stride, uint32_t len, uint64_t tokens, uint32_t bytes) {
    if (!p || misaligned(p, 16)) return DF11_E_INVALID_ARG;
    if (tokens > 1 && (stride < len || stride > (1ull << 40) || stride * bytes % 16))
        return DF11_E_INVALID_ARG;
    return DF11_OK;
}

int check_common(const uint16_t *x, uint64_t x_stride, uint64_t tokens, uint32_t cols,
                 const uint16_t *a, const uint16_t *b, const float *scale,
                 const int32_t *adapter) {
    const int rc = check_rows(x, x_stride, cols, tokens, 2);
    if (rc) return rc;
    if (!a || !b || !adapter || misaligned(a, 16) || misaligned(b, 16) || misaligned(scale, 4) ||
        misaligned(adapter, 4))
        return DF11_E_INVALID_ARG;
    return DF11_OK;
}

int check_workspace(const void *ws, uint64_t have, uint64_t need) {
    if (have < need) return DF11_E_BUFFER_TOO_SMALL;
    return need && (!ws || misaligned(ws, 16)) ? DF11_E_INVALID_ARG : DF11_OK;
}

// Whether `shrink` gives each wave tiles of its own.  Its workgroups are fewer and
// take four times as long, but read w for many more tokens at once: where they are
// many, or where a read of w for every 16 tokens would come to more than 64 MB.
// Us, wide and not: 574 tokens x (14336 + 4096) columns, rank 24, fp32 31.6 and
// 19.6; 1604 x 4096, rank 24 15.8 and 9.9; 6001 x 4096, rank 16 19.8 and 19.7; 8192
// x (4096 + 4096), rank 64 62 and 85; 1024 x 128,256, rank 16, fp32 111 and 131.
bool is_wide(uint64_t tokens, uint32_t rank, uint64_t columns) {
    if (tokens <= kFewTokens) return false;
    const uint64_t wgs = tokens / wide_tokens(rank, false) * std::min<uint64_t>(32, columns / 512);
    return wgs >= 512 || tokens / kTile * rank * columns * 2 > (64ull << 20);
}

// Columns of a split and how many splits: about 1024 workgroups in all, each of
// at least 512 columns, at most 32 sums to add.
void split_columns(uint32_t len, uint64_t tokens, uint32_t rank, uint32_t n_adapters, bool wide,
                   ShrinkJob *j) {
    uint64_t wgs = (tokens + kTile - 1) / kTile;
    if (tokens <= kFewTokens) wgs *= std::min<uint64_t>({16, n_adapters, tokens});
    if (wide) wgs = (tokens + wide_tokens(rank, false) - 1) / wide_tokens(rank, false);
    const uint32_t most = std::min(32u, std::max(1u, len / 512));
    const uint32_t want = static_cast<uint32_t>(std::min<uint64_t>(most, (1024 + wgs - 1) / wgs));
    j->len = len;
    j->per = static_cast<uint32_t>(up((len + want - 1) / want, 256));
    j->splits = (len + j->per - 1) / j->per;
}

// Tokens of a chunk of the gradients: about 512 workgroups, chunks of at least 128
// tokens, and at most 128 MB of partial sums.
uint64_t chunk_tokens(uint64_t tokens, uint32_t cols, uint32_t rows, uint32_t rank,
                      uint32_t n_adapters) {
    const uint64_t blocks = (cols + 255) / 256 + (rows + 255) / 256;
    const uint64_t each = 4ull * n_adapters * rank * (uint64_t{cols} + rows);
    uint64_t chunks = std::min((512 + blocks - 1) / blocks, (tokens + 127) / 128);
    chunks = std::max<uint64_t>(1, std::min<uint64_t>(chunks, (128ull << 20) / each));
    return up((tokens + chunks - 1) / chunks, 32);
}

template <class T, bool kWide>
int launch_shrink(const ShrinkArgs &s, hipStream_t stream) {
    const uint64_t tile = kWide ? wide_tokens(s.rank, T::kVec == 4) : kTile;
    const dim3 grid((s.tokens + tile - 1) / tile, s.job[0].splits + s.job[1].splits,
                    s.tokens <= kFewTokens ? std::min<uint64_t>({16, s.n_adapters, s.tokens}) : 1);
    const dim3 block(kThreads);
    const uint32_t ranks = (s.rank + 15) / 16;
    if (ranks == 1)
        hipLaunchKernelGGL((lora_shrink_kernel<T, 1, kWide>), grid, block, 0, stream, s);
    else if (ranks == 2)
        hipLaunchKernelGGL((lora_shrink_kernel<T, 2, kWide>), grid, block, 0, stream, s);
    else if (ranks <= 4)
        hipLaunchKernelGGL((lora_shrink_kernel<T, 4, kWide>), grid, block, 0, stream, s);
    else
        hipLaunchKernelGGL((lora_shrink_kernel<T, 8, kWide>), grid, block, 0, stream, s);
    return launched();
}

int launch_shrink(const ShrinkArgs &s, uint32_t dtype, bool wide, hipStream_t stream) {
    if (wide)
        return dtype == DF11_F32 ? launch_shrink<F32, true>(s, stream)
                                 : launch_shrink<BF16, true>(s, stream);
    return dtype == DF11_F32 ? launch_shrink<F32, false>(s, stream)
                             : launch_shrink<BF16, false>(s, stream);
}

int launch_expand_few(const ExpandArgs &e, uint32_t dtype, hipStream_t stream) {
    const dim3 grid((e.len + kThreads - 1) / kThreads, e.tokens), block(kThreads);
    if (dtype == DF11_F32)
        hipLaunchKernelGGL(lora_expand_few_kernel<F32>, grid, block, 0, stream, e);
    else
        hipLaunchKernelGGL(lora_expand_few_kernel<BF16>, grid, block, 0, stream, e);
    return launched();
}

template <class T, uint32_t kTiles>
int launch_expand(ExpandArgs e, hipStream_t stream) {
    e.blocks = (e.len + 255) / 256;
    const uint64_t wgs = (e.tokens + kTile * kTiles - 1) / (kTile * kTiles) * e.blocks;
    const dim3 grid(wgs, 1,
                    kTiles == 1 ? std::min<uint64_t>({16, e.n_adapters + 1ull, e.tokens}) : 1);
    const dim3 block(kThreads);
    if (e.rank <= 16)
        hipLaunchKernelGGL((lora_expand_kernel<T, 0, kTiles>), grid, block, 0, stream, e);
    else if (e.rank <= 32)
        hipLaunchKernelGGL((lora_expand_kernel<T, 1, kTiles>), grid, block, 0, stream, e);
    else if (e.rank <= 64)
        hipLaunchKernelGGL((lora_expand_kernel<T, 2, kTiles>), grid, block, 0, stream, e);
    else
        hipLaunchKernelGGL((lora_expand_kernel<T, 4, kTiles>), grid, block, 0, stream, e);
    return launched();
}

int launch_expand(const ExpandArgs &e, uint32_t dtype, hipStream_t stream) {
    if (e.tokens <= kFewTokens)
        return dtype == DF11_F32 ? launch_expand<F32, 1>(e, stream)
                                 : launch_expand<BF16, 1>(e, stream);
    return dtype == DF11_F32 ? launch_expand<F32, kManyTiles>(e, stream)
                             : launch_expand<BF16, kManyTiles>(e, stream);
}

template <class T>
int launch_outer(const OuterArgs &o, uint64_t chunks, hipStream_t stream) {
    const dim3 grid(o.job[0].blocks + o.job[1].blocks, chunks, o.n_adapters), block(kThreads);
    const uint32_t ranks = (o.rank + 15) / 16;
    if (ranks == 1)
        hipLaunchKernelGGL((lora_outer_kernel<T, 1>), grid, block, 0, stream, o);
    else if (ranks == 2)
        hipLaunchKernelGGL((lora_outer_kernel<T, 2>), grid, block, 0, stream, o);
    else if (ranks <= 4)
        hipLaunchKernelGGL((lora_outer_kernel<T, 4>), grid, block, 0, stream, o);
    else
        hipLaunchKernelGGL((lora_outer_kernel<T, 8>), grid, block, 0, stream, o);
    return launched();
}

// The backward pass's workspace, in bytes from its start.
struct Space {
    uint64_t bt, at, u, v, rows, terms, present, db, da, bytes;
    uint64_t padded, per, chunks;
    ShrinkJob ju, jv;
    bool wide;
};
Space space_of(uint64_t tokens, uint32_t cols, uint32_t rows, uint32_t rank, uint32_t n_adapters) {
    Space s{};
    s.padded = up(tokens, 32);
    s.wide = is_wide(tokens, rank, uint64_t{rows} + cols);
    split_columns(rows, std::max<uint64_t>(tokens, 1), rank, n_adapters, s.wide, &s.ju);
    split_columns(cols, std::max<uint64_t>(tokens, 1), rank, n_adapters, s.wide, &s.jv);
    s.per = std::max<uint64_t>(32, chunk_tokens(tokens, cols, rows, rank, n_adapters));
    s.chunks = std::max<uint64_t>(1, (tokens + s.per - 1) / s.per);
    uint64_t at = 0;
    const auto take = [&](uint64_t bytes) {
        const uint64_t from = at;
        at += up(bytes, 256);
        return from;
    };
    s.bt = take(2ull * n_adapters * rows * rank);
    s.at = take(2ull * n_adapters * cols * rank);
    s.u = take(4ull * s.ju.splits * tokens * rank);
    s.v = take(4ull * s.jv.splits * tokens * rank);
    s.rows = take(2ull * kTerms * rank * tokens);
    s.terms = take(4ull * kTerms * rank * s.padded);
    s.present = take(4ull * s.chunks * n_adapters);
    s.db = take(s.chunks > 1 ? 4ull * s.chunks * n_adapters * rows * rank : 0);
    s.da = take(s.chunks > 1 ? 4ull * s.chunks * n_adapters * cols * rank : 0);
    s.bytes = at;
    return s;
}

}  // namespace

extern "C" {

int df11_lora_workspace_bytes(uint64_t tokens, uint32_t cols, uint32_t rows, uint32_t rank,
                              uint32_t n_adapters, uint64_t *bytes) {
    if (!bytes) return DF11_E_INVALID_ARG;
    const int rc = check_shapes(tokens, cols, rows, rank, n_adapters);
    if (rc) return rc;
    ShrinkJob j{};
    if (tokens)
        split_columns(cols, tokens, rank, n_adapters, is_wide(tokens, rank, cols), &j);
    // the parts, and their sum as three terms where there are more than few values
    *bytes = tokens * rank * (4 * j.splits + (tokens * rank > kFewValues ? 2 * kTerms : 0));
    return DF11_OK;
}

int df11_lora(const uint16_t *x, uint64_t x_stride, uint64_t tokens, uint32_t cols, uint32_t rows,
              uint32_t rank, uint32_t n_adapters, const uint16_t *a, const uint16_t *b,
              const float *scale, const int32_t *adapter, const void *base, uint64_t base_stride,
              void *out, uint64_t out_stride, uint32_t dtype, void *workspace,
              uint64_t workspace_bytes, hipStream_t stream) {
    uint64_t need = 0;
    int rc = df11_lora_workspace_bytes(tokens, cols, rows, rank, n_adapters, &need);
    if (rc) return rc;
    if (dtype > DF11_BF16) return DF11_E_INVALID_ARG;
    if (!tokens) return DF11_OK;
    const uint32_t size = elem_bytes(dtype);
    rc = check_common(x, x_stride, tokens, cols, a, b, scale, adapter);
    if (!rc && base) rc = check_rows(base, base_stride, rows, tokens, size);
    if (!rc) rc = check_rows(out, out_stride, rows, tokens, size);
    if (!rc && base == out && tokens > 1 && base_stride != out_stride) rc = DF11_E_INVALID_ARG;
    if (!rc) rc = check_workspace(workspace, workspace_bytes, need);
    if (rc) return rc;
    ShrinkArgs s{};
    s.job[0].x = x;
    s.job[0].w = a;
    s.job[0].part = static_cast<float *>(workspace);
    s.job[0].stride = x_stride;
    const bool wide = is_wide(tokens, rank, cols);
    split_columns(cols, tokens, rank, n_adapters, wide, &s.job[0]);
    s.adapter = adapter;
    s.tokens = tokens;
    s.rank = rank;
    s.n_adapters = n_adapters;
    if ((rc = launch_shrink(s, DF11_BF16, wide, stream))) return rc;
    const float *part = s.job[0].part;
    auto *terms = reinterpret_cast<uint16_t *>(s.job[0].part + s.job[0].splits * tokens * rank);
    const ExpandArgs e{part, scale, terms, b, adapter, base, out, tokens, base_stride,
                       out_stride, rows, rank, n_adapters, s.job[0].splits, 0};
    if (tokens * rank <= kFewValues) return launch_expand_few(e, dtype, stream);
    const PrepareArgs p{{{part, terms, nullptr, s.job[0].splits}, {}},
                        scale, adapter, tokens, 0, rank, n_adapters};
    hipLaunchKernelGGL(lora_prepare_kernel, dim3((tokens + 31) / 32), dim3(kThreads), 0, stream,
                       p);
    if ((rc = launched())) return rc;
    return launch_expand(e, dtype, stream);
}

int df11_lora_backward_workspace_bytes(uint64_t tokens, uint32_t cols, uint32_t rows,
                                       uint32_t rank, uint32_t n_adapters, uint64_t *bytes) {
    if (!bytes) return DF11_E_INVALID_ARG;
    const int rc = check_shapes(tokens, cols, rows, rank, n_adapters);
    if (rc) return rc;
    *bytes = tokens ? space_of(tokens, cols, rows, rank, n_adapters).bytes : 0;
    return DF11_OK;
}

int df11_lora_backward(const uint16_t *x, uint64_t x_stride, uint64_t tokens, uint32_t cols,
                       uint32_t rows, uint32_t rank, uint32_t n_adapters, const uint16_t *a,
                       const uint16_t *b, const float *scale, const int32_t *adapter,
                       const void *dy, uint64_t dy_stride, uint32_t dy_dtype,
                       const uint16_t *dx_base, uint64_t dx_base_stride, uint16_t *dx,
                       uint64_t dx_stride, float *da, float *db, void *workspace,
                       uint64_t workspace_bytes, hipStream_t stream) {
    uint64_t need = 0;
    int rc = df11_lora_backward_workspace_bytes(tokens, cols, rows, rank, n_adapters, &need);
    if (rc) return rc;
    if (dy_dtype > DF11_BF16 || !da != !db || (!dx && !da)) return DF11_E_INVALID_ARG;
    if (misaligned(da, 16) || misaligned(db, 16)) return DF11_E_INVALID_ARG;
    if (!tokens) {
        if (!da) return DF11_OK;
        hipLaunchKernelGGL(lora_zero_kernel, dim3(256), dim3(kThreads), 0, stream, da,
                           uint64_t{n_adapters} * cols * rank);
        if ((rc = launched())) return rc;
        hipLaunchKernelGGL(lora_zero_kernel, dim3(256), dim3(kThreads), 0, stream, db,
                           uint64_t{n_adapters} * rows * rank);
        return launched();
    }
    rc = check_common(x, x_stride, tokens, cols, a, b, scale, adapter);
    if (!rc) rc = check_rows(dy, dy_stride, rows, tokens, elem_bytes(dy_dtype));
    if (!rc && dx) rc = check_rows(dx, dx_stride, cols, tokens, 2);
    if (!rc && dx_base) rc = check_rows(dx_base, dx_base_stride, cols, tokens, 2);
    if (!rc && dx_base && dx_base == dx && tokens > 1 && dx_base_stride != dx_stride)
        rc = DF11_E_INVALID_ARG;
    if (!rc) rc = check_workspace(workspace, workspace_bytes, need);
    // dA and dB are made of x and dy after dx is written
    if (!rc && da && dx && (dx == x || dx == dy)) rc = DF11_E_INVALID_ARG;
    if (rc) return rc;

    const Space s = space_of(tokens, cols, rows, rank, n_adapters);
    char *ws = static_cast<char *>(workspace);
    auto *bt = reinterpret_cast<uint16_t *>(ws + s.bt);
    auto *at = reinterpret_cast<uint16_t *>(ws + s.at);
    auto *u = reinterpret_cast<float *>(ws + s.u), *v = reinterpret_cast<float *>(ws + s.v);
    auto *terms = reinterpret_cast<uint16_t *>(ws + s.terms);

    const TransposeArgs t{{{b, bt, rows, rank}, {a, at, rank, cols}}};
    const uint32_t sides = (rank + 63) / 64 * ((std::max(rows, cols) + 63) / 64);
    hipLaunchKernelGGL(lora_transpose_kernel, dim3(sides, dx ? 2 : 1, n_adapters), dim3(kThreads),
                       0, stream, t);
    if ((rc = launched())) return rc;

    ShrinkArgs h{};
    h.job[0] = s.ju;
    h.job[0].x = dy;
    h.job[0].w = bt;
    h.job[0].part = u;
    h.job[0].stride = dy_stride;
    if (da) {
        h.job[1] = s.jv;
        h.job[1].x = x;
        h.job[1].w = a;
        h.job[1].part = v;
        h.job[1].stride = x_stride;
    }
    h.adapter = adapter;
    h.tokens = tokens;
    h.rank = rank;
    h.n_adapters = n_adapters;
    if ((rc = launch_shrink(h, dy_dtype, s.wide, stream))) return rc;

    auto *by_row = reinterpret_cast<uint16_t *>(ws + s.rows);
    const PrepareArgs p{{{u, dx ? by_row : nullptr, da ? terms : nullptr, s.ju.splits},
                         {v, nullptr, terms + kTerms * rank * s.padded, s.jv.splits}},
                        scale, adapter, tokens, s.padded, rank, n_adapters};
    hipLaunchKernelGGL(lora_prepare_kernel, dim3(s.padded / 32, da ? 2 : 1), dim3(kThreads), 0,
                       stream, p);
    if ((rc = launched())) return rc;

    if (dx) {
        const ExpandArgs e{u, scale, by_row, at, adapter, dx_base, dx, tokens,
                           dx_base_stride, dx_stride, cols, rank, n_adapters, s.ju.splits, 0};
        if ((rc = launch_expand(e, DF11_BF16, stream))) return rc;
    }
    if (!da) return DF11_OK;

    const bool many = s.chunks > 1;
    auto *present = reinterpret_cast<uint32_t *>(ws + s.present);
    auto *pb = reinterpret_cast<float *>(ws + s.db), *pa = reinterpret_cast<float *>(ws + s.da);
    const uint64_t fb = uint64_t{n_adapters} * rows * rank, fa = uint64_t{n_adapters} * cols * rank;
    // dB takes v, the second pair of terms, and dA takes u, the first
    const OuterArgs o{{{dy, terms + kTerms * rank * s.padded, many ? pb : db, dy_stride, fb, rows,
                        (rows + 255) / 256, false},
                       {x, terms, many ? pa : da, x_stride, fa, cols, (cols + 255) / 256, true}},
                      adapter, many ? present : nullptr, tokens, s.padded, s.per, rank, n_adapters};
    rc = dy_dtype == DF11_F32 ? launch_outer<F32>(o, s.chunks, stream)
                              : launch_outer<BF16>(o, s.chunks, stream);
    if (rc || !many) return rc;
    const JoinArgs j{{pb, pa}, {db, da}, present, {uint64_t{rows} * rank, uint64_t{cols} * rank},
                     {fb, fa}, static_cast<uint32_t>(s.chunks), n_adapters};
    const uint64_t wgs = (std::max(fa, fb) / 4 + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(lora_join_kernel, dim3(std::min<uint64_t>(wgs, 8192), 2), dim3(kThreads), 0,
                       stream, j);
    return launched();
}

}  // extern "C"
