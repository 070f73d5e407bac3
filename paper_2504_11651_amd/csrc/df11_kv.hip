// Appending to a paged cache of keys and values, the position rotation applied on
// the way: the fp32 rows of the q, k and v products are read once, and what
// attention needs of them is written once, rounded once.

#include "df11_kv_common.h"

namespace {

using namespace df11ops;

constexpr uint32_t kThreads = 256;
// 1 / (2 pi) as the sum of two
constexpr double kTurns = 0.15915494309189533577, kTurnsRest = -9.839338337591243e-18;

struct AppendArgs {
    const void *q, *k, *v;
    uint64_t q_stride, k_stride, v_stride;
    const float *inv_freq;
    uint16_t *cache_k, *cache_v, *q_out;
    uint64_t page_k, page_v, out_stride;
    Batch batch;
    uint32_t pages, page_shift, heads, kv_heads, rotary, interleaved;
};

// Eight values as floats, and as they are stored.
template <class S>
__device__ inline void load8(const typename S::raw *p, float (&x)[8]) {
    const uint4 a = load16(p);
    if constexpr (S::kVec == 8) {
        for (uint32_t e = 0; e < 8; e++) x[e] = S::get(a, e);
    } else {
        const uint4 b = load16(p + 4);
        for (uint32_t e = 0; e < 4; e++) x[e] = S::get(a, e), x[4 + e] = S::get(b, e);
    }
}
template <class C>
__device__ inline void store8(uint16_t *p, const float (&x)[8]) {
    uint32_t w[4];
    for (uint32_t e = 0; e < 4; e++)
        w[e] = C::store(x[2 * e]) | static_cast<uint32_t>(C::store(x[2 * e + 1])) << 16;
    store16(p, uint4{w[0], w[1], w[2], w[3]});
}

// A workgroup appends one row.  The angles' cosines and sines are made once for all
// heads and lie in LDS; a thread then takes 16 values at a time that turn together:
// eight and the eight half the rotary part further, or 16 neighbours.  Many rows are bound
// by memory (8191 of 32 + 2 x 8 heads of 128, fp32 to BF16: 57 us, 5.3 TB/s), few by the
// loads after one another (64 rows of 64 + 2 x 8 heads 4.4 us, one row 2.8).
template <class S, class C, uint32_t D>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs a) {
    __shared__ __attribute__((aligned(16))) float turn[2][D / 2];
    const uint32_t row = blockIdx.x;
    const Owner o = owner(a.batch, row);
    if (o.s == ~0u) return;
    const int64_t place = int64_t{a.batch.length[o.s]} - (o.end - row);
    if (threadIdx.x < a.rotary / 2) {
        // Turns of one position with what 53 bits leave out of them; of p of them the whole
        // ones go before anything is rounded (products of 53 bits were off by 10^-8 of a
        // turn at 2^28 and ten times that at 2^32).  What 32 bits then round is a fraction
        // of a turn
        const double f = a.inv_freq[threadIdx.x];
        const double p = static_cast<double>(place + a.batch.prefix_len);
        const double each = f * kTurns, each_rest = fma(f, kTurns, -each) + f * kTurnsRest;
        const double t = fma(p, each, -rint(p * each)) + p * each_rest;
        float s, c;
        sincospif(static_cast<float>(2.0 * t), &s, &c);
        turn[0][threadIdx.x] = c;
        turn[1][threadIdx.x] = s;
    }
    bool keep = place >= 0 && place >> a.page_shift < a.batch.width;
    uint32_t page = 0;
    if (keep) page = a.batch.table[o.s * a.batch.table_stride + (place >> a.page_shift)];
    keep = keep && page < a.pages;
    const uint64_t in_page = (place & ((1 << a.page_shift) - 1)) * D;
    __syncthreads();
    constexpr uint32_t kUnits = D / 16;  // of a head
    const uint32_t units = (a.heads + 2 * a.kv_heads) * kUnits;
    for (uint32_t i = threadIdx.x; i < units; i += kThreads) {
        const uint32_t u = i % kUnits, h = i / kUnits;
        const bool is_q = h < a.heads, is_k = !is_q && h < a.heads + a.kv_heads;
        if (!is_q && !keep) break;
        const bool turns = u * 16 < a.rotary && (is_q || is_k);
        const bool apart = turns && !a.interleaved;
        const uint32_t at = apart ? u * 8 : u * 16;
        const uint32_t next = apart ? at + a.rotary / 2 : at + 8;
        const uint32_t head = is_q ? h : is_k ? h - a.heads : h - a.heads - a.kv_heads;
        const uint64_t stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
        const void *from = is_q ? a.q : is_k ? a.k : a.v;
        const auto *src = static_cast<const typename S::raw *>(from) + row * stride + head * D;
        uint16_t *dst = is_q ? a.q_out + row * a.out_stride + head * D
                             : (is_k ? a.cache_k + page * a.page_k : a.cache_v + page * a.page_v) +
                                   (uint64_t{head * D} << a.page_shift) + in_page;
        float x[8], y[8];
        load8<S>(src + at, x);
        load8<S>(src + next, y);
        if (apart) {
            for (uint32_t e = 0; e < 8; e++) {
                const float c = turn[0][u * 8 + e], s = turn[1][u * 8 + e];
                const float p = x[e], q = y[e];
                x[e] = p * c - q * s;
                y[e] = q * c + p * s;
            }
        } else if (turns) {
            for (uint32_t e = 0; e < 8; e++) {
                const float c = turn[0][u * 8 + e], s = turn[1][u * 8 + e];
                float &p = e < 4 ? x[2 * e] : y[2 * e - 8];
                float &q = e < 4 ? x[2 * e + 1] : y[2 * e - 7];
                const float p0 = p, q0 = q;
                p = p0 * c - q0 * s;
                q = q0 * c + p0 * s;
            }
        }
        store8<C>(dst + at, x);
        store8<C>(dst + next, y);
    }
}

template <class S, class C>
int launch(const AppendArgs &a, uint32_t dim, hipStream_t stream) {
    const dim3 grid(a.batch.rows), block(kThreads);
    if (dim == 128)
        hipLaunchKernelGGL((kv_append_kernel<S, C, 128>), grid, block, 0, stream, a);
    else
        hipLaunchKernelGGL((kv_append_kernel<S, C, 64>), grid, block, 0, stream, a);
    return launched();
}

}  // namespace

extern "C" {

int df11_kv_append(const void *q, uint64_t q_stride, const void *k, uint64_t k_stride,
                   const void *v, uint64_t v_stride, uint32_t dtype, uint64_t tokens,
                   uint32_t heads, const float *inv_freq, uint32_t rotary, uint32_t interleaved,
                   const df11_kv_cache *cache, const df11_kv_batch *batch, void *q_out,
                   uint64_t q_out_stride, hipStream_t stream) {
    int rc = check_cache(cache);
    if (!rc) rc = check_batch(batch);
    if (rc) return rc;
    if (dtype > DF11_F16 || !heads || heads >> 20 || tokens > kMaxSequences ||
        tokens * heads >> 31)
        return DF11_E_INVALID_ARG;
    if (tokens >= kMaxGrid) return DF11_E_UNSUPPORTED;
    if (rotary % 16 || rotary > cache->dim || (rotary && (!inv_freq || misaligned(inv_freq, 4))))
        return DF11_E_INVALID_ARG;
    if (!tokens || !batch->sequences) return DF11_OK;
    const uint64_t q_cols = uint64_t{heads} * cache->dim;
    const uint64_t kv_cols = uint64_t{cache->heads} * cache->dim;
    const uint32_t size = elem_bytes(dtype);
    rc = check_strided(q, q_stride, q_cols, tokens, size);
    if (!rc) rc = check_strided(k, k_stride, kv_cols, tokens, size);
    if (!rc) rc = check_strided(v, v_stride, kv_cols, tokens, size);
    if (!rc) rc = check_strided(q_out, q_out_stride, q_cols, tokens, 2);
    if (!rc && q_out == q && (dtype != cache->dtype || (tokens > 1 && q_stride != q_out_stride)))
        rc = DF11_E_INVALID_ARG;
    if (rc) return rc;
    const AppendArgs a{q, k, v, q_stride, k_stride, v_stride, inv_freq,
                       static_cast<uint16_t *>(cache->k), static_cast<uint16_t *>(cache->v),
                       static_cast<uint16_t *>(q_out), cache->k_stride, cache->v_stride,
                       q_out_stride, device_batch(*batch, tokens), cache->pages,
                       static_cast<uint32_t>(__builtin_ctz(cache->page_size)), heads, cache->heads,
                       rotary, interleaved};
    if (cache->dtype == DF11_BF16)
        return dtype == DF11_F32    ? launch<F32, BF16>(a, cache->dim, stream)
               : dtype == DF11_BF16 ? launch<BF16, BF16>(a, cache->dim, stream)
                                    : launch<F16, BF16>(a, cache->dim, stream);
    return dtype == DF11_F32    ? launch<F32, F16>(a, cache->dim, stream)
           : dtype == DF11_BF16 ? launch<BF16, F16>(a, cache->dim, stream)
                                : launch<F16, F16>(a, cache->dim, stream);
}

}  // extern "C"
