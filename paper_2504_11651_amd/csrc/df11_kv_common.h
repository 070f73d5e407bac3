// The paged cache of keys and values and the batch that uses it: checks of the
// arguments, and on the device which sequence a row belongs to and where its
// tokens lie.
#pragma once

#include "df11_ops_common.h"

namespace df11ops {

constexpr uint32_t kMaxSequences = 1u << 24;
constexpr uint32_t kMaxGrid = 1u << 24;  // times 256 threads: what a launch does not hold

// What the kernels take of a df11_kv_batch; `rows` is the call's.
struct Batch {
    const int32_t *start, *length, *table, *prefix_table;
    uint64_t table_stride;
    uint32_t sequences, width, prefix_pages, prefix_len, rows;
    // start[s], whatever memory holds: a row number of this call
    __device__ uint32_t first(uint32_t s) const {
        return static_cast<uint32_t>(min(max(start[s], 0), static_cast<int32_t>(rows)));
    }
};

// The largest s in [0, n) with f(s) <= x where f never falls; ~0 if none.  The
// wave looks at 64 places at once: one round of loads for 64 sequences, two for
// 4096.  All lanes take part and agree.
template <class F>
__device__ inline uint32_t wave_search(uint32_t n, uint32_t x, F f) {
    const uint32_t lane = threadIdx.x & 63;
    uint32_t lo = 0;
    for (;;) {
        const uint32_t step = (n + 63) / 64;
        const bool in = lane * step < n;
        const uint64_t reached = __ballot(in && f(lo + lane * step) <= x);
        if (!reached) return ~0u;
        const uint32_t at = (__popcll(reached) - 1) * step;
        lo += at;
        if (step == 1) return lo;
        n = min(step, n - at);
    }
}

// The sequence of a row and the row after its last; s = ~0: of none.
struct Owner {
    uint32_t s, end;
};
__device__ inline Owner owner(const Batch &b, uint32_t row) {
    uint32_t s = wave_search(b.sequences, row, [&](uint32_t i) { return b.first(i); });
    s = __builtin_amdgcn_readfirstlane(s);
    if (s == ~0u) return {s, 0};
    const uint32_t end = b.first(s + 1);
    return row < end ? Owner{s, end} : Owner{~0u, 0};
}

inline uint64_t head_values(const df11_kv_cache &c) {
    return uint64_t{c.heads} * c.page_size * c.dim;
}

// The sizes alone: what a workspace's size goes by.
inline int check_cache_sizes(const df11_kv_cache *c) {
    if (!c || !c->heads || (c->dim != 64 && c->dim != 128)) return DF11_E_INVALID_ARG;
    if (c->dtype != DF11_BF16 && c->dtype != DF11_F16) return DF11_E_INVALID_ARG;
    if (c->page_size < DF11_MIN_PAGE || c->page_size > DF11_MAX_PAGE ||
        (c->page_size & (c->page_size - 1)))
        return DF11_E_INVALID_ARG;
    return head_values(*c) < (1ull << 31) ? DF11_OK : DF11_E_INVALID_ARG;
}

inline int check_cache(const df11_kv_cache *c) {
    const int rc = check_cache_sizes(c);
    if (rc) return rc;
    if (!c->k || !c->v || misaligned(c->k, 16) || misaligned(c->v, 16) || !c->pages ||
        c->pages > INT32_MAX)
        return DF11_E_INVALID_ARG;
    for (const uint64_t stride : {c->k_stride, c->v_stride})
        if (c->pages > 1 && (stride < head_values(*c) || stride % 8 || stride >> 40))
            return DF11_E_INVALID_ARG;
    return DF11_OK;
}

inline int check_batch_sizes(const df11_kv_batch *b) {
    if (!b || b->sequences > kMaxSequences || b->prefix_len > INT32_MAX) return DF11_E_INVALID_ARG;
    return DF11_OK;
}

inline int check_batch(const df11_kv_batch *b) {
    const int rc = check_batch_sizes(b);
    if (rc || !b->sequences) return rc;
    if (!b->start || !b->length || (b->width && !b->table) || misaligned(b->start, 4) ||
        misaligned(b->length, 4) || misaligned(b->table, 4))
        return DF11_E_INVALID_ARG;
    if (b->sequences > 1 && (b->table_stride < b->width || b->table_stride >> 32))
        return DF11_E_INVALID_ARG;
    return DF11_OK;
}

inline Batch device_batch(const df11_kv_batch &b, uint64_t rows) {
    return {b.start, b.length, b.table, b.prefix_table, b.sequences > 1 ? b.table_stride : 0,
            b.sequences, b.width, b.prefix_pages, b.prefix_len, static_cast<uint32_t>(rows)};
}

// Rows of `size`-byte elements that are loaded 16 bytes at a time.
inline int check_strided(const void *p, uint64_t stride, uint64_t cols, uint64_t rows,
                         uint32_t size) {
    if (!p || misaligned(p, 16)) return DF11_E_INVALID_ARG;
    return rows > 1 && (stride < cols || stride * size % 16 || stride >> 40) ? DF11_E_INVALID_ARG
                                                                            : DF11_OK;
}

}  // namespace df11ops
