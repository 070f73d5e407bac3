// Low-rank adapters of many requests beside a shared projection, and their
// gradients.
#include "df11_ops_common.h"

namespace {

using namespace df11ops;

constexpr uint32_t kThreads = 256;

// low[t][r] = scale * sum_c x[t][c] * w[i][r * wr + c * wc], one wave each; 0
// for a token without an adapter.
struct ShrinkArgs {
    const void *x;
    const uint16_t *w;
    const float *scale;
    const int32_t *adapter;
    float *low;
    uint64_t x_stride;
    uint32_t len, rank, n_adapters, wr, wc;
};

template <class T>
__global__ __launch_bounds__(64) void lora_shrink_kernel(ShrinkArgs g) {
    const uint64_t t = blockIdx.x;
    const uint32_t r = blockIdx.y;
    const int32_t i = g.adapter[t];
    if (i < 0 || static_cast<uint32_t>(i) >= g.n_adapters) {
        if (threadIdx.x == 0) g.low[t * g.rank + r] = 0.0f;
        return;
    }
    const auto *x = static_cast<const typename T::raw *>(g.x) + t * g.x_stride;
    const uint16_t *w = g.w + static_cast<uint64_t>(i) * g.len * g.rank + static_cast<uint64_t>(r) * g.wr;
    float s = 0.0f;
    for (uint32_t c = threadIdx.x; c < g.len; c += 64)
        s += T::load(x[c]) * BF16::load(w[static_cast<uint64_t>(c) * g.wc]);
    s = wave_sum(s);
    if (threadIdx.x == 0) g.low[t * g.rank + r] = s * (g.scale ? g.scale[i] : 1.0f);
}

// out[t][c] = base[t][c] + sum_r low[t][r] * w[i][c * wc + r * wr]
struct ExpandArgs {
    const float *low;
    const uint16_t *w;
    const int32_t *adapter;
    const void *base;
    void *out;
    uint64_t base_stride, out_stride;
    uint32_t len, rank, n_adapters, wr, wc;
};

template <class T>
__global__ __launch_bounds__(kThreads) void lora_expand_kernel(ExpandArgs g) {
    const uint64_t t = blockIdx.x;
    const uint32_t c = blockIdx.y * kThreads + threadIdx.x;
    if (c >= g.len) return;
    const int32_t i = g.adapter[t];
    float s = g.base ? T::load(static_cast<const typename T::raw *>(g.base)[t * g.base_stride + c]) : 0.0f;
    if (i >= 0 && static_cast<uint32_t>(i) < g.n_adapters) {
        const uint16_t *w = g.w + static_cast<uint64_t>(i) * g.len * g.rank + static_cast<uint64_t>(c) * g.wc;
        float d = 0.0f;
        for (uint32_t r = 0; r < g.rank; ++r)
            d += g.low[t * g.rank + r] * BF16::load(w[static_cast<uint64_t>(r) * g.wr]);
        s += d;
    }
    static_cast<typename T::raw *>(g.out)[t * g.out_stride + c] = T::store(s);
}

// d[i][c * wc + r * wr] = sum_{t of i} low[t][r] * x[t][c]
struct OuterArgs {
    const void *x;
    const float *low;
    const int32_t *adapter;
    float *d;
    uint64_t x_stride, tokens;
    uint32_t len, rank, wr, wc;
};

template <class T>
__global__ __launch_bounds__(kThreads) void lora_outer_kernel(OuterArgs g) {
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x, r = blockIdx.y, i = blockIdx.z;
    if (c >= g.len) return;
    float s = 0.0f;
    for (uint64_t t = 0; t < g.tokens; ++t)
        if (g.adapter[t] == static_cast<int32_t>(i))
            s += g.low[t * g.rank + r] *
                 T::load(static_cast<const typename T::raw *>(g.x)[t * g.x_stride + c]);
    g.d[static_cast<uint64_t>(i) * g.len * g.rank + static_cast<uint64_t>(c) * g.wc +
        static_cast<uint64_t>(r) * g.wr] = s;
}

// ---- host side
int check_shapes(uint64_t tokens, uint32_t cols, uint32_t rows, uint32_t rank,
                 uint32_t n_adapters) {
    if (!cols || !rows || !rank || !n_adapters) return DF11_E_INVALID_ARG;
    if (cols % 64 || rows % 16 || rank % 8 || rank > DF11_MAX_RANK || tokens > 0x7FFFFFFFull ||
        n_adapters > 65535u || cols > (1u << 24) || rows > (1u << 24))
        return DF11_E_UNSUPPORTED;
    return DF11_OK;
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

}  // namespace

extern "C" {

int df11_lora_workspace_bytes(uint64_t tokens, uint32_t cols, uint32_t rows, uint32_t rank,
                              uint32_t n_adapters, uint64_t *bytes) {
    if (!bytes) return DF11_E_INVALID_ARG;
    const int rc = check_shapes(tokens, cols, rows, rank, n_adapters);
    if (rc) return rc;
    *bytes = 4 * tokens * rank;
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
    float *low = static_cast<float *>(workspace);
    ShrinkArgs s{x, a, scale, adapter, low, x_stride, cols, rank, n_adapters, cols, 1};
    hipLaunchKernelGGL(lora_shrink_kernel<BF16>, dim3(tokens, rank), dim3(64), 0, stream, s);
    if ((rc = launched())) return rc;
    ExpandArgs e{low, b, adapter, base, out, base_stride, out_stride, rows, rank, n_adapters, 1, rank};
    const dim3 grid(tokens, (rows + kThreads - 1) / kThreads);
    if (dtype == DF11_F32)
        hipLaunchKernelGGL(lora_expand_kernel<F32>, grid, dim3(kThreads), 0, stream, e);
    else
        hipLaunchKernelGGL(lora_expand_kernel<BF16>, grid, dim3(kThreads), 0, stream, e);
    return launched();
}

int df11_lora_backward_workspace_bytes(uint64_t tokens, uint32_t cols, uint32_t rows,
                                       uint32_t rank, uint32_t n_adapters, uint64_t *bytes) {
    const int rc = df11_lora_workspace_bytes(tokens, cols, rows, rank, n_adapters, bytes);
    if (rc) return rc;
    *bytes = 8 * tokens * rank;
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
    if (tokens) {
        rc = check_common(x, x_stride, tokens, cols, a, b, scale, adapter);
        if (!rc) rc = check_rows(dy, dy_stride, rows, tokens, elem_bytes(dy_dtype));
        if (!rc && dx) rc = check_rows(dx, dx_stride, cols, tokens, 2);
        if (!rc && dx_base) rc = check_rows(dx_base, dx_base_stride, cols, tokens, 2);
        if (!rc && dx_base && dx_base == dx && tokens > 1 && dx_base_stride != dx_stride)
            rc = DF11_E_INVALID_ARG;
        if (!rc) rc = check_workspace(workspace, workspace_bytes, need);
        if (rc) return rc;
    }
    float *u = static_cast<float *>(workspace), *v = u + tokens * rank;
    if (tokens) {
        ShrinkArgs s{dy, b, scale, adapter, u, dy_stride, rows, rank, n_adapters, 1, rank};
        if (dy_dtype == DF11_F32)
            hipLaunchKernelGGL(lora_shrink_kernel<F32>, dim3(tokens, rank), dim3(64), 0, stream, s);
        else
            hipLaunchKernelGGL(lora_shrink_kernel<BF16>, dim3(tokens, rank), dim3(64), 0, stream, s);
        if ((rc = launched())) return rc;
        if (dx) {
            ExpandArgs e{u, a, adapter, dx_base, dx, dx_base_stride, dx_stride, cols, rank,
                         n_adapters, cols, 1};
            hipLaunchKernelGGL(lora_expand_kernel<BF16>,
                               dim3(tokens, (cols + kThreads - 1) / kThreads), dim3(kThreads), 0,
                               stream, e);
            if ((rc = launched())) return rc;
        }
    }
    if (!da) return DF11_OK;
    if (tokens) {
        ShrinkArgs s{x, a, scale, adapter, v, x_stride, cols, rank, n_adapters, cols, 1};
        hipLaunchKernelGGL(lora_shrink_kernel<BF16>, dim3(tokens, rank), dim3(64), 0, stream, s);
        if ((rc = launched())) return rc;
    }
    OuterArgs o{x, u, adapter, da, x_stride, tokens, cols, rank, cols, 1};
    hipLaunchKernelGGL(lora_outer_kernel<BF16>,
                       dim3((cols + kThreads - 1) / kThreads, rank, n_adapters), dim3(kThreads), 0,
                       stream, o);
    if ((rc = launched())) return rc;
    OuterArgs p{dy, v, adapter, db, dy_stride, tokens, rows, rank, 1, rank};
    const dim3 grid((rows + kThreads - 1) / kThreads, rank, n_adapters);
    if (dy_dtype == DF11_F32)
        hipLaunchKernelGGL(lora_outer_kernel<F32>, grid, dim3(kThreads), 0, stream, p);
    else
        hipLaunchKernelGGL(lora_outer_kernel<BF16>, grid, dim3(kThreads), 0, stream, p);
    return launched();
}

}  // extern "C"
