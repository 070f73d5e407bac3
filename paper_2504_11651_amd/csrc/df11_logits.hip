// Operators on rows of logits: log probabilities of given tokens with rank,
// entropy and top alternatives, distillation from a teacher's top log
// probabilities, and the gradients of both.  One workgroup per row.
#include "df11_ops_common.h"

namespace {

using namespace df11ops;

constexpr uint32_t kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr uint32_t kPart = 8192;  // values of a row that one workgroup of a gradient takes

// (v - m) / tau, of halves so that the difference of two finite values is finite
__device__ float scaled(float v, float m, float two_over_tau) {
    return fmaf(v, 0.5f, -0.5f * m) * two_over_tau;
}

struct LogprobArgs {
    const void *logits;
    const int64_t *tokens;
    float *logprob, *entropy, *top_logprob, *stats;
    int64_t *rank, *top_index;
    uint64_t stride;
    uint32_t vocab, top;
    float two_over_tau;
};

template <class T>
__global__ __launch_bounds__(kThreads) void logprob_rows_kernel(LogprobArgs g) {
    __shared__ float red[kWaves];
    __shared__ float best_v[kThreads];
    __shared__ uint32_t best_i[kThreads];
    const uint64_t row = blockIdx.x;
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    const int64_t token = g.tokens ? g.tokens[row] : -1;
    const bool asked = token >= 0 && token < g.vocab;
    const float zt = asked ? T::load(z[token]) : 0.0f;
    // the lowest finite value and no -inf: masked values then give exp(-inf)
    float m = -3.402823466e38f;
    for (uint32_t j = threadIdx.x; j < g.vocab; j += kThreads) m = fmaxf(m, T::load(z[j]));
    m = wg_max<kWaves>(m, red);
    float s = 0.0f, t = 0.0f, above = 0.0f;
    for (uint32_t j = threadIdx.x; j < g.vocab; j += kThreads) {
        const float v = T::load(z[j]);
        const float x = scaled(v, m, g.two_over_tau);
        const float e = expf(x);
        s += e;
        t += e * fmaxf(x, -200.0f);  // e is 0 below; no 0 * inf
        above += v > zt || (v == zt && j < static_cast<uint64_t>(token)) ? 1.0f : 0.0f;
    }
    s = wg_sum<kWaves>(s, red);
    t = wg_sum<kWaves>(t, red);
    above = wg_sum<kWaves>(above, red);  // below 2^24 by its parts' sizes up to that vocabulary
    const bool broken = !(s >= 0.0f) || s == INFINITY;
    const bool empty = s == 0.0f;
    const float ln_s = logf(s);
    const float nan = __builtin_nanf("");
    if (threadIdx.x == 0) {
        float lp = empty ? -INFINITY : scaled(zt, m, g.two_over_tau) - ln_s;
        const float h = broken ? nan : empty ? 0.0f : ln_s - t / s;
        if (token < 0) lp = 0.0f;
        if ((token >= 0 && !asked) || broken) lp = nan;
        if (g.logprob) g.logprob[row] = lp;
        if (g.rank) g.rank[row] = asked && !broken ? static_cast<int64_t>(above) : -1;
        if (g.entropy) g.entropy[row] = h;
        if (g.stats) {
            g.stats[4 * row] = m;
            g.stats[4 * row + 1] = ln_s;
            g.stats[4 * row + 2] = h;
            g.stats[4 * row + 3] = lp;
        }
    }
    // one alternative a pass: the largest after the last one
    float last_v = INFINITY;
    uint32_t last_i = 0;
    for (uint32_t k = 0; k < g.top; ++k) {
        float v = -INFINITY;
        uint32_t i = ~0u;
        for (uint32_t j = threadIdx.x; j < g.vocab; j += kThreads) {
            const float w = T::load(z[j]);
            const bool after = k == 0 || w < last_v || (w == last_v && j > last_i);
            if (after && w > v) {
                v = w;
                i = j;
            }
        }
        best_v[threadIdx.x] = v;
        best_i[threadIdx.x] = i;
        __syncthreads();
        for (uint32_t d = kThreads / 2; d; d >>= 1) {
            if (threadIdx.x < d) {
                const float w = best_v[threadIdx.x + d];
                const uint32_t j = best_i[threadIdx.x + d];
                if (w > best_v[threadIdx.x] || (w == best_v[threadIdx.x] && j < best_i[threadIdx.x])) {
                    best_v[threadIdx.x] = w;
                    best_i[threadIdx.x] = j;
                }
            }
            __syncthreads();
        }
        last_v = best_v[0];
        last_i = best_i[0];
        const bool none = last_i == ~0u;
        __syncthreads();
        if (threadIdx.x == 0) {
            g.top_logprob[row * g.top + k] =
                broken ? nan : none ? -INFINITY : scaled(last_v, m, g.two_over_tau) - ln_s;
            g.top_index[row * g.top + k] = broken || none ? -1 : static_cast<int64_t>(last_i);
        }
    }
}

struct LogprobGradArgs {
    const void *logits;
    void *grad;
    const int64_t *tokens;
    const float *stats, *grad_logprob, *grad_entropy;
    uint64_t stride, grad_stride;
    uint32_t vocab, parts;
    float two_over_tau;
};

template <class T>
__global__ __launch_bounds__(kThreads) void logprob_grad_kernel(LogprobGradArgs g) {
    const uint64_t row = blockIdx.x / g.parts;
    const uint32_t from = (blockIdx.x % g.parts) * kPart;
    const uint32_t to = min(g.vocab, from + kPart);
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    auto *out = static_cast<typename T::raw *>(g.grad) + row * g.grad_stride;
    const int64_t token = g.tokens ? g.tokens[row] : -1;
    const float m = g.stats[4 * row], ln_s = g.stats[4 * row + 1], h = g.stats[4 * row + 2];
    float gl = g.grad_logprob && token >= 0 ? g.grad_logprob[row] : 0.0f;
    if (token >= static_cast<int64_t>(g.vocab)) gl = __builtin_nanf("");
    const float ge = g.grad_entropy ? g.grad_entropy[row] : 0.0f;
    const bool empty = ln_s == -INFINITY;
    for (uint32_t j = from + threadIdx.x; j < to; j += kThreads) {
        const float lp = scaled(T::load(z[j]), m, g.two_over_tau) - ln_s;
        const float p = expf(lp);
        float d = -p * (gl + ge * (fmaxf(lp, -200.0f) + h));
        if (token == static_cast<int64_t>(j)) d += gl;
        out[j] = T::store(empty ? 0.0f : d * (0.5f * g.two_over_tau));
    }
}

struct DistillArgs {
    const void *logits;
    void *grad;
    const int64_t *index;
    const float *teacher, *weight;
    float *loss, *stats;
    uint64_t stride, grad_stride;
    uint32_t vocab, top, tail, parts;
    float two_over_tau;
};

// The teacher's entries of a row in LDS: place (~0 where there is none) and
// probability.  Returns whether an entry is bad.
template <class A>
__device__ bool load_teacher(const A &g, uint64_t row, uint32_t *place, float *prob) {
    bool bad = false;
    for (uint32_t k = threadIdx.x; k < g.top; k += kThreads) {
        const int64_t i = g.index[row * g.top + k];
        const float lp = g.teacher[row * g.top + k];
        if (i >= 0 && (i >= static_cast<int64_t>(g.vocab) || !(lp < INFINITY))) bad = true;
        place[k] = i < 0 ? ~0u : static_cast<uint32_t>(i);
        prob[k] = i < 0 ? 0.0f : expf(lp);
    }
    return __syncthreads_or(bad);
}

template <class T>
__global__ __launch_bounds__(kThreads) void distill_rows_kernel(DistillArgs g) {
    __shared__ float red[kWaves];
    __shared__ uint32_t place[DF11_MAX_TOP];
    __shared__ float prob[DF11_MAX_TOP];
    const uint64_t row = blockIdx.x;
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    const bool bad = load_teacher(g, row, place, prob);
    float m = -3.402823466e38f;
    for (uint32_t j = threadIdx.x; j < g.vocab; j += kThreads) m = fmaxf(m, T::load(z[j]));
    m = wg_max<kWaves>(m, red);
    float s = 0.0f, rest = 0.0f;
    for (uint32_t j = threadIdx.x; j < g.vocab; j += kThreads) {
        const float e = expf(scaled(T::load(z[j]), m, g.two_over_tau));
        bool named = false;
        for (uint32_t k = 0; k < g.top; ++k) named |= place[k] == j;
        s += e;
        rest += named ? 0.0f : e;
    }
    s = wg_sum<kWaves>(s, red);
    rest = wg_sum<kWaves>(rest, red);
    const float ln_s = logf(s);
    float mass = 0.0f, some = 0.0f;
    for (uint32_t k = threadIdx.x; k < g.top; k += kThreads) {
        mass += prob[k];
        some += place[k] != ~0u ? 1.0f : 0.0f;
    }
    mass = wg_sum<kWaves>(mass, red);
    some = wg_sum<kWaves>(some, red);
    const float scale = g.tail ? 1.0f : 1.0f / mass, ln_mass = g.tail ? 0.0f : logf(mass);
    float loss = 0.0f;
    if (!bad)
        for (uint32_t k = threadIdx.x; k < g.top; k += kThreads)
            if (prob[k] > 0.0f) {
                const float lq = scaled(T::load(z[place[k]]), m, g.two_over_tau) - ln_s;
                loss += prob[k] * scale * (g.teacher[row * g.top + k] - ln_mass - lq);
            }
    loss = wg_sum<kWaves>(loss, red);
    if (threadIdx.x == 0) {
        const float left = rest / s, r = fmaxf(0.0f, 1.0f - mass);
        float other = 1.0f, inv_mass = scale;
        if (g.tail) {
            if (r > 0.0f) loss += r * (logf(r) - logf(left));
            other = r > 0.0f ? (left > 0.0f ? 1.0f - r / left : 0.0f) : 1.0f;
        }
        if (s == 0.0f) {
            inv_mass = -1.0f;
            loss = INFINITY;
        }
        if (!(s >= 0.0f) || s == INFINITY) loss = other = __builtin_nanf("");
        if (some == 0.0f || (!g.tail && mass == 0.0f)) {
            loss = 0.0f;
            inv_mass = -1.0f;
        }
        if (bad) loss = other = inv_mass = __builtin_nanf("");
        g.loss[row] = loss;
        g.stats[4 * row] = m;
        g.stats[4 * row + 1] = ln_s;
        g.stats[4 * row + 2] = other;
        g.stats[4 * row + 3] = inv_mass;
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void distill_grad_kernel(DistillArgs g) {
    __shared__ uint32_t place[DF11_MAX_TOP];
    __shared__ float prob[DF11_MAX_TOP];
    const uint64_t row = blockIdx.x / g.parts;
    const uint32_t from = (blockIdx.x % g.parts) * kPart;
    const uint32_t to = min(g.vocab, from + kPart);
    const auto *z = static_cast<const typename T::raw *>(g.logits) + row * g.stride;
    auto *out = static_cast<typename T::raw *>(g.grad) + row * g.grad_stride;
    load_teacher(g, row, place, prob);
    const float m = g.stats[4 * row], ln_s = g.stats[4 * row + 1];
    const float other = g.stats[4 * row + 2], inv_mass = g.stats[4 * row + 3];
    const float w = (g.weight ? g.weight[row] : 1.0f) * (0.5f * g.two_over_tau);
    for (uint32_t j = from + threadIdx.x; j < to; j += kThreads) {
        const float q = expf(scaled(T::load(z[j]), m, g.two_over_tau) - ln_s);
        bool named = false;
        float p = 0.0f;
        for (uint32_t k = 0; k < g.top; ++k)
            if (place[k] == j) {
                named = true;
                p += prob[k];
            }
        const float d = inv_mass != inv_mass ? inv_mass : named ? q - p * inv_mass : q * other;
        out[j] = T::store(inv_mass < 0.0f ? 0.0f : d * w);
    }
}

// ---- host side
constexpr uint64_t kMostParts = 1ull << 23;

uint32_t parts_of(uint32_t vocab) { return (vocab - 1) / kPart + 1; }

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
    *bytes = 0;
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
    (void)workspace;
    (void)workspace_bytes;
    LogprobArgs g{logits, tokens, logprob, entropy, top_logprob, stats, rank, top_index,
                  row_stride, vocab, top, 2.0f / temperature};
    DF11_BY_DTYPE(dtype, logprob_rows_kernel, rows, kThreads, stream, g);
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
                      grad_stride, vocab, parts_of(vocab), 2.0f / temperature};
    DF11_BY_DTYPE(dtype, logprob_grad_kernel, rows * g.parts, kThreads, stream, g);
    return launched();
}

int df11_distill_workspace_bytes(uint32_t dtype, uint64_t rows, uint32_t vocab, uint64_t *bytes) {
    if (!bytes) return DF11_E_INVALID_ARG;
    static const float some = 0.0f;
    const int rc = check_logits(&some, dtype, rows, vocab, vocab);
    if (rc) return rc;
    *bytes = 0;
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
    (void)workspace;
    (void)workspace_bytes;
    DistillArgs g{logits, grad, teacher_index, teacher_logprob, weight, loss, stats, row_stride,
                  grad_stride, vocab, top, tail, parts_of(vocab), 2.0f / temperature};
    DF11_BY_DTYPE(dtype, distill_rows_kernel, rows, kThreads, stream, g);
    if ((rc = launched()) || !grad) return rc;
    DF11_BY_DTYPE(dtype, distill_grad_kernel, rows * g.parts, kThreads, stream, g);
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
    DistillArgs g{logits, grad, teacher_index, teacher_logprob, grad_loss, nullptr,
                  const_cast<float *>(stats), row_stride, grad_stride, vocab, top, tail,
                  parts_of(vocab), 2.0f / temperature};
    DF11_BY_DTYPE(dtype, distill_grad_kernel, rows * g.parts, kThreads, stream, g);
    return launched();
}

}  // extern "C"
