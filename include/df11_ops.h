/*
 * df11_ops.h -- C ABI of the operators around a frozen, compressed model:
 *   - low-rank adapters of many requests beside a shared projection, with
 *     the adapters' and the activations' gradients;
 *   - log probabilities of given tokens with their rank, the entropy and the
 *     top alternatives, with the logits' gradient;
 *   - distillation from a teacher's top log probabilities, loss and gradient;
 *   - a paged cache of keys and values: appending to it with the position
 *     rotation, and attention of a batch to a prefix that it shares and to
 *     each sequence's own tokens.
 *
 * The conventions are those of df11.h: the caller owns every buffer, device
 * pointers except where a size is returned, work is enqueued on `stream` and
 * the call returns without waiting, DF11_OK or a negative DF11_E_* code,
 * every argument that the host can see is checked before anything is
 * enqueued, nothing is allocated, no state is kept between calls, no atomics
 * on results: equal inputs give bit-identical outputs.  A workspace holds
 * nothing between calls; calls that overlap in time need one each.
 *
 * Floating types: DF11_F32, DF11_BF16, DF11_F16.  Sums, maxima, statistics
 * and low-rank intermediates are held in 32 bits; an output is rounded once.
 */
#ifndef DF11_OPS_H
#define DF11_OPS_H

#include "df11.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DF11_F32 0
#define DF11_BF16 1
#define DF11_F16 2

#define DF11_MAX_TOP 128  /* alternatives of a row */
#define DF11_MAX_RANK 128 /* of an adapter */
#define DF11_MIN_PAGE 16  /* tokens of a cache's page, a power of two */
#define DF11_MAX_PAGE 1024

/* ---- Log probabilities of given tokens.
 *
 * For every row z of the logits (rows x vocab values of `dtype`, row r at
 * logits + r * row_stride elements, row_stride >= vocab; any alignment that
 * the type itself needs) at temperature tau > 0, with m = max z,
 *   S = sum_j exp((z_j - m) / tau),  lp_j = (z_j - m) / tau - ln S:
 *   logprob[r]     lp of tokens[r];
 *   rank[r]        values above z[tokens[r]], plus equal ones of lower index:
 *                  the token's place in the order of the alternatives;
 *   entropy[r]     -sum_j p_j lp_j, p = exp lp (0 where p_j is 0);
 *   top_logprob, top_index (rows x top): the `top` largest, largest first,
 *                  equal ones by ascending index;
 *   stats          rows x 4 floats for the backward pass: m, ln S, the
 *                  entropy, 1/S.
 * tokens may be null (then logprob and rank must be); each output may be
 * null, top_logprob and top_index with top = 0 only.
 *   - A masked value (-inf) has probability 0.  Where fewer than `top`
 *     values are not masked, the other alternatives have index -1 and log
 *     probability -inf.  The type's lowest finite value is an ordinary one.
 *   - A row of masked values alone: logprob -inf, entropy 0, alternatives
 *     as above, gradient 0.
 *   - A row that holds a NaN or +inf has no distribution: logprob, entropy
 *     and top_logprob are NaN, rank and top_index -1, its gradient NaN.
 *   - A negative token asks nothing: logprob 0, rank -1, no gradient from
 *     logprob.  A token >= vocab: logprob NaN, rank -1, gradient NaN.
 * top <= DF11_MAX_TOP and <= vocab; vocab < 2^31; rows = 0 launches nothing.
 * DF11_E_UNSUPPORTED for more than 2^23 rows times parts of 8192 values.
 *
 * Backward: grad[r][j] = 1/tau * (grad_logprob[r] * (delta_{j,token} - p_j)
 *                                 - grad_entropy[r] * p_j * (lp_j + entropy[r])),
 * `dtype` values, rows at grad_stride >= vocab; grad_logprob and grad_entropy
 * may be null (zero) but not both; grad may be the logits themselves (with
 * their stride), which it replaces.  The alternatives carry no gradient. */
int df11_logprobs_workspace_bytes(uint32_t dtype, uint64_t rows, uint32_t vocab, uint32_t top,
                                  uint64_t *bytes);
int df11_logprobs(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                  uint64_t row_stride, const int64_t *tokens, uint32_t top, float temperature,
                  float *logprob, int64_t *rank, float *entropy, float *top_logprob,
                  int64_t *top_index, float *stats, void *workspace, uint64_t workspace_bytes,
                  hipStream_t stream);
int df11_logprobs_backward(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                           uint64_t row_stride, const int64_t *tokens, const float *stats,
                           const float *grad_logprob, const float *grad_entropy,
                           float temperature, void *grad, uint64_t grad_stride,
                           hipStream_t stream);

/* ---- Distillation from a teacher's top log probabilities.
 *
 * The teacher gives for each row `top` places teacher_index (rows x top,
 * negative: none) and its log probabilities there, teacher_logprob (rows x
 * top, over its whole vocabulary).  With p_k = exp teacher_logprob, P = sum
 * p_k and q = softmax(z / tau) of the student's row:
 *   tail != 0:  the rest of the vocabulary is one more outcome, of teacher
 *       probability r = max(0, 1 - P) and student probability Q = sum of q
 *       over the places not named:
 *       loss = sum_k p_k (ln p_k - ln q_k) + r (ln r - ln Q)
 *       gradient q_j - p_j at a named place, q_j (1 - r/Q) elsewhere;
 *   tail == 0:  p is scaled to sum to one:
 *       loss = sum_k p_k/P (ln p_k - ln P - ln q_k)
 *       gradient q_j - p_j/P at a named place, q_j elsewhere;
 * the gradient with respect to z times weight[r] / tau (weight null: 1).
 *   - A term with p_k = 0 (or r = 0) counts 0.  A place named more than once
 *     counts each of its entries.
 *   - Where all places but the named ones are masked (Q = 0), an r of up to
 *     2^-18 counts as 0: that much the logarithms' 32 bits may leave of 1.
 *   - A row whose teacher names no place, or (tail == 0) gives none of them
 *     a probability above 0, has loss 0 and gradient 0.
 *   - A student's row of masked values alone has gradient 0 (and the loss
 *     +inf that the formula gives); one that holds a NaN or +inf has loss
 *     and gradient NaN.  A named place that is masked: loss +inf, gradient
 *     by the formula.
 *   - A place >= vocab, or a teacher_logprob of NaN or +inf at a named
 *     place: the row's loss and gradient are NaN.
 * stats: rows x 4 floats for df11_distill_backward.  df11_distill writes the
 * gradient too where grad is not null (weights known beforehand: the usual
 * training step); df11_distill_backward writes it from stats, with grad_loss
 * in place of weight.  grad: `dtype`, rows at grad_stride >= vocab; it may be
 * the logits themselves (with their stride), which it replaces.
 * Logits, sizes and limits as above; 1 <= top <= DF11_MAX_TOP. */
int df11_distill_workspace_bytes(uint32_t dtype, uint64_t rows, uint32_t vocab, uint64_t *bytes);
int df11_distill(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                 uint64_t row_stride, const int64_t *teacher_index, const float *teacher_logprob,
                 uint32_t top, uint32_t tail, float temperature, const float *weight, float *loss,
                 float *stats, void *grad, uint64_t grad_stride, void *workspace,
                 uint64_t workspace_bytes, hipStream_t stream);
int df11_distill_backward(const void *logits, uint32_t dtype, uint64_t rows, uint32_t vocab,
                          uint64_t row_stride, const int64_t *teacher_index,
                          const float *teacher_logprob, uint32_t top, uint32_t tail,
                          float temperature, const float *stats, const float *grad_loss,
                          void *grad, uint64_t grad_stride, hipStream_t stream);

/* ---- Low-rank adapters beside a shared projection.
 *
 * For every token t with i = adapter[t] in [0, n_adapters):
 *   out[t] = base[t] + scale[i] * B_i (A_i x[t])
 * and out[t] = base[t] for any other value of adapter[t] (base null: zero).
 *   x        tokens x cols BF16, row t at x + t * x_stride;
 *   a        n_adapters x rank x cols BF16, b: n_adapters x rows x rank BF16;
 *   scale    n_adapters floats (null: 1); adapter: tokens int32;
 *   base, out  tokens x rows of `dtype` (DF11_F32, as df11_block_gemm gives
 *            its products, or DF11_BF16), strides in elements; out may be
 *            base itself (with its stride).
 * Any order of adapters is right; tokens of one adapter side by side share
 * its loads.  The low-rank intermediate (and an fp32 dy below) meets the matrix
 * cores as three BF16 terms, which hold all its bits, whatever the type of out.
 * (An infinity in an operand that meets such terms may come out as a NaN: a
 * term can be 0.  It stays with the tokens, rows or adapters it belongs to.)
 * rank a multiple of 8, 8 <= rank <= DF11_MAX_RANK; cols a multiple of 64 and
 * rows of 16 (as df11_matrix); tokens <= 2^24; rows of every tensor 16-byte
 * aligned (strides: multiples of 8 BF16 or 4 floats).  tokens = 0 launches
 * nothing.  DF11_E_UNSUPPORTED for more than 2^24 - 1 pieces of 64 tokens times
 * pieces of 256 of the rows, or of the cols (2^38 values).
 *
 * Backward, for the gradient dy of out (tokens x rows, DF11_F32 or DF11_BF16),
 * with u[t] = scale[i] * B_i^T dy[t] and v[t] = A_i x[t]:
 *   dx[t] = dx_base[t] + A_i^T u[t]      BF16 (dx_base null: zero; it may be dx);
 *   da[i] = sum_{t of i} u[t] x[t]^T     n_adapters x rank x cols floats;
 *   db[i] = sum_{t of i} scale[i] dy[t] v[t]^T   n_adapters x rows x rank floats;
 * an adapter without tokens gets zeros.  dx, or da and db together, may be
 * null; with da and db, dx must not be x or dy, which are read after it is
 * written. */
int df11_lora_workspace_bytes(uint64_t tokens, uint32_t cols, uint32_t rows, uint32_t rank,
                              uint32_t n_adapters, uint64_t *bytes);
int df11_lora(const uint16_t *x, uint64_t x_stride, uint64_t tokens, uint32_t cols, uint32_t rows,
              uint32_t rank, uint32_t n_adapters, const uint16_t *a, const uint16_t *b,
              const float *scale, const int32_t *adapter, const void *base, uint64_t base_stride,
              void *out, uint64_t out_stride, uint32_t dtype, void *workspace,
              uint64_t workspace_bytes, hipStream_t stream);
int df11_lora_backward_workspace_bytes(uint64_t tokens, uint32_t cols, uint32_t rows,
                                       uint32_t rank, uint32_t n_adapters, uint64_t *bytes);
int df11_lora_backward(const uint16_t *x, uint64_t x_stride, uint64_t tokens, uint32_t cols,
                       uint32_t rows, uint32_t rank, uint32_t n_adapters, const uint16_t *a,
                       const uint16_t *b, const float *scale, const int32_t *adapter,
                       const void *dy, uint64_t dy_stride, uint32_t dy_dtype,
                       const uint16_t *dx_base, uint64_t dx_base_stride, uint16_t *dx,
                       uint64_t dx_stride, float *da, float *db, void *workspace,
                       uint64_t workspace_bytes, hipStream_t stream);

/* ---- A paged cache of keys and values.
 *
 * df11_kv_cache: `pages` pages of page_size tokens for each of `heads` heads of
 * `dim` values, k and v alike: token i of page p and head h is the dim values at
 * k + p * k_stride + (h * page_size + i) * dim (elements; v with v_stride).
 *   dtype      DF11_BF16 or DF11_F16;
 *   page_size  a power of two, DF11_MIN_PAGE .. DF11_MAX_PAGE;
 *   dim        64 or 128;  heads * page_size * dim < 2^31;
 *   k_stride, v_stride  at least heads * page_size * dim, multiples of 8; k and v
 *              16-byte aligned.  (Layers side by side, or k and v, are strides.)
 *
 * df11_kv_batch: the batch's sequences, in device memory but for the sizes, so
 * that a captured call follows the values:
 *   start      sequences + 1 row numbers, ascending from 0: sequence s has rows
 *              start[s] .. start[s + 1] - 1 of the call's tensors, its last tokens
 *              in their order (none, one, or a prompt's).  Rows from
 *              start[sequences] on belong to no sequence: they are not read, and
 *              what a call writes is left as it was there;
 *   length     per sequence, the tokens of its own cache with this call's rows:
 *              row r has the place length[s] - (start[s + 1] - r) in it;
 *   table      sequences x width page numbers, row s at table + s * table_stride:
 *              place i of sequence s is token i % page_size of page
 *              table[s][i / page_size].  Entries that no place needs are not looked at;
 *   prefix_table, prefix_pages, prefix_len   the pages of the prefix that all
 *              sequences share, and its tokens (0: none).  A row's position is
 *              prefix_len + its place.
 * What the library reads in device memory leads to no access out of range: see
 * each call for page numbers outside the cache.  Two rows that share a page and a
 * token of it write over one another in any order.
 *
 * df11_kv_append: for each row r of a sequence, with place i >= 0 and position p,
 *   q_out[r] = R_p q[r],  cache.k <- R_p k[r],  cache.v <- v[r]   (at place i)
 * where R_p turns, in every head, pair j of `rotary` values by the angle
 * p * inv_freq[j] (a, b -> a cos - b sin, b cos + a sin).  Pair j is values j and
 * j + rotary / 2, or 2 j and 2 j + 1 where `interleaved`; values from rotary on
 * stay.  The angle is a product of 64 bits, taken to a turn's fraction before it is
 * rounded: as exact at the far end of a long context as at its beginning.
 *   q, k, v    rows of `dtype` (DF11_F32, as df11_block_gemm gives its products,
 *              DF11_BF16 or DF11_F16), heads * dim values in q, cache.heads * dim
 *              in k and v, strides in elements, rows 16-byte aligned;
 *   inv_freq   rotary / 2 floats (rotary = 0: no rotation, inv_freq may be null);
 *   rotary     a multiple of 16, at most dim;
 *   q_out      tokens x heads * dim of the cache's type; it may be q itself where
 *              the types are the same (with its stride).
 * A row whose place is negative, lies past the table's width or on a page outside
 * the cache is not appended; its q_out is written as any other's.  Of the batch's
 * prefix only prefix_len is looked at (prefix_table may be null).  tokens <= 2^24 - 1
 * (DF11_E_UNSUPPORTED for 2^24). */
typedef struct {
    void *k, *v;
    uint32_t dtype, pages, heads, page_size, dim;
    uint64_t k_stride, v_stride;
} df11_kv_cache;

typedef struct {
    const int32_t *start, *length, *table;
    uint32_t sequences, width;
    uint64_t table_stride;
    const int32_t *prefix_table;
    uint32_t prefix_pages, prefix_len;
} df11_kv_batch;

int df11_kv_append(const void *q, uint64_t q_stride, const void *k, uint64_t k_stride,
                   const void *v, uint64_t v_stride, uint32_t dtype, uint64_t tokens,
                   uint32_t heads, const float *inv_freq, uint32_t rotary, uint32_t interleaved,
                   const df11_kv_cache *cache, const df11_kv_batch *batch, void *q_out,
                   uint64_t q_out_stride, hipStream_t stream);

/* ---- Attention to a shared prefix and to each sequence's own tokens.
 *
 * For each row r of a sequence and each of `heads` query heads h, head
 * h / (heads / cache.heads) of the cache, over the prefix_len tokens of the prefix
 * and the sequence's places up to the row's own:
 *   s_j = scale q . k_j,  lse = ln sum_j exp s_j,  out = sum_j exp(s_j - lse) v_j.
 *   q, out     tokens x heads * dim of the cache's type, strides in elements, rows
 *              16-byte aligned; out may be q itself (with its stride);
 *   lse        tokens x heads floats, may be null;
 *   heads      a multiple of cache.heads; tokens * heads < 2^31; scale a normal
 *              number above 0.
 * Products are summed in 32 bits on the matrix cores, the softmax is held in 32 bits;
 * exp(s_j - m) is rounded to the cache's type where it meets v (in DF11_F16 in steps that
 * end at 2^-31 of the row's largest).
 *   - A row that sees nothing (no prefix and a negative place), or scores of -inf
 *     alone: out 0, lse -inf.
 *   - What lies behind a row's place (in pages, or later rows' keys and values) has
 *     no effect on it, NaN and infinities included.
 *   - A row that sees a place past the table's width or a page outside the cache has
 *     no result: out and lse NaN.
 * How the work is laid out goes by the call's sizes, the table's width among them, since
 * lengths lie in device memory:
 *   - in shares that are joined through the workspace: the rows of all sequences read the
 *     prefix together, once for 128 rows of a head of the cache;
 *   - in one kernel without a workspace, where a workgroup reads the prefix and the own
 *     tokens of 128 rows of one sequence by itself: for sequences of 64 rows of a head of
 *     the cache or more on average whose tiles fill half the GPU, and for short contexts
 *     (prefix and the table's width 512 places; 1,024 or 1,536 where rows are many).
 * So a table much wider than its sequences costs up to twice the time where they are short
 * (a prompt of 512 tokens 41 us for 22), and prompts and single tokens behind long contexts
 * are faster in a call each (four tokens of 30,000 beside a prompt of 1024 tokens, 32 heads
 * over 8: 515 us in one call, 135 in two).
 * tokens = 0 launches nothing.  DF11_E_UNSUPPORTED for tokens * heads of 2^26 or 2^37 /
 * cache.heads tokens (sequences times what a table row holds, prompts' and the prefix'
 * times their rows / 128) with a workspace, and for more than 2^24 - 1 workgroups (tokens *
 * heads / 128 + sequences * cache.heads) without. */
int df11_prefix_attention_workspace_bytes(uint64_t tokens, uint32_t heads,
                                          const df11_kv_cache *cache, const df11_kv_batch *batch,
                                          uint64_t *bytes);
int df11_prefix_attention(const void *q, uint64_t q_stride, uint64_t tokens, uint32_t heads,
                          float scale, const df11_kv_cache *cache, const df11_kv_batch *batch,
                          void *out, uint64_t out_stride, float *lse, void *workspace,
                          uint64_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* DF11_OPS_H */
