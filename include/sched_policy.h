/*
 * sched_policy.h -- operators of an agent that proposes device mappings and is
 * trained on what the search's scores say of them, on one AMD Instinct MI355X.
 *
 * The paper's scheduler is a language model that answers with one mode per
 * tool (Section 3.3); sched_search.h scores such answers.  The calls below
 * take it from there: advantages of sampled mappings from their makespans, a
 * clipped policy loss with a KL term and a preference loss over pairs of a
 * better and a worse mapping, each with its gradient, the log-probabilities of
 * an answer's tokens, the embedding lookup with its gradient, and attention
 * over ragged sequences and caches with its backward pass.
 *
 * Library, error codes and workspaces are those of sched_search.h, with one
 * difference.  All tensors live on the device and every result stays there, so
 * these calls check their arguments, enqueue their work on hip_stream and
 * return: results are valid in stream order, and an error of the GPU's shows
 * at a later synchronisation.  They allocate nothing and copy nothing to the
 * host, so a stream that is being captured takes them.  The caller keeps
 * inputs and workspace unchanged until the stream has passed the call.
 * Results depend on the inputs alone, bit by bit: no sum's order varies.
 *
 * Types: 32-bit, 16-bit and bfloat16 floating point (SCHED_F32, SCHED_F16,
 * SCHED_BF16).  Sums, softmax statistics and losses are held in 32 bits or
 * more; results are rounded once to their type.  Probabilities below 2^-126
 * count as zero.  Tokens are 32- or 64-bit integers; one outside [0, vocab) (-1,
 * say) is padding: it carries no loss, looks up zeros and takes no part in a
 * gradient.  Tensors have up to 2^31 - 1024 rows and columns.  Offsets are
 * 32-bit integers on the device, ascending; sequence i of n holds the rows
 * offsets[i] .. offsets[i+1] - 1 of its packed tensor, perhaps none, and the n
 * sequences cover it.  Offsets that leave the tensor are cut to it.
 */
#ifndef SCHED_POLICY_H
#define SCHED_POLICY_H

#include "sched_search.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SCHED_F32 0
#define SCHED_F16 1
#define SCHED_BF16 2

/* A row-major matrix on the device: rows `stride` elements apart, the elements
 * of a row next to each other; data aligned to its element.  An output's rows
 * may not overlap (stride >= cols). */
typedef struct {
    void *data;
    int32_t dtype;
    int64_t rows, cols, stride;
} sched_matrix;

/* n tokens next to each other on the device, of 32 or 64 bits each. */
typedef struct {
    const void *data;
    int32_t bits;
    int64_t n;
} sched_tokens;

/* Errors of the calls below: SCHED_E_NULL (a required pointer is null),
 * SCHED_E_SIZE (a negative or too large size, or sizes that do not match),
 * SCHED_E_VALUE (a type, flag, factor, stride or alignment that is not
 * taken), SCHED_E_WORKSPACE (null, misaligned to 256 B or too small),
 * SCHED_E_DEVICE (a launch failed).  On the first four nothing has been
 * enqueued. */

/* Embedding lookup: out[i] = scale * table[tokens[i]], zeros for padding.
 * table: vocab x dim; out: n x dim of the same type. */
int sched_embed(const sched_matrix *table, const sched_tokens *tokens, float scale,
                const sched_matrix *out, void *hip_stream);

/* Its gradient: d_table[v] = scale * the sum of d_rows[i] over the i with
 * tokens[i] = v, zeros for tokens that do not occur; with accumulate = 1 the sum
 * is added to d_table.  d_table: vocab x dim, of d_rows' type or SCHED_F32.  The
 * tokens are sorted in the workspace, and each row is summed over its run, in 32
 * bits and in one order, which is not that of i: it follows from n, dim and where
 * the run lies in the sorted list.  dim <= 2^24. */
int sched_embed_grad_workspace_bytes(int64_t n, int64_t dim, size_t *out);
int sched_embed_grad(const sched_matrix *d_rows, const sched_tokens *tokens, float scale,
                     int32_t accumulate, const sched_matrix *d_table, void *d_workspace,
                     size_t ws_bytes, void *hip_stream);

/* Log-probabilities of tokens: logp[i] = z[tokens[i]] - log sum_j exp z[j] with
 * z = row i of logits / temperature (n 32-bit values; 0 for padding, whose rows
 * are not read).  A logit of -inf is a mode or token that is not allowed and
 * has log-probability -inf, as has every token of a row of nothing else.
 * temperature > 0, and log2(e) / temperature is finite in 32 bits. */
int sched_token_logprobs(const sched_matrix *logits, const sched_tokens *tokens,
                         float temperature, float *logp, void *hip_stream);

/* Its gradient: d_logits[i][j] = d_logp[i] * ((j == tokens[i]) - q[j]) /
 * temperature with q the row's probabilities (logp, the result of the call
 * above, is what they may be taken from); zeros for padding and for tokens with
 * logp = -inf.  d_logits: of logits' type and size; it may be logits itself. */
int sched_token_logprobs_grad(const sched_matrix *logits, const sched_tokens *tokens,
                              float temperature, const float *logp, const float *d_logp,
                              const sched_matrix *d_logits, void *hip_stream);

/* Advantages of sampled answers from the makespans of their mappings, per
 * token, and the tokens' weights in a loss.  Answer a's makespan counts as
 * m[a] = min(makespan_us[a], limit_us[g]) (an infeasible mapping, INT64_MAX, as
 * its group's limit); with mean and (population) standard deviation over its
 * group g (answers group_offsets[g] .. group_offsets[g+1] - 1 of the same
 * workflow) its advantage is (mean - m[a]) / deviation, 0 if all are equal.
 * Every token of the answer (rows offsets[a] .. offsets[a+1] - 1) gets it; its
 * weight is 1 / (tokens that are no padding) with mean = 0, and with mean = 1
 * 1 / (answers with such tokens * such tokens of its answer); 0 for padding.
 * advantages and weights: 32-bit values, tokens->n each.  tokens counts as
 * padding what is negative.  Up to 65,536 answers.  Workspace: 4 bytes per
 * answer. */
int sched_group_advantages(const int64_t *makespan_us, const int64_t *limit_us,
                           const int32_t *group_offsets, int32_t n_groups,
                           const int32_t *offsets, int32_t n_answers, const sched_tokens *tokens,
                           int32_t mean, float *advantages, float *weights, void *d_workspace,
                           size_t ws_bytes, void *hip_stream);

/* Clipped policy loss with a KL term, and its gradient, from the logits in one
 * pass.  For token i with log-probability l (as above), r = exp(l -
 * old_logp[i]), e = ref_logp[i] - l and advantage A:
 *
 *   losses[i] = weights[i] * (max(-A r, -A min(max(r, 1 - clip_low), 1 + clip_high))
 *                             + kl_weight * (exp(e) - e - 1))
 *
 * loss[0] is their sum, logp[i] = l, and d_logits the gradient of loss[0]
 * times loss_scale.  Where both terms of the max are equal the first one's
 * gradient counts.  ref_logp may be null if kl_weight is 0.  Padding and tokens
 * with logp = -inf have zero gradient; padding has losses and logp 0.  What is
 * no number shows in its token's loss and gradient and in loss[0].
 *
 * A group's advantages add up to zero, so loss[0] is mostly a small difference
 * of its terms: like its 32-bit inputs it is good to some 2^-24 of the sum of
 * their magnitudes, which, where that is 1,000 times the loss, is 6e-5 of the
 * loss itself.  The gradient has no such sum. */
typedef struct {
    sched_matrix logits;
    sched_tokens tokens;
    const float *old_logp, *ref_logp, *advantages, *weights;
    float clip_low, clip_high, kl_weight, temperature, loss_scale;
    float *loss, *losses, *logp;
    sched_matrix d_logits; /* of logits' type and size; may be logits itself */
} sched_policy_desc;
int sched_policy_loss(const sched_policy_desc *desc, void *hip_stream);

/* Preference loss over pairs (sequence 2p holds the tokens of the better
 * mapping, 2p + 1 those of the worse) from their log-probabilities:
 *
 *   margins[p] = beta * (sum over 2p of (logp - ref_logp) - the same over 2p + 1)
 *   loss[0] = loss_scale * mean over p of -(1 - smoothing) log s(margins[p])
 *             - smoothing log s(-margins[p]),   s(x) = 1 / (1 + exp(-x))
 *
 * and d_logp, the gradient of loss[0], for sched_token_logprobs_grad.
 * Negative tokens are padding: they take no part and have d_logp 0.  1 to
 * 2^23 - 1 pairs. */
int sched_preference_loss(const float *logp, const float *ref_logp, const sched_tokens *tokens,
                          const int32_t *offsets, int32_t n_pairs, float beta, float smoothing,
                          float loss_scale, float *loss, float *margins, float *d_logp,
                          void *hip_stream);

/* Heads of a packed sequence tensor on the device: element d of head h of row
 * r at data[r * row_stride + h * head_stride + d].  Strides are multiples of 8
 * elements and data is aligned to 16 bytes (a slice of a joint projection is
 * one of these). */
typedef struct {
    void *data;
    int64_t row_stride, head_stride;
} sched_heads;

/* Attention of packed sequences.  Sequence b has the query rows q_offsets[b]
 * .. q_offsets[b+1] - 1 and the first k_lengths[b] key rows of k_offsets[b] ..
 * k_offsets[b+1] - 1 (all of them where k_lengths is null): a cache is a tensor
 * of slots whose lengths grow, and what its other rows hold is not used.
 * Query head h reads key head h / (q_heads / kv_heads).  With causal = 1 the
 * last query row sees every key and each one before it one less (query i of
 * n_q sees the keys j <= i + n_k - n_q).  scale is applied to the products.
 * A row that sees no key gives zeros, lse = -inf and zero gradients.  Key rows
 * behind a length may hold anything; those of a sequence that causal = 1 alone
 * hides from a row have weight zero there and have to be finite.
 * head_dim: a multiple of 8 up to 128.  dtype: SCHED_F16 or SCHED_BF16; the
 * probabilities are rounded to it before they are multiplied with the values
 * (SCHED_F16: small ones in steps of 2^-31 of the row's largest).
 * q_rows * q_heads / 32 + n_seqs * kv_heads and k_rows * kv_heads / 64 + n_seqs *
 * kv_heads stay below 2^24 - 8, and a key head has up to 4096 query heads. */
typedef struct {
    sched_heads q, k, v, out; /* out: q_rows x q_heads x head_dim */
    float *lse;               /* q_heads x q_rows, natural logarithm */
    int32_t dtype, head_dim, q_heads, kv_heads;
    int64_t q_rows, k_rows;
    const int32_t *q_offsets, *k_offsets, *k_lengths;
    int32_t n_seqs, causal;
    float scale;
} sched_attention_desc;

/* out and lse are written.  With few query rows a sequence's keys are read by
 * several groups of waves, whose parts are joined through the workspace. */
int sched_attention_workspace_bytes(const sched_attention_desc *desc, size_t *out);
int sched_attention(const sched_attention_desc *desc, void *d_workspace, size_t ws_bytes,
                    void *hip_stream);

/* The backward pass: d_q, d_k and d_v from d_out and the forward pass's out
 * and lse (read here); the probabilities are computed again.  They and the
 * products' gradients are rounded to dtype before they are multiplied (SCHED_F16:
 * held times powers of two that follow from their size).  Key rows of a slot
 * beyond its length get zeros.  With few rows or keys their sums too are joined
 * through the workspace. */
int sched_attention_grad_workspace_bytes(const sched_attention_desc *desc, size_t *out);
int sched_attention_grad(const sched_attention_desc *desc, const sched_heads *d_out,
                         const sched_heads *d_q, const sched_heads *d_k, const sched_heads *d_v,
                         void *d_workspace, size_t ws_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* SCHED_POLICY_H */
