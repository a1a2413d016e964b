// policy_api.cpp -- the C ABI of include/sched_policy.h: checks of arguments,
// then the launches.  Nothing here allocates or waits.
#include <hip/hip_runtime.h>

#include <cmath>

#include "policy_launch.h"

using namespace policy;

namespace {

constexpr int64_t kMostRows = (int64_t(1) << 31) - 1024;  // strides over rows stay in 32 bits
constexpr int64_t kMostDim = int64_t(1) << 24;    // of an embedding
constexpr int32_t kMostPairs = 1 << 23;
constexpr int32_t kMostAnswers = 1 << 16;         // every one's wave adds up all counts
constexpr int64_t kMostTiles = (1 << 24) - 8;     // blocks of 256 threads in a grid

int done(hipError_t e) { return e == hipSuccess ? SCHED_OK : SCHED_E_DEVICE; }

hipStream_t stream_of(void* s) { return static_cast<hipStream_t>(s); }

int check_matrix(const sched_matrix& m, bool output) {
  if (m.rows < 0 || m.cols < 0 || m.rows > kMostRows || m.cols > kMostRows) return SCHED_E_SIZE;
  if (element_bytes(m.dtype) == 0) return SCHED_E_VALUE;
  if (m.rows == 0 || m.cols == 0) return SCHED_OK;
  if (m.data == nullptr) return SCHED_E_NULL;
  if (m.stride < 0 || (output && m.rows > 1 && m.stride < m.cols)) return SCHED_E_VALUE;
  if (reinterpret_cast<uintptr_t>(m.data) % uintptr_t(element_bytes(m.dtype))) return SCHED_E_VALUE;
  return SCHED_OK;
}

int check_tokens(const sched_tokens& t) {
  if (t.n < 0 || t.n > kMostRows) return SCHED_E_SIZE;
  if (t.bits != 32 && t.bits != 64) return SCHED_E_VALUE;
  if (t.n > 0 && t.data == nullptr) return SCHED_E_NULL;
  if (reinterpret_cast<uintptr_t>(t.data) % uintptr_t(t.bits / 8)) return SCHED_E_VALUE;
  return SCHED_OK;
}

int check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return SCHED_OK;
  if (ws == nullptr || reinterpret_cast<uintptr_t>(ws) % 256 || have < need)
    return SCHED_E_WORKSPACE;
  return SCHED_OK;
}

bool positive(float x) { return std::isfinite(x) && x > 0; }

// A matrix of logits with a token per row and factors that can be used.
int check_logits(const sched_matrix& logits, const sched_tokens& tokens, float temperature) {
  if (int e = check_matrix(logits, false)) return e;
  if (int e = check_tokens(tokens)) return e;
  if (logits.rows != tokens.n || logits.cols < 1) return SCHED_E_SIZE;
  // The factor of the powers, log2(e) / temperature, is the largest that is used.
  if (!positive(temperature) || !std::isfinite(float(1.4426950408889634 / double(temperature))))
    return SCHED_E_VALUE;
  return SCHED_OK;
}

int check_d_logits(const sched_matrix& logits, const sched_matrix& d) {
  if (int e = check_matrix(d, true)) return e;
  if (d.rows != logits.rows || d.cols != logits.cols) return SCHED_E_SIZE;
  if (d.dtype != logits.dtype) return SCHED_E_VALUE;
  // In place is the same rows; anything between would be read after it is written.
  if (d.data == logits.data && d.stride != logits.stride && d.rows > 1) return SCHED_E_VALUE;
  return SCHED_OK;
}

// Heads of 16-bit values, 16-byte pieces of which are read or written at once.
int check_heads(const sched_heads& h, int64_t rows, int32_t heads, int32_t dim, bool output) {
  if (rows == 0) return SCHED_OK;
  if (h.data == nullptr) return SCHED_E_NULL;
  if (reinterpret_cast<uintptr_t>(h.data) % 16 || h.row_stride % 8 || h.head_stride % 8 ||
      h.row_stride < 0 || h.head_stride < 0)
    return SCHED_E_VALUE;
  // An output's heads may not overlap: rows of heads, or heads of rows.
  const bool rows_first = (heads == 1 || h.head_stride >= dim) &&
                          (rows == 1 || h.row_stride >= (heads - 1) * h.head_stride + dim);
  const bool heads_first = (rows == 1 || h.row_stride >= dim) &&
                           (heads == 1 || h.head_stride >= (rows - 1) * h.row_stride + dim);
  return output && !rows_first && !heads_first ? SCHED_E_VALUE : SCHED_OK;
}

int check_attention_sizes(const sched_attention_desc& d) {
  if (d.dtype != SCHED_F16 && d.dtype != SCHED_BF16) return SCHED_E_VALUE;
  if (d.head_dim < 8 || d.head_dim > 128 || d.head_dim % 8 || d.kv_heads < 1 ||
      d.kv_heads > 65535 || d.q_heads < 1 || d.q_heads % d.kv_heads ||
      d.q_heads / d.kv_heads > 4096 || d.n_seqs < 0 ||
      d.q_rows < 0 || d.k_rows < 0 || d.k_rows > kMostRows || d.q_rows > kMostRows ||
      d.q_rows * (d.q_heads / d.kv_heads) > kMostRows)
    return SCHED_E_SIZE;
  const int64_t q_tiles = d.q_rows * (d.q_heads / d.kv_heads) / 32 + d.n_seqs;
  const int64_t k_tiles = d.k_rows / 64 + d.n_seqs;
  if (q_tiles * d.kv_heads >= kMostTiles || k_tiles * d.kv_heads >= kMostTiles) return SCHED_E_SIZE;
  return SCHED_OK;
}

int check_attention(const sched_attention_desc& d) {
  if (int e = check_attention_sizes(d)) return e;
  if (!positive(d.scale) || (d.causal != 0 && d.causal != 1)) return SCHED_E_VALUE;
  if (int e = check_heads(d.q, d.q_rows, d.q_heads, d.head_dim, false)) return e;
  if (int e = check_heads(d.k, d.k_rows, d.kv_heads, d.head_dim, false)) return e;
  if (int e = check_heads(d.v, d.k_rows, d.kv_heads, d.head_dim, false)) return e;
  if (int e = check_heads(d.out, d.q_rows, d.q_heads, d.head_dim, true)) return e;
  if (d.n_seqs > 0 && (!d.q_offsets || !d.k_offsets)) return SCHED_E_NULL;
  if (d.q_rows > 0 && !d.lse) return SCHED_E_NULL;
  return SCHED_OK;
}

}  // namespace

extern "C" {

int sched_embed(const sched_matrix* table, const sched_tokens* tokens, float scale,
                const sched_matrix* out, void* hip_stream) {
  if (!table || !tokens || !out) return SCHED_E_NULL;
  if (int e = check_matrix(*table, false)) return e;
  if (int e = check_matrix(*out, true)) return e;
  if (int e = check_tokens(*tokens)) return e;
  if (out->rows != tokens->n || out->cols != table->cols) return SCHED_E_SIZE;
  if (out->dtype != table->dtype || !std::isfinite(scale)) return SCHED_E_VALUE;
  return done(launch_embed(*table, *tokens, scale, *out, stream_of(hip_stream)));
}

int sched_embed_grad_workspace_bytes(int64_t n, int64_t dim, size_t* out) {
  if (!out) return SCHED_E_NULL;
  if (n < 0 || n > kMostRows || dim < 0 || dim > kMostDim) return SCHED_E_SIZE;
  *out = embed_grad_bytes(n, dim);
  return SCHED_OK;
}

int sched_embed_grad(const sched_matrix* d_rows, const sched_tokens* tokens, float scale,
                     int32_t accumulate, const sched_matrix* d_table, void* d_workspace,
                     size_t ws_bytes, void* hip_stream) {
  if (!d_rows || !tokens || !d_table) return SCHED_E_NULL;
  if (int e = check_matrix(*d_rows, false)) return e;
  if (int e = check_matrix(*d_table, true)) return e;
  if (int e = check_tokens(*tokens)) return e;
  if (d_rows->rows != tokens->n || d_rows->cols != d_table->cols || d_table->cols > kMostDim)
    return SCHED_E_SIZE;
  if ((d_table->dtype != d_rows->dtype && d_table->dtype != SCHED_F32) || !std::isfinite(scale) ||
      (accumulate != 0 && accumulate != 1))
    return SCHED_E_VALUE;
  if (int e = check_workspace(d_workspace, ws_bytes, embed_grad_bytes(tokens->n, d_table->cols)))
    return e;
  return done(launch_embed_grad(*d_rows, *tokens, scale, accumulate != 0, *d_table, d_workspace,
                                stream_of(hip_stream)));
}

int sched_token_logprobs(const sched_matrix* logits, const sched_tokens* tokens, float temperature,
                         float* logp, void* hip_stream) {
  if (!logits || !tokens) return SCHED_E_NULL;
  if (int e = check_logits(*logits, *tokens, temperature)) return e;
  if (tokens->n > 0 && !logp) return SCHED_E_NULL;
  return done(launch_logprobs(*logits, *tokens, temperature, logp, stream_of(hip_stream)));
}

int sched_token_logprobs_grad(const sched_matrix* logits, const sched_tokens* tokens,
                              float temperature, const float* logp, const float* d_logp,
                              const sched_matrix* d_logits, void* hip_stream) {
  if (!logits || !tokens || !d_logits) return SCHED_E_NULL;
  if (int e = check_logits(*logits, *tokens, temperature)) return e;
  if (int e = check_d_logits(*logits, *d_logits)) return e;
  if (tokens->n > 0 && (!logp || !d_logp)) return SCHED_E_NULL;
  return done(launch_logprobs_grad(*logits, *tokens, temperature, logp, d_logp, *d_logits,
                                   stream_of(hip_stream)));
}

int sched_group_advantages(const int64_t* makespan_us, const int64_t* limit_us,
                           const int32_t* group_offsets, int32_t n_groups, const int32_t* offsets,
                           int32_t n_answers, const sched_tokens* tokens, int32_t mean,
                           float* advantages, float* weights, void* d_workspace, size_t ws_bytes,
                           void* hip_stream) {
  if (!tokens) return SCHED_E_NULL;
  if (int e = check_tokens(*tokens)) return e;
  if (n_answers < 0 || n_answers > kMostAnswers || n_groups < 0 || (n_answers > 0 && n_groups < 1))
    return SCHED_E_SIZE;
  if (mean != 0 && mean != 1) return SCHED_E_VALUE;
  if (n_answers > 0 && (!makespan_us || !limit_us || !group_offsets || !offsets))
    return SCHED_E_NULL;
  if (tokens->n > 0 && (!advantages || !weights)) return SCHED_E_NULL;
  if (int e = check_workspace(d_workspace, ws_bytes, size_t(n_answers) * 4)) return e;
  return done(launch_advantages(makespan_us, limit_us, group_offsets, n_groups, offsets, n_answers,
                                *tokens, mean, advantages, weights,
                                static_cast<int32_t*>(d_workspace), stream_of(hip_stream)));
}

int sched_policy_loss(const sched_policy_desc* d, void* hip_stream) {
  if (!d) return SCHED_E_NULL;
  if (int e = check_logits(d->logits, d->tokens, d->temperature)) return e;
  if (int e = check_d_logits(d->logits, d->d_logits)) return e;
  if (!d->loss) return SCHED_E_NULL;
  if (d->tokens.n > 0 &&
      (!d->old_logp || !d->advantages || !d->weights || !d->losses || !d->logp ||
       (!d->ref_logp && d->kl_weight != 0)))
    return SCHED_E_NULL;
  if (!(d->clip_low >= 0) || !(d->clip_high >= 0) || !std::isfinite(d->clip_low) ||
      !std::isfinite(d->clip_high) || !std::isfinite(d->kl_weight) || !std::isfinite(d->loss_scale))
    return SCHED_E_VALUE;
  return done(launch_policy(*d, stream_of(hip_stream)));
}

int sched_preference_loss(const float* logp, const float* ref_logp, const sched_tokens* tokens,
                          const int32_t* offsets, int32_t n_pairs, float beta, float smoothing,
                          float loss_scale, float* loss, float* margins, float* d_logp,
                          void* hip_stream) {
  if (!tokens) return SCHED_E_NULL;
  if (int e = check_tokens(*tokens)) return e;
  if (n_pairs < 1 || n_pairs >= kMostPairs) return SCHED_E_SIZE;
  if (!offsets || !loss || !margins || (tokens->n > 0 && (!logp || !ref_logp || !d_logp)))
    return SCHED_E_NULL;
  if (!std::isfinite(beta) || !std::isfinite(loss_scale) || !(smoothing >= 0) || !(smoothing <= 1))
    return SCHED_E_VALUE;
  return done(launch_preference(logp, ref_logp, *tokens, offsets, n_pairs, beta, smoothing,
                                loss_scale, loss, margins, d_logp, stream_of(hip_stream)));
}

int sched_attention_workspace_bytes(const sched_attention_desc* d, size_t* out) {
  if (!d || !out) return SCHED_E_NULL;
  if (int e = check_attention_sizes(*d)) return e;
  *out = attention_bytes(*d);
  return SCHED_OK;
}

int sched_attention(const sched_attention_desc* d, void* d_workspace, size_t ws_bytes,
                    void* hip_stream) {
  if (!d) return SCHED_E_NULL;
  if (int e = check_attention(*d)) return e;
  if (int e = check_workspace(d_workspace, ws_bytes, attention_bytes(*d))) return e;
  return done(launch_attention(*d, d_workspace, stream_of(hip_stream)));
}

int sched_attention_grad_workspace_bytes(const sched_attention_desc* d, size_t* out) {
  if (!d || !out) return SCHED_E_NULL;
  if (int e = check_attention_sizes(*d)) return e;
  *out = attention_grad_bytes(*d);
  return SCHED_OK;
}

int sched_attention_grad(const sched_attention_desc* d, const sched_heads* d_out,
                         const sched_heads* d_q, const sched_heads* d_k, const sched_heads* d_v,
                         void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (!d || !d_out || !d_q || !d_k || !d_v) return SCHED_E_NULL;
  if (int e = check_attention(*d)) return e;
  if (int e = check_heads(*d_out, d->q_rows, d->q_heads, d->head_dim, false)) return e;
  if (int e = check_heads(*d_q, d->q_rows, d->q_heads, d->head_dim, true)) return e;
  if (int e = check_heads(*d_k, d->k_rows, d->kv_heads, d->head_dim, true)) return e;
  if (int e = check_heads(*d_v, d->k_rows, d->kv_heads, d->head_dim, true)) return e;
  if (int e = check_workspace(d_workspace, ws_bytes, attention_grad_bytes(*d))) return e;
  return done(launch_attention_grad(*d, *d_out, *d_q, *d_k, *d_v, d_workspace,
                                    stream_of(hip_stream)));
}

}  // extern "C"
