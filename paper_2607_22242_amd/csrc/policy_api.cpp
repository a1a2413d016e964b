// policy_api.cpp -- the C ABI of include/sched_policy.h: checks of arguments,
// then the launches.  Nothing here allocates or waits.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "policy_launch.h"

using namespace policy;

namespace {

constexpr int64_t kMostRows = (int64_t(1) << 31) - 1024;  // strides over rows stay in 32 bits
constexpr int64_t kMostDim = int64_t(1) << 24;    // of an embedding
constexpr int32_t kMostPairs = 1 << 23;
constexpr int32_t kMostAnswers = 1 << 16;         // every one's wave adds up all counts
constexpr int32_t kMostHeads = 1 << 16;
constexpr int32_t kMostBeams = 128;
constexpr int64_t kMostChoices = int64_t(1) << 22;  // logits that a beam chooses among
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

// The factor of the powers, log2(e) / temperature, is the largest that is used.
int check_temperature(float temperature) {
  if (!positive(temperature) || !std::isfinite(float(1.4426950408889634 / double(temperature))))
    return SCHED_E_VALUE;
  return SCHED_OK;
}

// A matrix of logits with a token per row and factors that can be used.
int check_logits(const sched_matrix& logits, const sched_tokens& tokens, float temperature) {
  if (int e = check_matrix(logits, false)) return e;
  if (int e = check_tokens(tokens)) return e;
  if (logits.rows != tokens.n || logits.cols < 1) return SCHED_E_SIZE;
  return check_temperature(temperature);
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

int check_shared_sizes(const sched_shared_desc& x) {
  const sched_attention_desc& d = x.own;
  if (int e = check_attention_sizes(d)) return e;
  if (x.n_groups < 0 || x.prefix_rows < 0 || x.prefix_rows > kMostRows) return SCHED_E_SIZE;
  // Blocks of both kinds are in one grid.
  const int64_t rows = d.q_rows * (d.q_heads / d.kv_heads);
  const int64_t q_tiles = rows / 32 * 2 + int64_t(d.n_seqs) + x.n_groups;
  const int64_t k_tiles = (d.k_rows + x.prefix_rows) / 64 + int64_t(d.n_seqs) + x.n_groups + 16;
  if (q_tiles * d.kv_heads >= kMostTiles || k_tiles * d.kv_heads >= kMostTiles) return SCHED_E_SIZE;
  return SCHED_OK;
}
int check_shared(const sched_shared_desc& x) {
  if (int e = check_shared_sizes(x)) return e;
  if (int e = check_attention(x.own)) return e;
  const sched_attention_desc& d = x.own;
  if (int e = check_heads(x.prefix_k, x.prefix_rows, d.kv_heads, d.head_dim, false)) return e;
  if (int e = check_heads(x.prefix_v, x.prefix_rows, d.kv_heads, d.head_dim, false)) return e;
  // Offsets are read for empty tensors too.
  if (x.n_groups > 0 &&
      (!x.prefix_offsets || !x.group_offsets || !d.q_offsets || !d.k_offsets))
    return SCHED_E_NULL;
  return SCHED_OK;
}

// Where tensors are the same memory they have to be the same rows and heads.
bool in_step(const sched_heads& a, const sched_heads& b) {
  return a.data != b.data || (a.row_stride == b.row_stride && a.head_stride == b.head_stride);
}

// Heads of 32-bit values are read in two such pieces: their alignment is the same.
int check_rotate_sizes(const sched_norm_rotate_desc& d) {
  if (element_bytes(d.dtype) == 0 || d.norm < 0 || d.norm > 1) return SCHED_E_VALUE;
  if (d.head_dim < 8 || d.head_dim > 256 || d.head_dim % 8 || d.q_heads < 1 || d.kv_heads < 1 ||
      d.q_heads > kMostHeads || d.kv_heads > kMostHeads || d.rows < 0 || d.rows > kMostRows)
    return SCHED_E_SIZE;
  return SCHED_OK;
}
int check_rotate(const sched_norm_rotate_desc& d) {
  if (int e = check_rotate_sizes(d)) return e;
  if (d.turned < 0 || d.turned > d.head_dim || d.turned % 2 || d.out_rows < 0 ||
      d.out_rows > kMostRows)
    return SCHED_E_SIZE;
  if (d.interleaved < 0 || d.interleaved > 1 || !std::isfinite(d.eps) || d.eps < 0 ||
      (!d.norm && (d.q_weight || d.k_weight)))
    return SCHED_E_VALUE;
  if (int e = check_tokens(d.positions)) return e;
  if (d.positions.n != d.rows) return SCHED_E_SIZE;
  if (d.places.data) {
    if (int e = check_tokens(d.places)) return e;
    if (d.places.n != d.rows) return SCHED_E_SIZE;
  } else if (d.out_rows != d.rows) {
    return SCHED_E_SIZE;
  }
  if (d.turned > 0 && !d.frequencies) return SCHED_E_NULL;
  if (int e = check_heads(d.q, d.rows, d.q_heads, d.head_dim, false)) return e;
  return check_heads(d.k, d.rows, d.kv_heads, d.head_dim, false);
}

int check_beam(const sched_beam_desc& d) {
  if (d.n_groups < 0 || d.n_groups > kMostBlocks || d.beams < 1 || d.beams > kMostBeams ||
      d.width < 1 || d.width > kMostBeams || d.logits.cols < 1 || d.logits.cols > kMostChoices)
    return SCHED_E_SIZE;
  if (int e = check_matrix(d.logits, false)) return e;
  if (d.logits.rows != int64_t(d.n_groups) * d.beams) return SCHED_E_SIZE;
  if (d.stay < 0 || d.stay > 1) return SCHED_E_VALUE;
  if (d.stay && d.width != d.beams) return SCHED_E_SIZE;
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

int sched_shared_attention_workspace_bytes(const sched_shared_desc* d, size_t* out) {
  if (!d || !out) return SCHED_E_NULL;
  if (int e = check_shared_sizes(*d)) return e;
  *out = shared_bytes(*d);
  return SCHED_OK;
}

int sched_shared_attention(const sched_shared_desc* d, void* d_workspace, size_t ws_bytes,
                           void* hip_stream) {
  if (!d) return SCHED_E_NULL;
  if (int e = check_shared(*d)) return e;
  if (int e = check_workspace(d_workspace, ws_bytes, shared_bytes(*d))) return e;
  return done(launch_shared(*d, d_workspace, stream_of(hip_stream)));
}

int sched_shared_attention_grad_workspace_bytes(const sched_shared_desc* d, size_t* out) {
  if (!d || !out) return SCHED_E_NULL;
  if (int e = check_shared_sizes(*d)) return e;
  *out = shared_grad_bytes(*d);
  return SCHED_OK;
}

int sched_shared_attention_grad(const sched_shared_desc* x, const sched_shared_grads* g,
                                void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (!x || !g) return SCHED_E_NULL;
  if (int e = check_shared(*x)) return e;
  const sched_attention_desc& d = x->own;
  if (int e = check_heads(g->d_out, d.q_rows, d.q_heads, d.head_dim, false)) return e;
  if (int e = check_heads(g->d_q, d.q_rows, d.q_heads, d.head_dim, true)) return e;
  if (int e = check_heads(g->d_k, d.k_rows, d.kv_heads, d.head_dim, true)) return e;
  if (int e = check_heads(g->d_v, d.k_rows, d.kv_heads, d.head_dim, true)) return e;
  if (int e = check_heads(g->d_prefix_k, x->prefix_rows, d.kv_heads, d.head_dim, true)) return e;
  if (int e = check_heads(g->d_prefix_v, x->prefix_rows, d.kv_heads, d.head_dim, true)) return e;
  if (int e = check_workspace(d_workspace, ws_bytes, shared_grad_bytes(*x))) return e;
  return done(launch_shared_grad(*x, *g, d_workspace, stream_of(hip_stream)));
}

int sched_norm_rotate(const sched_norm_rotate_desc* d, void* hip_stream) {
  if (!d) return SCHED_E_NULL;
  if (int e = check_rotate(*d)) return e;
  const int32_t dim = d->head_dim, heads = d->kv_heads;
  const bool placed = d->places.data != nullptr, values = d->v.data != nullptr;
  if (int e = check_heads(d->q_out, d->rows, d->q_heads, dim, true)) return e;
  if (int e = check_heads(d->k_out, d->out_rows, heads, dim, true)) return e;
  if (values) {
    if (int e = check_heads(d->v, d->rows, heads, dim, false)) return e;
    if (int e = check_heads(d->v_out, d->out_rows, heads, dim, true)) return e;
  }
  // In place is the same rows and heads; a row that goes to another's place is not.
  // Without rows tensors have no memory, and one address.
  if (d->rows > 0 && (!in_step(d->q, d->q_out) || !in_step(d->k, d->k_out) ||
                      (values && !in_step(d->v, d->v_out))))
    return SCHED_E_VALUE;
  if (placed && d->rows > 0 &&
      (d->k.data == d->k_out.data || (values && d->v.data == d->v_out.data)))
    return SCHED_E_VALUE;
  return done(launch_norm_rotate(*d, stream_of(hip_stream)));
}

int sched_norm_rotate_grad_workspace_bytes(const sched_norm_rotate_desc* d, size_t* out) {
  if (!d || !out) return SCHED_E_NULL;
  if (int e = check_rotate_sizes(*d)) return e;
  *out = norm_rotate_grad_bytes(*d);
  return SCHED_OK;
}

int sched_norm_rotate_grad(const sched_norm_rotate_desc* d, const sched_heads* d_q_out,
                           const sched_heads* d_k_out, const sched_heads* d_q,
                           const sched_heads* d_k, float* d_q_weight, float* d_k_weight,
                           void* d_workspace, size_t ws_bytes, void* hip_stream) {
  if (!d || !d_q_out || !d_k_out || !d_q || !d_k) return SCHED_E_NULL;
  if (int e = check_rotate(*d)) return e;
  const int32_t dim = d->head_dim;
  if (int e = check_heads(*d_q_out, d->rows, d->q_heads, dim, false)) return e;
  if (int e = check_heads(*d_k_out, d->out_rows, d->kv_heads, dim, false)) return e;
  if (int e = check_heads(*d_q, d->rows, d->q_heads, dim, true)) return e;
  if (int e = check_heads(*d_k, d->rows, d->kv_heads, dim, true)) return e;
  if (!d->norm && (d_q_weight || d_k_weight)) return SCHED_E_VALUE;
  if (d->rows > 0 &&
      (!in_step(*d_q, d->q) || !in_step(*d_q, *d_q_out) || !in_step(*d_k, d->k) ||
       !in_step(*d_k, *d_k_out) || (d->places.data && d_k->data == d_k_out->data)))
    return SCHED_E_VALUE;
  if (d_q_weight || d_k_weight)
    if (int e = check_workspace(d_workspace, ws_bytes, norm_rotate_grad_bytes(*d))) return e;
  return done(launch_norm_rotate_grad(*d, *d_q_out, *d_k_out, *d_q, *d_k, d_q_weight, d_k_weight,
                                      d_workspace, stream_of(hip_stream)));
}

int sched_beam_workspace_bytes(const sched_beam_desc* d, size_t* out) {
  if (!d || !out) return SCHED_E_NULL;
  if (int e = check_beam(*d)) return e;
  *out = beam_bytes(*d);
  return SCHED_OK;
}

int sched_beam_select(const sched_beam_desc* d, void* d_workspace, size_t ws_bytes,
                      void* hip_stream) {
  if (!d) return SCHED_E_NULL;
  if (int e = check_beam(*d)) return e;
  if (d->last.data) {
    if (int e = check_tokens(d->last)) return e;
    if (d->last.n != d->logits.rows) return SCHED_E_SIZE;
  }
  const sched_tokens tokens = {d->tokens, d->token_bits, int64_t(d->n_groups) * d->width};
  if (int e = check_tokens(tokens)) return e;
  if (d->end_token < -1 || (d->token_bits == 32 && d->end_token > INT32_MAX)) return SCHED_E_VALUE;
  if (int e = check_temperature(d->temperature)) return e;
  if (d->n_groups > 0 && (!d->scores || !d->new_scores || !d->parents)) return SCHED_E_NULL;
  // In place a group's results take the place of its own beams, which it alone reads.
  if (d->n_groups > 0 && ((d->new_scores == d->scores && d->width != d->beams) ||
                          (d->last.data && d->tokens == d->last.data &&
                           (d->width != d->beams || d->token_bits != d->last.bits))))
    return SCHED_E_VALUE;
  if (int e = check_workspace(d_workspace, ws_bytes, beam_bytes(*d))) return e;
  return done(launch_beam_select(*d, d_workspace, stream_of(hip_stream)));
}

int sched_beam_reorder(const sched_states* x, const int32_t* parents, const int32_t* lengths,
                       int32_t beams, void* hip_stream) {
  if (!x) return SCHED_E_NULL;
  if (beams < 1 || beams > kMostBeams || x->outer < 0 || x->slots < 0 || x->rows < 0 ||
      x->row_bytes < 0 || x->slots > kMostRows || x->slots % beams || x->rows > kMostRows ||
      x->row_bytes > kMostRows || x->outer > kMostRows)
    return SCHED_E_SIZE;
  if (x->outer == 0 || x->slots == 0 || x->rows == 0 || x->row_bytes == 0) return SCHED_OK;
  if (!x->data || !parents) return SCHED_E_NULL;
  // Rows, slots and tensors one behind the other, in this order or with the
  // slots outermost: none may overlap.
  if (x->row_stride < 0 || x->slot_stride < 0 || x->outer_stride < 0) return SCHED_E_VALUE;
  struct Axis {
    int64_t n, stride;
  } axes[3] = {{x->rows, x->row_stride}, {x->slots, x->slot_stride}, {x->outer, x->outer_stride}};
  std::sort(axes, axes + 3, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
  int64_t extent = x->row_bytes;
  for (const Axis& axis : axes) {
    if (axis.n == 1) continue;
    if (axis.stride < extent || axis.stride > (int64_t(1) << 62) / axis.n) return SCHED_E_VALUE;
    extent = axis.stride * (axis.n - 1) + extent;
  }
  return done(launch_beam_reorder(*x, parents, lengths, beams, stream_of(hip_stream)));
}

}  // extern "C"
