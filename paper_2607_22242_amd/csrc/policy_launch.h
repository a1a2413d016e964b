// policy_launch.h -- host-side entry points into the kernels of sched_policy.h
// (internal): arguments have been checked.
#pragma once
#include <hip/hip_runtime.h>

#include "sched_policy.h"

namespace policy {

// Blocks of a launch at most (a grid has less than 2^32 threads a side); more
// work is launched in parts.
constexpr int64_t kMostBlocks = (int64_t(1) << 22) - 1;

// Bytes of the matrix' element, 0 for a type that is not taken.
inline int element_bytes(int32_t dtype) {
  return dtype == SCHED_F32 ? 4 : dtype == SCHED_F16 || dtype == SCHED_BF16 ? 2 : 0;
}

hipError_t launch_embed(const sched_matrix& table, const sched_tokens& tokens, float scale,
                        const sched_matrix& out, hipStream_t s);
size_t embed_grad_bytes(int64_t n, int64_t dim);
hipError_t launch_embed_grad(const sched_matrix& d_rows, const sched_tokens& tokens, float scale,
                             bool accumulate, const sched_matrix& d_table, void* ws, hipStream_t s);
hipError_t launch_logprobs(const sched_matrix& logits, const sched_tokens& tokens,
                           float temperature, float* logp, hipStream_t s);
hipError_t launch_logprobs_grad(const sched_matrix& logits, const sched_tokens& tokens,
                                float temperature, const float* logp, const float* d_logp,
                                const sched_matrix& d_logits, hipStream_t s);
hipError_t launch_advantages(const int64_t* makespan, const int64_t* limit, const int32_t* groups,
                             int32_t n_groups, const int32_t* offsets, int32_t n_answers,
                             const sched_tokens& tokens, int32_t mean, float* advantages,
                             float* weights, int32_t* counts, hipStream_t s);
hipError_t launch_policy(const sched_policy_desc& d, hipStream_t s);
hipError_t launch_preference(const float* logp, const float* ref, const sched_tokens& tokens,
                             const int32_t* offsets, int32_t n_pairs, float beta, float smoothing,
                             float loss_scale, float* loss, float* margins, float* d_logp,
                             hipStream_t s);
size_t attention_bytes(const sched_attention_desc& d);
hipError_t launch_attention(const sched_attention_desc& d, void* ws, hipStream_t s);
size_t attention_grad_bytes(const sched_attention_desc& d);
hipError_t launch_attention_grad(const sched_attention_desc& d, const sched_heads& d_out,
                                 const sched_heads& d_q, const sched_heads& d_k,
                                 const sched_heads& d_v, void* ws, hipStream_t s);
size_t shared_bytes(const sched_shared_desc& d);
hipError_t launch_shared(const sched_shared_desc& d, void* ws, hipStream_t s);
size_t shared_grad_bytes(const sched_shared_desc& d);
hipError_t launch_shared_grad(const sched_shared_desc& d, const sched_shared_grads& g, void* ws,
                              hipStream_t s);
hipError_t launch_norm_rotate(const sched_norm_rotate_desc& d, hipStream_t s);
size_t norm_rotate_grad_bytes(const sched_norm_rotate_desc& d);
hipError_t launch_norm_rotate_grad(const sched_norm_rotate_desc& d, const sched_heads& d_q_out,
                                   const sched_heads& d_k_out, const sched_heads& d_q,
                                   const sched_heads& d_k, float* d_q_weight, float* d_k_weight,
                                   void* ws, hipStream_t s);
size_t beam_bytes(const sched_beam_desc& d);
hipError_t launch_beam_select(const sched_beam_desc& d, void* ws, hipStream_t s);
hipError_t launch_beam_reorder(const sched_states& x, const int32_t* parents,
                               const int32_t* lengths, int32_t beams, hipStream_t s);

}  // namespace policy
