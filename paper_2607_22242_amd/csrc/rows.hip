// rows.hip -- rows of logits: log-probabilities of tokens, their gradient, and
// the clipped policy loss with the logits' gradient; and the small sums around
// them (advantages, weights, the preference loss).
//
// A row x of V logits, z = x / T, gives lse = log sum_j exp z_j and for its
// token t the log-probability l = z_t - lse; a factor g on l moves the logits
// by g (e_t - exp(z - lse)) / T.  All in base 2: z_j log2(e) = x_j c with
// c = log2(e) / T, and the difference to the row's maximum (or to x_t, where l
// is known) is taken before the product, so that rows of a type's lowest
// value do not overflow.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "policy_launch.h"
#include "tensors.h"

namespace policy {
namespace {

constexpr int kRowThreads = 256;

struct RowArgs {
  const void* logits;
  int64_t n, vocab, stride;
  int64_t first;   // row that the launch starts with
  Tokens tokens;
  float c, inv_t;  // log2(e) / T, 1 / T
  // log-probabilities
  float* logp;
  // gradient
  const float* logp_in;
  const float* d_logp;
  void* d_logits;
  int64_t d_stride;
  // policy loss
  const float *old_logp, *ref_logp, *advantages, *weights;
  float lo, hi, kl, loss_scale;
  float* losses;
};

// Maximum and sum of powers of part of a row: sum_j 2^((x_j - m) c) = s.
struct Soft {
  float m, s;
};

// 0 in place of a maximum of -inf: powers of -inf then are zeros.
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ Soft join(Soft a, Soft b, float c) {
  const float m = fmaxf(a.m, b.m), f = finite_max(m);
  return {m, a.s * pow2((a.m - f) * c) + b.s * pow2((b.m - f) * c)};
}

template <int N>
__device__ __forceinline__ void take(Soft& a, const float (&x)[N], float c) {
  float m = a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  const float f = finite_max(m);
  float s = a.s * pow2((a.m - f) * c);
#pragma unroll
  for (int i = 0; i < N; ++i) s += pow2((x[i] - f) * c);
  a = {m, s};
}

__device__ __forceinline__ Soft wave_join(Soft a, float c) {
#pragma unroll
  for (int d = 32; d; d >>= 1) a = join(a, {__shfl_xor(a.m, d), __shfl_xor(a.s, d)}, c);
  return a;
}

__device__ __forceinline__ Soft block_join(Soft a, float c, Soft* part) {
  a = wave_join(a, c);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = a;
  __syncthreads();
  a = part[0];
  for (int i = 1; i < int(blockDim.x) / kWave; ++i) a = join(a, part[i], c);
  return a;
}

// Log-probability of a token with logit x in a row with these statistics.
__device__ __forceinline__ float log_prob(float x, Soft r, float c) {
  return r.s == 0.f ? -INFINITY : ((x - finite_max(r.m)) * c - log_2(r.s)) * kLn2;
}

template <class T, int N>
__device__ __forceinline__ void widen(float (&x)[N], typename Vec<T>::type v) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = float(v[i]);
}

// Statistics of a row, read once by a block.
template <class T>
__device__ __forceinline__ Soft row_soft(const T* row, int64_t vocab, float c, Soft* part) {
  constexpr int N = Vec<T>::kN;
  Soft a = {-INFINITY, 0.f};
  const int64_t whole = vocab / N * N;
  for (int64_t j = int64_t(threadIdx.x) * N; j < whole; j += kRowThreads * N) {
    float x[N];
    widen<T>(x, load16(row + j));
    take(a, x, c);
  }
  if (whole + threadIdx.x < vocab) {
    const float x[1] = {float(row[whole + threadIdx.x])};
    take(a, x, c);
  }
  return block_join(a, c, part);
}

// d_logits of a row: gain (e_t - 2^((x - f) c + u)).  Every element is read
// and written by the same thread, so that the two may be one.
template <class T>
__device__ __forceinline__ void row_grad(const T* row, T* out, int64_t vocab, float c, float f,
                                         float u, float gain, int64_t t) {
  constexpr int N = Vec<T>::kN;
  const int64_t whole = vocab / N * N;
  for (int64_t j = int64_t(threadIdx.x) * N; j < whole; j += kRowThreads * N) {
    float x[N];
    widen<T>(x, load16(row + j));
    typename Vec<T>::type v;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float p = pow2(__builtin_fmaf(x[i] - f, c, u));
      v[i] = T(gain * (j + i == t ? 1.f - p : -p));
    }
    store16(out + j, v);
  }
  const int64_t j = whole + threadIdx.x;
  if (j < vocab) {
    const float p = pow2(__builtin_fmaf(float(row[j]) - f, c, u));
    out[j] = T(gain * (j == t ? 1.f - p : -p));
  }
}

template <class T>
__device__ __forceinline__ void row_zero(T* out, int64_t vocab) {
  constexpr int N = Vec<T>::kN;
  const int64_t whole = vocab / N * N;
  for (int64_t j = int64_t(threadIdx.x) * N; j < whole; j += kRowThreads * N)
    store16(out + j, typename Vec<T>::type(T(0)));
  if (whole + threadIdx.x < vocab) out[whole + threadIdx.x] = T(0);
}

template <class T>
__global__ __launch_bounds__(kRowThreads) void logprobs_kernel(RowArgs a) {
  __shared__ Soft part[kRowThreads / kWave];
  const int64_t i = a.first + blockIdx.x;
  const int64_t t = token_in(a.tokens, i, a.vocab);
  if (t < 0) {
    if (threadIdx.x == 0) a.logp[i] = 0.f;
    return;
  }
  const T* row = static_cast<const T*>(a.logits) + i * a.stride;
  const Soft r = row_soft(row, a.vocab, a.c, part);
  if (threadIdx.x == 0) a.logp[i] = log_prob(float(row[t]), r, a.c);
}

template <class T>
__global__ __launch_bounds__(kRowThreads) void logprobs_grad_kernel(RowArgs a) {
  const int64_t i = a.first + blockIdx.x;
  const int64_t t = token_in(a.tokens, i, a.vocab);
  T* out = static_cast<T*>(a.d_logits) + i * a.d_stride;
  const float l = a.logp_in[i];
  if (t < 0 || l == -INFINITY) return row_zero(out, a.vocab);
  const T* row = static_cast<const T*>(a.logits) + i * a.stride;
  const float xt = float(row[t]);
  __syncthreads();  // every thread has the token's logit before one writes there
  row_grad(row, out, a.vocab, a.c, xt, l * kLog2e, a.d_logp[i] * a.inv_t, t);
}

// Loss of one token with log-probability l, and its derivative.
struct TokenLoss {
  float loss, slope;
};
__device__ __forceinline__ TokenLoss token_loss(const RowArgs& a, int64_t i, float l) {
  const float w = a.weights[i], adv = a.advantages[i];
  const float r = pow2((l - a.old_logp[i]) * kLog2e);
  const float free = -adv * r, held = -adv * fminf(fmaxf(r, a.lo), a.hi);
  float loss = fmaxf(free, held), slope = free >= held ? free : 0.f;
  if (a.kl != 0.f) {
    const float e = a.ref_logp[i] - l, k = pow2(e * kLog2e);
    loss += a.kl * (k - e - 1.f);
    slope += a.kl * (1.f - k);
  }
  return {w * loss, w * slope * a.loss_scale};
}

template <class T>
__global__ __launch_bounds__(kRowThreads) void policy_kernel(RowArgs a) {
  __shared__ Soft part[kRowThreads / kWave];
  const int64_t i = a.first + blockIdx.x;
  const int64_t t = token_in(a.tokens, i, a.vocab);
  T* out = static_cast<T*>(a.d_logits) + i * a.d_stride;
  if (t < 0) {
    if (threadIdx.x == 0) a.losses[i] = a.logp[i] = 0.f;
    return row_zero(out, a.vocab);
  }
  const T* row = static_cast<const T*>(a.logits) + i * a.stride;
  const float xt = float(row[t]);
  const Soft r = row_soft(row, a.vocab, a.c, part);
  const float l = log_prob(xt, r, a.c);
  const TokenLoss k = token_loss(a, i, l);
  if (threadIdx.x == 0) {
    a.losses[i] = k.loss;
    a.logp[i] = l;
  }
  if (l == -INFINITY) return row_zero(out, a.vocab);
  row_grad(row, out, a.vocab, a.c, finite_max(r.m), -log_2(r.s), k.slope * a.inv_t, t);
}

// loss[0] = scale * the sum of n values, added in a fixed order in 64 bits.
__global__ __launch_bounds__(1024) void total_kernel(const float* __restrict__ x, int64_t n,
                                                     float scale, float* loss) {
  __shared__ double part[16];
  double s = 0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += double(x[i]);
  s = block_sum(s, part);
  if (threadIdx.x == 0) loss[0] = float(s * scale);
}

// Tokens that are no padding, per answer; a wave each.
__global__ __launch_bounds__(256) void count_kernel(const int32_t* offsets, int n_answers,
                                                    Tokens tokens, int n, int32_t* counts) {
  const int a = int(blockIdx.x) * 4 + int(threadIdx.x) / kWave;
  if (a >= n_answers) return;
  const int b = offset_at(offsets, a, n), e = offset_at(offsets, a + 1, n);
  int c = 0;
  for (int i = b + int(threadIdx.x) % kWave; i < e; i += kWave) c += token_at(tokens, i) >= 0;
#pragma unroll
  for (int d = 32; d; d >>= 1) c += __shfl_xor(c, d);
  if (threadIdx.x % kWave == 0) counts[a] = c;
}

struct AdvArgs {
  const int64_t *makespan, *limit;
  const int32_t *groups, *offsets, *counts;
  int32_t n_groups, n_answers, n, mean;
  Tokens tokens;
  float *advantages, *weights;
};

// A wave per answer: its group's mean and deviation in 64 bits, the number the
// weights are divided by, then its tokens.
__global__ __launch_bounds__(256) void advantages_kernel(AdvArgs a) {
  const int id = int(blockIdx.x) * 4 + int(threadIdx.x) / kWave, lane = int(threadIdx.x) % kWave;
  if (id >= a.n_answers) return;
  const int g = sequence_of(a.groups, a.n_groups, id);
  const int b = offset_at(a.groups, g, a.n_answers), e = offset_at(a.groups, g + 1, a.n_answers);
  const int64_t cap = a.limit[g];
  double sum = 0, most = -1e300, least = 1e300;
  for (int i = b + lane; i < e; i += kWave) {
    const double m = double(a.makespan[i] < cap ? a.makespan[i] : cap);
    sum += m;
    most = fmax(most, m);
    least = fmin(least, m);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    sum += __shfl_xor(sum, d);
    most = fmax(most, __shfl_xor(most, d));
    least = fmin(least, __shfl_xor(least, d));
  }
  const int size = e - b;
  const double mean = size > 0 ? sum / size : 0;
  double var = 0;
  for (int i = b + lane; i < e; i += kWave) {
    const double m = double(a.makespan[i] < cap ? a.makespan[i] : cap) - mean;
    var += m * m;
  }
  int64_t parts = 0;  // tokens, or answers with tokens
  for (int i = lane; i < a.n_answers; i += kWave)
    parts += a.mean ? int64_t(a.counts[i] > 0) : int64_t(a.counts[i]);
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    var += __shfl_xor(var, d);
    parts += __shfl_xor(parts, d);
  }
  const double own = double(a.makespan[id] < cap ? a.makespan[id] : cap);
  const bool in = id >= b && id < e;
  const float adv = in && most > least ? float((mean - own) / sqrt(var / size)) : 0.f;
  const int count = a.counts[id];
  const float w = count > 0 ? float(1.0 / (double(parts) * (a.mean ? double(count) : 1.0))) : 0.f;
  const int first = offset_at(a.offsets, id, a.n), last = offset_at(a.offsets, id + 1, a.n);
  for (int i = first + lane; i < last; i += kWave) {
    a.advantages[i] = adv;
    a.weights[i] = token_at(a.tokens, i) >= 0 ? w : 0.f;
  }
}

struct PairArgs {
  const float *logp, *ref;
  Tokens tokens;
  const int32_t* offsets;
  int32_t n, n_pairs;
  float beta, smoothing, loss_scale;
  float *margins, *d_logp;
};

// A block per pair: both sums of differences in 64 bits (a sequence's
// log-probabilities add up to thousands, a margin is of order one), the
// margin, and the slope to every token.
__global__ __launch_bounds__(256) void pairs_kernel(PairArgs a) {
  __shared__ double part[4];
  const int p = int(blockIdx.x);
  const int b = offset_at(a.offsets, 2 * p, a.n), c = offset_at(a.offsets, 2 * p + 1, a.n),
            e = offset_at(a.offsets, 2 * p + 2, a.n);
  double sum = 0;
  for (int i = b + int(threadIdx.x); i < e; i += 256)
    if (token_at(a.tokens, i) >= 0) {
      const double d = double(a.logp[i]) - double(a.ref[i]);
      sum += i < c ? d : -d;
    }
  const double m = double(a.beta) * block_sum(sum, part);
  if (threadIdx.x == 0) a.margins[p] = float(m);
  // d loss / d m = -(1 - eps) s(-m) + eps s(m)
  const double eps = a.smoothing;
  const double slope = eps / (1 + exp(-m)) - (1 - eps) / (1 + exp(m));
  const float d = float(double(a.loss_scale) * double(a.beta) * slope / a.n_pairs);
  for (int i = b + int(threadIdx.x); i < e; i += 256)
    a.d_logp[i] = token_at(a.tokens, i) >= 0 ? (i < c ? d : -d) : 0.f;
}

// Mean of the pairs' losses: -log s(m) = max(-m, 0) + log(1 + exp(-|m|)).
__global__ __launch_bounds__(1024) void pairs_total_kernel(const float* margins, int n,
                                                           float smoothing, float scale,
                                                           float* loss) {
  __shared__ double part[16];
  const double eps = smoothing;
  double s = 0;
  for (int i = int(threadIdx.x); i < n; i += 1024) {
    const double m = margins[i], soft = log1p(exp(-fabs(m)));
    s += soft + (1 - eps) * fmax(-m, 0.0) + eps * fmax(m, 0.0);
  }
  s = block_sum(s, part);
  if (threadIdx.x == 0) loss[0] = float(s * double(scale) / n);
}

template <template <class> class K>
hipError_t by_type(int32_t dtype, RowArgs a, hipStream_t s) {
  hipError_t e = hipSuccess;
  for (a.first = 0; a.first < a.n && e == hipSuccess; a.first += kMostBlocks) {
    const dim3 grid(unsigned(std::min(a.n - a.first, kMostBlocks))), block(kRowThreads);
    if (dtype == SCHED_F32) hipLaunchKernelGGL(K<float>::fn, grid, block, 0, s, a);
    else if (dtype == SCHED_F16) hipLaunchKernelGGL(K<f16>::fn, grid, block, 0, s, a);
    else hipLaunchKernelGGL(K<bf16>::fn, grid, block, 0, s, a);
    e = hipGetLastError();
  }
  return e;
}
template <class T> struct LogprobsK { static constexpr auto fn = logprobs_kernel<T>; };
template <class T> struct LogprobsGradK { static constexpr auto fn = logprobs_grad_kernel<T>; };
template <class T> struct PolicyK { static constexpr auto fn = policy_kernel<T>; };

Tokens tokens_of(const sched_tokens& t) { return {t.data, t.bits == 64}; }

RowArgs row_args(const sched_matrix& logits, const sched_tokens& tokens, float temperature) {
  RowArgs a = {};
  a.logits = logits.data;
  a.n = logits.rows;
  a.vocab = logits.cols;
  a.stride = logits.stride;
  a.tokens = tokens_of(tokens);
  a.c = float(1.4426950408889634 / double(temperature));
  a.inv_t = float(1.0 / double(temperature));
  return a;
}

}  // namespace

hipError_t launch_logprobs(const sched_matrix& logits, const sched_tokens& tokens,
                           float temperature, float* logp, hipStream_t s) {
  RowArgs a = row_args(logits, tokens, temperature);
  a.logp = logp;
  return by_type<LogprobsK>(logits.dtype, a, s);
}

hipError_t launch_logprobs_grad(const sched_matrix& logits, const sched_tokens& tokens,
                                float temperature, const float* logp, const float* d_logp,
                                const sched_matrix& d_logits, hipStream_t s) {
  RowArgs a = row_args(logits, tokens, temperature);
  a.logp_in = logp;
  a.d_logp = d_logp;
  a.d_logits = d_logits.data;
  a.d_stride = d_logits.stride;
  return by_type<LogprobsGradK>(logits.dtype, a, s);
}

hipError_t launch_policy(const sched_policy_desc& d, hipStream_t s) {
  RowArgs a = row_args(d.logits, d.tokens, d.temperature);
  a.old_logp = d.old_logp;
  a.ref_logp = d.ref_logp;
  a.advantages = d.advantages;
  a.weights = d.weights;
  a.lo = 1.f - d.clip_low;
  a.hi = 1.f + d.clip_high;
  a.kl = d.kl_weight;
  a.loss_scale = d.loss_scale;
  a.losses = d.losses;
  a.logp = d.logp;
  a.d_logits = d.d_logits.data;
  a.d_stride = d.d_logits.stride;
  const hipError_t e = by_type<PolicyK>(d.logits.dtype, a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(total_kernel, dim3(1), dim3(1024), 0, s, d.losses, d.logits.rows, 1.f, d.loss);
  return hipGetLastError();
}

hipError_t launch_advantages(const int64_t* makespan, const int64_t* limit, const int32_t* groups,
                             int32_t n_groups, const int32_t* offsets, int32_t n_answers,
                             const sched_tokens& tokens, int32_t mean, float* advantages,
                             float* weights, int32_t* counts, hipStream_t s) {
  if (n_answers == 0) return hipSuccess;
  const dim3 grid(static_cast<unsigned>((n_answers + 3) / 4)), block(256);
  hipLaunchKernelGGL(count_kernel, grid, block, 0, s, offsets, n_answers, tokens_of(tokens),
                     int(tokens.n), counts);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const AdvArgs a = {makespan, limit, groups, offsets, counts, n_groups, n_answers, int(tokens.n),
                     mean, tokens_of(tokens), advantages, weights};
  hipLaunchKernelGGL(advantages_kernel, grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_preference(const float* logp, const float* ref, const sched_tokens& tokens,
                             const int32_t* offsets, int32_t n_pairs, float beta, float smoothing,
                             float loss_scale, float* loss, float* margins, float* d_logp,
                             hipStream_t s) {
  const PairArgs a = {logp, ref, tokens_of(tokens), offsets, int(tokens.n), n_pairs, beta,
                      smoothing, loss_scale, margins, d_logp};
  hipLaunchKernelGGL(pairs_kernel, dim3(unsigned(n_pairs)), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(pairs_total_kernel, dim3(1), dim3(1024), 0, s, margins, n_pairs, smoothing,
                     loss_scale, loss);
  return hipGetLastError();
}

}  // namespace policy
