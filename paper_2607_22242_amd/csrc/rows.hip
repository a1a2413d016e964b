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

struct RowArgs {
  const void* logits;
  int64_t n, vocab, stride;
  int64_t first;   // row that the launch starts with
  Tokens tokens;
  float t, c, inv_t;  // T, log2(e) / T, 1 / T
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

// What a row's gradient takes its probabilities from, p_j = k 2^((x_j - f) c + u):
// its statistics (f the maximum, k one over the sum: the large ones then have
// small exponents, which are rounded least), or a token's logit and
// log-probability.  d_j = gain (e_t - p_j).
struct Grad {
  float f, u, gain, gain_k;
  __device__ __forceinline__ float at(float x, float c, bool token) const {
    return __builtin_fmaf(-gain_k, pow2(__builtin_fmaf(x - f, c, u)), token ? gain : 0.f);
  }
};

// 0 in place of a maximum of -inf: powers of -inf then are zeros.
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ Grad grad_of(Soft a, float gain) {
  return {finite_max(a.m), 0.f, gain, gain / a.s};
}

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

// Log-probability of a token with logit x in a row with these statistics.  Not in
// base 2, where the type's lowest logit, a mask, would leave the range; and by
// T itself: a rounded factor shifts all of a loss's terms the same way, which
// shows in their sum.
__device__ __forceinline__ float log_prob(const RowArgs& a, float x, Soft r) {
  return r.s == 0.f ? -INFINITY : (x - finite_max(r.m)) / a.t - ln(r.s);
}

template <class T, int N>
__device__ __forceinline__ void widen(float (&x)[N], typename Vec<T>::type v) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = float(v[i]);
}

// How a row is taken.  Rows of up to 64 logits: a power of two of lanes each, a
// logit a lane.  Rows whose 16-byte pieces fit the registers of a wave or of a
// block (kVecs pieces a thread): read once, so that a loss with its gradient
// costs one read and one write.  Longer ones: read twice by a block of 1024,
// two of which fill a unit: no more rows are under way than the last cache
// holds, and the second read comes from there.  131072 logits in bf16 (8,000
// rows): 885 us; when block sizes were compared 0.95 ms so, 1.15 with blocks of 512
// and 1.22 with 256.
constexpr int kBlock = 256;  // of rows of lanes or waves
constexpr int kLongThreads = 1024;

// A row's logits in registers: pieces i * kThreads + t of thread t, and one of
// the logits behind the last whole piece.
template <class T, int kThreads, int kVecs>
struct Held {
  static constexpr int N = Vec<T>::kN;
  typedef typename Vec<T>::type V;
  V v[kVecs];
  float tail;

  __device__ __forceinline__ void load(const T* row, int vocab, int t) {
    const int pieces = vocab / N;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      v[i] = V(T(-INFINITY));
      if (i * kThreads + t < pieces) v[i] = load16(row + int64_t(i * kThreads + t) * N);
    }
    tail = -INFINITY;
    if (pieces * N + t < vocab) tail = float(row[pieces * N + t]);
  }
  // Keeps the compiler from holding the logits in 32 bits too between two uses,
  // which takes twice the registers.
  __device__ __forceinline__ void fresh() {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      typedef uint32_t Raw __attribute__((ext_vector_type(4)));
      Raw x = __builtin_bit_cast(Raw, v[i]);
      asm volatile("" : "+v"(x));
      v[i] = __builtin_bit_cast(V, x);
    }
  }
  __device__ __forceinline__ float most() const {
    float m = tail;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) m = fmaxf(m, float(v[i][e]));
    return m;
  }
  __device__ __forceinline__ float sum(float f, float c) const {
    float s = pow2((tail - f) * c);
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) s += pow2((float(v[i][e]) - f) * c);
    return s;
  }
  // The gradient to the row's place.
  __device__ __forceinline__ void store(T* out, int vocab, int t, float c, const Grad& g,
                                        int token) const {
    const int pieces = vocab / N;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int at = (i * kThreads + t) * N;
      if (i * kThreads + t >= pieces) continue;
      V d;
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = T(g.at(float(v[i][e]), c, at + e == token));
      store16(out + at, d);
    }
    const int at = pieces * N + t;
    if (at < vocab) out[at] = T(g.at(tail, c, at == token));
  }
  __device__ __forceinline__ static void zero(T* out, int vocab, int t) {
    const int pieces = vocab / N;
    for (int i = t; i < pieces; i += kThreads) store16(out + int64_t(i) * N, V(T(0)));
    if (pieces * N + t < vocab) out[pieces * N + t] = T(0);
  }
};

// Loss of one token with log-probability l, and its derivative.
struct TokenLoss {
  float loss, slope;
};
__device__ __forceinline__ TokenLoss token_loss(const RowArgs& a, int64_t i, float l) {
  const float w = a.weights[i], adv = a.advantages[i];
  const float r = pow2((l - a.old_logp[i]) * kLog2e);
  // By comparisons that keep what is no number, where fmin and fmax drop it.  A
  // ratio beyond 32 bits times an advantage of 0 is 0.
  const float free = adv == 0.f && r == INFINITY ? 0.f : -adv * r;
  const float held = -adv * (r < a.lo ? a.lo : r > a.hi ? a.hi : r);
  float loss = held > free ? held : free, slope = held > free ? 0.f : free;
  if (a.kl != 0.f) {
    // exp(e) - 1 as such: e is mostly small, and the term is of its square.
    const float e = a.ref_logp[i] - l, k = expm1f(e);
    loss += a.kl * (k == INFINITY ? k : k - e);
    slope -= a.kl * k;
  }
  return {w * loss, w * slope * a.loss_scale};
}

// What a row is taken for: its token's log-probability, the policy loss with the
// gradient, or the gradient of log-probabilities that are known.
enum For { kLogp, kPolicy, kGrad };

// `lanes` (a power of two up to 64) of a wave take a row of at most as many
// logits, lane t of them logit t.
template <class T>
__device__ __forceinline__ Soft lanes_soft(const RowArgs& a, int64_t i, int t, bool on, int lanes,
                                           float& x) {
  x = on && t < int(a.vocab) ? float(static_cast<const T*>(a.logits)[i * a.stride + t]) : -INFINITY;
  Soft r = {x, 0.f};
  for (int d = 1; d < lanes; d <<= 1) r.m = fmaxf(r.m, __shfl_xor(r.m, d));
  r.s = pow2((x - finite_max(r.m)) * a.c);
  for (int d = 1; d < lanes; d <<= 1) r.s += __shfl_xor(r.s, d);
  return r;
}

template <class T, For kFor>
__global__ __launch_bounds__(kBlock) void lanes_kernel(RowArgs a, int lanes) {
  const int64_t i = a.first + int64_t(blockIdx.x) * (kBlock / lanes) + int(threadIdx.x) / lanes;
  if (i >= a.n) return;  // all of a row's lanes
  const int t = int(threadIdx.x) % lanes, vocab = int(a.vocab);
  const int token = int(token_in(a.tokens, i, a.vocab));
  float x;
  const Soft r = lanes_soft<T>(a, i, t, token >= 0, lanes, x);
  const float xt = __shfl(x, (int(threadIdx.x) % kWave) / lanes * lanes + max(token, 0));
  const float l = token < 0 ? 0.f : log_prob(a, xt, r);
  if (t == 0) a.logp[i] = l;
  if (kFor == kLogp) return;
  TokenLoss k = {0.f, 0.f};
  if (token >= 0) k = token_loss(a, i, l);
  if (t == 0) a.losses[i] = k.loss;
  if (t >= vocab) return;
  float d = 0.f;
  if (token >= 0 && l != -INFINITY) d = grad_of(r, k.slope * a.inv_t).at(x, a.c, t == token);
  static_cast<T*>(a.d_logits)[i * a.d_stride + t] = T(d);
}

// A wave (kThreads = 64, four rows a block) or a block takes a row that its
// registers hold.
template <class T, For kFor, int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads < kBlock ? kBlock : kThreads) void held_kernel(RowArgs a) {
  constexpr bool kWaves = kThreads == kWave;
  __shared__ float part[2][kWaves ? 1 : kThreads / kWave];
  const int64_t i = a.first + (kWaves ? int64_t(blockIdx.x) * (kBlock / kWave) + threadIdx.x / kWave
                                      : int64_t(blockIdx.x));
  if (i >= a.n) return;
  const int t = int(threadIdx.x) % kThreads, vocab = int(a.vocab);
  const int token = int(token_in(a.tokens, i, a.vocab));
  typedef Held<T, kThreads, kVecs> Row;
  T* const out = kFor != kLogp ? static_cast<T*>(a.d_logits) + i * a.d_stride : nullptr;
  if (kFor == kGrad && (token < 0 || a.logp_in[i] == -INFINITY)) return Row::zero(out, vocab, t);
  if (token < 0) {
    if (t == 0) {
      a.logp[i] = 0.f;
      if (kFor == kPolicy) a.losses[i] = 0.f;
    }
    if (kFor == kPolicy) Row::zero(out, vocab, t);
    return;
  }
  const T* const row = static_cast<const T*>(a.logits) + i * a.stride;
  const float xt = float(row[token]);
  Row r;
  r.load(row, vocab, t);
  float m = wave_max(r.most());
  r.fresh();
  if (!kWaves) {
    if (t % kWave == 0) part[0][t / kWave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) m = fmaxf(m, part[0][w]);
  }
  const float f = finite_max(m);
  float sum = wave_sum(r.sum(f, a.c));
  r.fresh();
  if (!kWaves) {
    if (t % kWave == 0) part[1][t / kWave] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) sum += part[1][w];
  }
  if (kFor == kGrad)
    return r.store(out, vocab, t, a.c, grad_of({m, sum}, a.d_logp[i] * a.inv_t), token);
  const float l = log_prob(a, xt, {m, sum});
  if (t == 0) a.logp[i] = l;
  if (kFor == kLogp) return;
  const TokenLoss k = token_loss(a, i, l);
  if (t == 0) a.losses[i] = k.loss;
  if (l == -INFINITY) return Row::zero(out, vocab, t);
  r.store(out, vocab, t, a.c, grad_of({m, sum}, k.slope * a.inv_t), token);
}

// Statistics of a long row, four pieces of a thread under way at once.
template <class T, int kThreads>
__device__ __forceinline__ Soft row_soft(const T* row, int64_t vocab, float c, Soft* part) {
  constexpr int N = Vec<T>::kN;
  Soft a = {-INFINITY, 0.f};
  const int64_t whole = vocab / N * N, step = int64_t(kThreads) * N;
  int64_t j = int64_t(threadIdx.x) * N;
  for (; j + 3 * step < whole; j += 4 * step) {
    typename Vec<T>::type v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = load16(row + j + k * step);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float x[N];
      widen<T>(x, v[k]);
      take(a, x, c);
    }
  }
  for (; j < whole; j += step) {
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

// d_logits of a row by kThreads threads.  Every element is read and written by the
// same thread, so that the two may be one.
// kPast: past the caches, which then hold more rows that are still to be read.
template <class T, int kThreads, bool kPast>
__device__ __forceinline__ void row_grad(const T* row, T* out, int64_t vocab, float c,
                                         const Grad& g, int64_t token) {
  constexpr int N = Vec<T>::kN;
  const int64_t whole = vocab / N * N;
  for (int64_t j = int64_t(threadIdx.x) * N; j < whole; j += kThreads * N) {
    float x[N];
    widen<T>(x, load16(row + j));
    typename Vec<T>::type v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = T(g.at(x[i], c, j + i == token));
    if (kPast) stream16(out + j, v);
    else store16(out + j, v);
  }
  const int64_t j = whole + threadIdx.x;
  if (j < vocab) out[j] = T(g.at(float(row[j]), c, j == token));
}

template <class T, int kThreads>
__device__ __forceinline__ void row_zero(T* out, int64_t vocab) {
  constexpr int N = Vec<T>::kN;
  const int64_t whole = vocab / N * N;
  for (int64_t j = int64_t(threadIdx.x) * N; j < whole; j += kThreads * N)
    store16(out + j, typename Vec<T>::type(T(0)));
  if (whole + threadIdx.x < vocab) out[whole + threadIdx.x] = T(0);
}

template <class T, For kFor, int kThreads>
__global__ __launch_bounds__(kThreads) void long_kernel(RowArgs a) {
  __shared__ Soft part[kThreads / kWave];
  const int64_t i = a.first + blockIdx.x;
  const int64_t token = token_in(a.tokens, i, a.vocab);
  T* const out = kFor == kPolicy ? static_cast<T*>(a.d_logits) + i * a.d_stride : nullptr;
  if (token < 0) {
    if (threadIdx.x == 0) {
      a.logp[i] = 0.f;
      if (kFor == kPolicy) a.losses[i] = 0.f;
    }
    if (kFor == kPolicy) row_zero<T, kThreads>(out, a.vocab);
    return;
  }
  const T* row = static_cast<const T*>(a.logits) + i * a.stride;
  const float xt = float(row[token]);
  const Soft r = row_soft<T, kThreads>(row, a.vocab, a.c, part);
  const float l = log_prob(a, xt, r);
  if (threadIdx.x == 0) a.logp[i] = l;
  if (kFor == kLogp) return;
  const TokenLoss k = token_loss(a, i, l);
  if (threadIdx.x == 0) a.losses[i] = k.loss;
  if (l == -INFINITY) return row_zero<T, kThreads>(out, a.vocab);
  row_grad<T, kThreads, true>(row, out, a.vocab, a.c, grad_of(r, k.slope * a.inv_t), token);
}

// The gradient alone, of rows of more than 64 logits: 1024 threads a row from
// 32,768 logits on (48 pairs, 50021 logits: 589 us, 626 with 256), else 256.
// Powers count from the token's logit and its log-probability l, two numbers of
// the size of l: where their roundings, some 3e-8 |l| of every probability, would
// show beside those of the result, the row's statistics are taken again.  That is
// from -32 on in 16 bits (a token that was all but ruled out).  In 32 bits rows
// that registers hold go by their statistics at all times (held_kernel; 8,000 rows
// of 32003 logits 375 us, 426 here), longer ones, which are read twice for them
// (3,000 rows of 131072: 835 us, 589 in one pass), from -4 on.
template <class T>
constexpr float kFar = sizeof(T) == 4 ? -4.f : -32.f;
template <class T, int kThreads>
__global__ __launch_bounds__(kThreads) void grad_kernel(RowArgs a) {
  const int64_t i = a.first + blockIdx.x;
  const int64_t token = token_in(a.tokens, i, a.vocab);
  T* out = static_cast<T*>(a.d_logits) + i * a.d_stride;
  const float l = a.logp_in[i];
  if (token < 0 || l == -INFINITY) return row_zero<T, kThreads>(out, a.vocab);
  const T* row = static_cast<const T*>(a.logits) + i * a.stride;
  const float gain = a.d_logp[i] * a.inv_t;
  Grad g = {float(row[token]), l * kLog2e, gain, gain};
  if (l < kFar<T>) {
    __shared__ Soft part[kThreads / kWave];
    const Soft r = row_soft<T, kThreads>(row, a.vocab, a.c, part);
    g = grad_of(r, gain);
  }
  __syncthreads();  // every thread has the token's logit before one writes there
  row_grad<T, kThreads, false>(row, out, a.vocab, a.c, g, token);
}

template <class T>
__global__ __launch_bounds__(kBlock) void lanes_grad_kernel(RowArgs a, int lanes) {
  const int64_t i = a.first + int64_t(blockIdx.x) * (kBlock / lanes) + int(threadIdx.x) / lanes;
  const int t = int(threadIdx.x) % lanes;
  if (i >= a.n) return;  // all of a row's lanes
  const int token = int(token_in(a.tokens, i, a.vocab));
  float x;
  const Soft r = lanes_soft<T>(a, i, t, token >= 0, lanes, x);
  if (t >= int(a.vocab)) return;
  float d = 0.f;
  if (token >= 0 && a.logp_in[i] != -INFINITY)
    d = grad_of(r, a.d_logp[i] * a.inv_t).at(x, a.c, t == token);
  static_cast<T*>(a.d_logits)[i * a.d_stride + t] = T(d);
}

// loss[0] = the sum of n values, added in a fixed order in 64 bits, eight pieces
// of a thread under way at once.
__global__ __launch_bounds__(1024) void total_kernel(const float* __restrict__ x, int64_t n,
                                                     float* loss) {
  constexpr int kAhead = 8;
  __shared__ double part[16];
  const int64_t whole = n / 4 * 4;
  double s = 0;
  for (int64_t i = int64_t(threadIdx.x) * 4; i < whole; i += 4096 * kAhead) {
    Vec<float>::type v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      v[k] = i + k * 4096 < whole ? load16(x + i + k * 4096) : Vec<float>::type(0.f);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) s += double(v[k][e]);
  }
  if (whole + threadIdx.x < n) s += double(x[whole + threadIdx.x]);
  s = block_sum(s, part);
  if (threadIdx.x == 0) loss[0] = float(s);
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
    // A side of no weight adds nothing, be its margin infinite.
    s += soft + (eps < 1 ? (1 - eps) * fmax(-m, 0.0) : 0.0) + (eps > 0 ? eps * fmax(m, 0.0) : 0.0);
  }
  s = block_sum(s, part);
  if (threadIdx.x == 0) loss[0] = float(s * double(scale) / n);
}

// Launches over all rows, `per` of them a block.
template <class K, class... A>
hipError_t over_rows(K kernel, RowArgs a, int per, int threads, hipStream_t s, A... more) {
  const int64_t blocks = (a.n + per - 1) / per;
  hipError_t e = hipSuccess;
  for (int64_t b = 0; b < blocks && e == hipSuccess; b += kMostBlocks) {
    a.first = b * per;
    hipLaunchKernelGGL(kernel, dim3(unsigned(std::min(blocks - b, kMostBlocks))), dim3(threads), 0,
                       s, a, more...);
    e = hipGetLastError();
  }
  return e;
}

int lanes_for(int64_t vocab) {
  int l = 1;
  while (l < vocab) l *= 2;
  return l;
}

// Rows of more than 64 logits that registers hold.
template <class T>
constexpr int64_t kMostHeld = 8192 * Vec<T>::kN + Vec<T>::kN - 1;
template <class T, For kFor>
hipError_t held_rows(const RowArgs& a, hipStream_t s) {
  const int64_t pieces = a.vocab / Vec<T>::kN;
  constexpr int kPer = kBlock / kWave;
  if (pieces <= 64) return over_rows(held_kernel<T, kFor, 64, 1>, a, kPer, kBlock, s);
  if (pieces <= 128) return over_rows(held_kernel<T, kFor, 64, 2>, a, kPer, kBlock, s);
  if (pieces <= 256) return over_rows(held_kernel<T, kFor, 64, 4>, a, kPer, kBlock, s);
  if (pieces <= 512) return over_rows(held_kernel<T, kFor, 64, 8>, a, kPer, kBlock, s);
  if (pieces <= 1024) return over_rows(held_kernel<T, kFor, 256, 4>, a, 1, 256, s);
  if (pieces <= 2048) return over_rows(held_kernel<T, kFor, 256, 8>, a, 1, 256, s);
  if (pieces <= 4096) return over_rows(held_kernel<T, kFor, 256, 16>, a, 1, 256, s);
  return over_rows(held_kernel<T, kFor, 512, 16>, a, 1, 512, s);
}

template <class T, For kFor>
hipError_t rows_of(const RowArgs& a, hipStream_t s) {
  if (a.vocab <= kWave) {
    const int lanes = lanes_for(a.vocab);
    return over_rows(lanes_kernel<T, kFor>, a, kBlock / lanes, kBlock, s, lanes);
  }
  if (a.vocab <= kMostHeld<T>) return held_rows<T, kFor>(a, s);
  return over_rows(long_kernel<T, kFor, kLongThreads>, a, 1, kLongThreads, s);
}

template <class T>
hipError_t grads_of(const RowArgs& a, hipStream_t s) {
  if (a.vocab <= kWave) {
    const int lanes = lanes_for(a.vocab);
    return over_rows(lanes_grad_kernel<T>, a, kBlock / lanes, kBlock, s, lanes);
  }
  if constexpr (sizeof(T) == 4) {
    if (a.vocab <= kMostHeld<T>) return held_rows<T, kGrad>(a, s);
  } else if (a.vocab < 32768) {
    return over_rows(grad_kernel<T, 256>, a, 1, 256, s);
  }
  return over_rows(grad_kernel<T, 1024>, a, 1, 1024, s);
}

template <For kFor>
hipError_t rows_by_type(int32_t dtype, const RowArgs& a, hipStream_t s) {
  return dtype == SCHED_F32   ? rows_of<float, kFor>(a, s)
         : dtype == SCHED_F16 ? rows_of<f16, kFor>(a, s)
                              : rows_of<bf16, kFor>(a, s);
}

Tokens tokens_of(const sched_tokens& t) { return {t.data, t.bits == 64}; }

RowArgs row_args(const sched_matrix& logits, const sched_tokens& tokens, float temperature) {
  RowArgs a = {};
  a.logits = logits.data;
  a.n = logits.rows;
  a.vocab = logits.cols;
  a.stride = logits.stride;
  a.tokens = tokens_of(tokens);
  a.t = temperature;
  a.c = float(1.4426950408889634 / double(temperature));
  a.inv_t = float(1.0 / double(temperature));
  return a;
}

}  // namespace

hipError_t launch_logprobs(const sched_matrix& logits, const sched_tokens& tokens,
                           float temperature, float* logp, hipStream_t s) {
  RowArgs a = row_args(logits, tokens, temperature);
  a.logp = logp;
  return rows_by_type<kLogp>(logits.dtype, a, s);
}

hipError_t launch_logprobs_grad(const sched_matrix& logits, const sched_tokens& tokens,
                                float temperature, const float* logp, const float* d_logp,
                                const sched_matrix& d_logits, hipStream_t s) {
  RowArgs a = row_args(logits, tokens, temperature);
  a.logp_in = logp;
  a.d_logp = d_logp;
  a.d_logits = d_logits.data;
  a.d_stride = d_logits.stride;
  return logits.dtype == SCHED_F32   ? grads_of<float>(a, s)
         : logits.dtype == SCHED_F16 ? grads_of<f16>(a, s)
                                     : grads_of<bf16>(a, s);
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
  const hipError_t e = rows_by_type<kPolicy>(d.logits.dtype, a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(total_kernel, dim3(1), dim3(1024), 0, s, d.losses, d.logits.rows, d.loss);
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
