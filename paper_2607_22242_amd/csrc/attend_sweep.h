// attend_sweep.h -- what the forward kernels of attention share: a wave's query
// rows against tiles of keys, and the join of sums over parts of the keys.
#pragma once
#include "attend.h"

namespace policy {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsOfBlock = 128;  // 32 of each wave
constexpr int kKeys = 64;          // of a tile
// How far scores may pass the reference of a row's powers (2^8) before the
// reference moves: the sums stay in 32 bits, and rescaling is rare.
constexpr float kSlack = 8.f;

// A wave's 32 query rows (lane l has row l % 32) and what has been added up
// over the keys so far, 32 kSubs of them at a time.
template <class T, int D, int kSubs, bool kFine = false>
struct Sweep {
  typename Frag<T>::type q[D / 16];
  Acc o[D / 32];
  float most, sum;  // reference of the powers; their sum over this lane's half of the keys

  // What is taken from the scores, to the base 2.
  __device__ __forceinline__ float reference(float c) const {
    return (most == -INFINITY ? 0.f : most) * c - kLift<T>;
  }

  __device__ __forceinline__ void start(const T* q_row, int dim, bool on) {
    const int h = int(threadIdx.x) % kWave / 32;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) q[k] = piece(q_row, 16 * k + 8 * h, dim, on);
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = Acc(0.f);
    most = -INFINITY;
    sum = 0.f;
  }

  // Adds the keys of a tile from its row `row` on, the first of them key j0; the
  // lane's row sees key j if sees(j) (`whole`: all rows of the wave see all).
  template <class Sees>
  __device__ __forceinline__ void add(const T* k_tile, const T* v_tile, int row, int j0,
                                      const Sees& sees, bool whole, float c,
                                      const Places<D>& places) {
    const Rows<T, D> ks = {k_tile, places.fresh()}, vs = {v_tile, ks.places};
    Acc x[kSubs];
    scores(ks, row, x);
    weigh(vs, row, x, j0, sees, whole, c);
  }

  // The two halves of it: products with the keys, and what follows from them.
  __device__ __forceinline__ void scores(const Rows<T, D>& ks, int row, Acc (&x)[kSubs]) const {
#pragma unroll
    for (int t = 0; t < kSubs; ++t) {
      x[t] = Acc(0.f);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) x[t] = product(ks.along(row + 32 * t, k), q[k], x[t]);
    }
  }
  template <class Sees>
  __device__ __forceinline__ void weigh(const Rows<T, D>& vs, int row, Acc (&x)[kSubs], int j0,
                                        const Sees& sees, bool whole, float c) {
    if (!whole) {
#pragma unroll
      for (int t = 0; t < kSubs; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!sees(j0 + 32 * t + c_row(i))) x[t][i] = -INFINITY;
    }
    float m = -INFINITY;
#pragma unroll
    for (int t = 0; t < kSubs; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, x[t][i]);
    m = fmaxf(m, __shfl_xor(m, 32));
    if (__any(m * c > most * c + kSlack)) {
      const float up = fmaxf(m, most), f = up == -INFINITY ? 0.f : up;
      const float keep = pow2((most - f) * c);
      most = up;
      sum *= keep;
#pragma unroll
      for (int d = 0; d < D / 32; ++d) o[d] *= keep;
    }
    const float fc = reference(c);
#pragma unroll
    for (int t = 0; t < kSubs; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[t][i] = pow2(__builtin_fmaf(x[t][i], c, -fc));
        sum += x[t][i];
      }
#pragma unroll
    for (int t = 0; t < kSubs; ++t)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const auto b = narrow<T>(x[t], p);
        typename Frag<T>::type rest;
        if (kFine) rest = rest_of<T>(x[t], p, b);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const auto v = vs.across(row + 32 * t + 16 * p, d);
          o[d] = product(v, b, o[d]);
          if (kFine) o[d] = product(v, rest, o[d]);
        }
      }
  }
};

// Keys up to one.
struct UpTo {
  int last;
  __device__ __forceinline__ bool operator()(int j) const { return j <= last; }
};

// Sums over parts of a row's keys, in 32 bits and each with a reference of its own.
struct Split {
  float* sums;     // a part: D of a row's sums and, behind all of them,
  float* weights;  // reference (to the base 2) and sum of powers
  int parts;       // of a row
};
__device__ __forceinline__ int64_t part_of(const AttendArgs& a, const Split& p, int64_t row,
                                           int head, int part) {
  return (row * a.q_heads + head) * p.parts + part;
}

// A wave joins the parts of row i / q_heads, head i % q_heads.
template <class T, int D>
__device__ __forceinline__ void join_row(const AttendArgs& a, const Split& p, int64_t i) {
  constexpr int kAhead = 8;  // parts under way at once
  const int lane = int(threadIdx.x) % kWave;
  const float* const weights = p.weights + i * p.parts * 2;
  float most = -INFINITY;
  for (int k = lane; k < p.parts; k += kWave)
    if (weights[2 * k + 1] != 0.f) most = fmaxf(most, weights[2 * k]);
  most = wave_max(most);
  float o[D / kWave] = {}, sum = 0.f;
  for (int k0 = 0; k0 < p.parts; k0 += kWave) {
    // A part's factor and sum, by the lane that has it.
    float f = 0.f, s = 0.f;
    if (k0 + lane < p.parts && weights[2 * (k0 + lane) + 1] != 0.f) {
      f = pow2(weights[2 * (k0 + lane)] - most);
      s = weights[2 * (k0 + lane) + 1] * f;
    }
    sum += wave_sum(s);
    for (int k = 0; k < min(kWave, p.parts - k0); k += kAhead) {
      float g[kAhead], x[kAhead][D / kWave];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int part = min(k0 + k + n, p.parts - 1);
        g[n] = k0 + k + n < p.parts ? __shfl(f, k + n) : 0.f;
#pragma unroll
        for (int d = 0; d < D / kWave; ++d)
          x[n][d] = p.sums[(i * p.parts + part) * D + d * kWave + lane];
      }
#pragma unroll
      for (int n = 0; n < kAhead; ++n)
#pragma unroll
        for (int d = 0; d < D / kWave; ++d)  // what a part of no weight holds is not used
          o[d] += g[n] == 0.f ? 0.f : g[n] * x[n][d];
    }
  }
  const int64_t row = i / a.q_heads;
  const int head = int(i % a.q_heads);
  T* const out = head_row<T>(a.out, row, head);
#pragma unroll
  for (int d = 0; d < D / kWave; ++d)
    if (d * kWave + lane < a.dim) out[d * kWave + lane] = T(sum == 0.f ? 0.f : o[d] / sum);
  if (lane == 0)
    a.lse[int64_t(head) * a.q_rows + row] =
        sum == 0.f ? -INFINITY : __builtin_fmaf(most, kLn2, ln(sum));
}

}  // namespace
}  // namespace policy
