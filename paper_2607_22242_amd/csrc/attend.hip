// attend.hip -- attention of packed sequences.
//
// For a query row with scores s_j = scale q . k_j over the keys it sees:
// out = sum_j exp(s_j - lse) v_j, lse = log sum_j exp s_j, in one pass over the
// keys: the running maximum and sum of powers rescale what has been added
// when the maximum moves.  4 D operations per pair of a query row and a key.
#include <hip/hip_runtime.h>

#include "attend.h"
#include "policy_launch.h"

namespace policy {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsOfBlock = 128;  // 32 of each wave
constexpr int kKeys = 64;          // of a tile

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) T k_tile[kKeys * D];
  __shared__ __attribute__((aligned(16))) T v_tile[kKeys * D];
  const Tile tile = tile_of(a.q_offsets, a.n_seqs, a.q_rows, a.group, kRowsOfBlock, int(blockIdx.x));
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kRowsOfBlock, rows = s.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
  const int kv = int(blockIdx.y), r = first + 32 * wave + lane % 32;
  const bool on = r < rows;
  const QueryRow me = query_row(a, kv, on ? r : 0);
  // Keys that a row sees: j <= last.
  const int ahead = s.keys - s.queries;
  const int last = !on ? -1 : a.causal ? min(s.keys - 1, me.query + ahead) : s.keys - 1;
  const int last_row = min(first + kRowsOfBlock, rows) - 1;
  const int end = a.causal ? min(s.keys, last_row / a.group + ahead + 1) : s.keys;

  typename Frag<T>::type q[D / 16];
  const T* q_row = head_row<T>(a.q, s.q0 + me.query, me.head);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) q[k] = piece(q_row, 16 * k + 8 * (lane / 32), a.dim, on);

  const float c = a.scale * kLog2e;
  const Rows<T, D> ks = {k_tile}, vs = {v_tile};
  Acc o[D / 32] = {};
  float most = -INFINITY, sum = 0.f;
  for (int j0 = 0; j0 < end; j0 += kKeys) {
    __syncthreads();
    for (int i = int(threadIdx.x); i < kKeys * (D / 8); i += kThreads) {
      const int row = i / (D / 8), d = i % (D / 8) * 8;
      const bool in = j0 + row < s.keys;
      const int64_t at = int64_t(s.k0) + (in ? j0 + row : 0);
      const auto kp = piece(head_row<T>(a.k, at, kv), d, a.dim, in);
      const auto vp = piece(head_row<T>(a.v, at, kv), d, a.dim, in);
      ks.put(row, d / 8, kp);
      vs.put(row, d / 8, vp);
    }
    __syncthreads();
    Acc x[kKeys / 32] = {};
    float m = most;
#pragma unroll
    for (int t = 0; t < kKeys / 32; ++t) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k) x[t] = product(ks.along(32 * t, k), q[k], x[t]);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (j0 + 32 * t + c_row(i) > last) x[t][i] = -INFINITY;
        m = fmaxf(m, x[t][i]);
      }
    }
    m = fmaxf(m, __shfl_xor(m, 32));
    const float f = m == -INFINITY ? 0.f : m, fc = f * c;
    const float keep = pow2((most - f) * c);
    most = m;
    sum *= keep;
#pragma unroll
    for (int t = 0; t < kKeys / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[t][i] = pow2(__builtin_fmaf(x[t][i], c, -fc));
        sum += x[t][i];
      }
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      o[d] *= keep;
#pragma unroll
      for (int t = 0; t < kKeys / 32; ++t)
#pragma unroll
        for (int p = 0; p < 2; ++p)
          o[d] = product(vs.across(32 * t + 16 * p, d), narrow<T>(x[t], p), o[d]);
    }
  }
  sum += __shfl_xor(sum, 32);
  if (!on) return;
  store_column<T, D>(head_row<T>(a.out, s.q0 + me.query, me.head), o, a.dim,
                     sum > 0.f ? 1.f / sum : 0.f);
  if (lane < 32)
    a.lse[int64_t(me.head) * a.q_rows + s.q0 + me.query] =
        sum > 0.f ? (most * c + log_2(sum)) * kLn2 : -INFINITY;
}

template <class T, int D>
hipError_t attend(const AttendArgs& a, int kv_heads, hipStream_t s) {
  const int64_t tiles = tile_count(int64_t(a.q_rows) * a.group, a.n_seqs, kRowsOfBlock);
  hipLaunchKernelGGL((attend_kernel<T, D>), dim3(unsigned(tiles), unsigned(kv_heads)),
                     dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

HeadsView view(const sched_heads& h) {
  return {static_cast<char*>(h.data), h.row_stride, h.head_stride};
}

}  // namespace

AttendArgs attend_args(const sched_attention_desc& d) {
  AttendArgs a = {};
  a.q = view(d.q);
  a.k = view(d.k);
  a.v = view(d.v);
  a.out = view(d.out);
  a.lse = d.lse;
  a.q_offsets = d.q_offsets;
  a.k_offsets = d.k_offsets;
  a.k_lengths = d.k_lengths;
  a.n_seqs = d.n_seqs;
  a.q_rows = int32_t(d.q_rows);
  a.k_rows = int32_t(d.k_rows);
  a.q_heads = d.q_heads;
  a.group = d.q_heads / d.kv_heads;
  a.dim = d.head_dim;
  a.causal = d.causal;
  a.scale = d.scale;
  return a;
}

size_t attention_bytes(const sched_attention_desc&) { return 0; }

hipError_t launch_attention(const sched_attention_desc& d, void*, hipStream_t s) {
  if (d.n_seqs == 0 || d.q_rows == 0) return hipSuccess;
  const AttendArgs a = attend_args(d);
  const bool wide = d.head_dim > 64;
  if (d.dtype == SCHED_F16)
    return wide ? attend<f16, 128>(a, d.kv_heads, s) : attend<f16, 64>(a, d.kv_heads, s);
  return wide ? attend<bf16, 128>(a, d.kv_heads, s) : attend<bf16, 64>(a, d.kv_heads, s);
}

}  // namespace policy
