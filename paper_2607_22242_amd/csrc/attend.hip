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
// How far scores may pass the reference of a row's powers (2^8) before the
// reference moves: the sums stay in 32 bits, and rescaling is rare.
constexpr float kSlack = 8.f;

// A wave's 32 query rows (lane l has row l % 32) and what has been added up
// over the keys so far.
template <class T, int D>
struct Sweep {
  typename Frag<T>::type q[D / 16];
  Acc o[D / 32];
  float most, sum;  // reference of the powers; their sum over this lane's half of the keys

  // Adds a tile of keys, of which the lane's row sees those up to `last`
  // (`whole`: all rows of the wave see all).
  __device__ __forceinline__ void add(const T* k_tile, const T* v_tile, int j0, int last,
                                      bool whole, float c, const Places<D>& places) {
    const Rows<T, D> ks = {k_tile, places.fresh()}, vs = {v_tile, ks.places};
    Acc x[kKeys / 32];
#pragma unroll
    for (int t = 0; t < kKeys / 32; ++t) {
      x[t] = Acc(0.f);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) x[t] = product(ks.along(32 * t, k), q[k], x[t]);
    }
    if (!whole) {
#pragma unroll
      for (int t = 0; t < kKeys / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (j0 + 32 * t + c_row(i) > last) x[t][i] = -INFINITY;
    }
    float m = -INFINITY;
#pragma unroll
    for (int t = 0; t < kKeys / 32; ++t)
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
    const float fc = (most == -INFINITY ? 0.f : most) * c;
#pragma unroll
    for (int t = 0; t < kKeys / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[t][i] = pow2(__builtin_fmaf(x[t][i], c, -fc));
        sum += x[t][i];
      }
#pragma unroll
    for (int t = 0; t < kKeys / 32; ++t)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const auto b = narrow<T>(x[t], p);
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
          o[d] = product(vs.across(32 * t + 16 * p, d), b, o[d]);
      }
  }
};

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendArgs a, int tiles) {
  __shared__ __attribute__((aligned(16))) T k_even[kKeys * D], v_even[kKeys * D];
  __shared__ __attribute__((aligned(16))) T k_odd[kKeys * D], v_odd[kKeys * D];
  const Work work = work_of(int(blockIdx.x), tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return;
  // The last tiles of a sequence see the most keys: they go first.
  const Tile tile = tile_of(a.q_offsets, a.n_seqs, a.q_rows, a.group, kRowsOfBlock,
                            tiles - 1 - work.tile);
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kRowsOfBlock, rows = s.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const int lane = int(threadIdx.x) % kWave, wave = wave_id();
  const int kv = work.kv, r = first + 32 * wave + lane % 32;
  const bool on = r < rows;
  const QueryRow me = query_row(a, kv, on ? r : 0);
  // Keys that a row sees: j <= last; those that all or any rows of the wave see.
  const int ahead = s.keys - s.queries;
  const int last = !on || !a.causal ? s.keys - 1 : min(s.keys - 1, me.query + ahead);
  const int last_row = min(first + kRowsOfBlock, rows) - 1;
  const int end = a.causal ? min(s.keys, last_row / a.group + ahead + 1) : s.keys;
  const int wave_first = min(first + 32 * wave, rows - 1);
  const int wave_last = min(wave_first + 31, rows - 1);
  const int all = !a.causal ? s.keys - 1 : min(s.keys - 1, wave_first / a.group + ahead);
  const int any = !a.causal ? s.keys - 1 : min(s.keys - 1, wave_last / a.group + ahead);

  Sweep<T, D> w;
  const T* q_row = head_row<T>(a.q, s.q0 + me.query, me.head);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) w.q[k] = piece(q_row, 16 * k + 8 * (lane / 32), a.dim, on);
#pragma unroll
  for (int d = 0; d < D / 32; ++d) w.o[d] = Acc(0.f);
  w.most = -INFINITY;
  w.sum = 0.f;
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const KeyTiles<T, D, kKeys, kThreads> tiles_of(a, s, kv);
  if (end > 0) tiles_of.fetch(0, k_even, v_even, a.dim);
  for (int j0 = 0; j0 < end; j0 += 2 * kKeys) {
    __syncthreads();  // the tile is there, and nobody reads the other buffer any more
    if (j0 + kKeys < end) tiles_of.fetch(j0 + kKeys, k_odd, v_odd, a.dim);
    if (j0 <= any) w.add(k_even, v_even, j0, last, j0 + kKeys - 1 <= all, c, places);
    if (j0 + kKeys >= end) break;
    __syncthreads();
    if (j0 + 2 * kKeys < end) tiles_of.fetch(j0 + 2 * kKeys, k_even, v_even, a.dim);
    if (j0 + kKeys <= any) w.add(k_odd, v_odd, j0 + kKeys, last, j0 + 2 * kKeys - 1 <= all, c, places);
  }
  const float sum = w.sum + __shfl_xor(w.sum, 32);
  if (!on) return;
  store_column<T, D>(head_row<T>(a.out, s.q0 + me.query, me.head), w.o, a.dim,
                     sum > 0.f ? 1.f / sum : 0.f);
  if (lane < 32)
    a.lse[int64_t(me.head) * a.q_rows + s.q0 + me.query] =
        sum > 0.f ? (w.most * c + log_2(sum)) * kLn2 : -INFINITY;
}

template <class T, int D>
hipError_t attend(const AttendArgs& a, int kv_heads, hipStream_t s) {
  const int64_t tiles = tile_count(int64_t(a.q_rows) * a.group, a.n_seqs, kRowsOfBlock);
  hipLaunchKernelGGL((attend_kernel<T, D>), dim3(unsigned(work_blocks(tiles, kv_heads))),
                     dim3(kThreads), 0, s, a, int(tiles));
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
  a.per_group = uint32_t(((uint64_t(1) << 32) + a.group - 1) / a.group);
  a.dim = d.head_dim;
  auto near = [](const sched_heads& h) {
    return h.row_stride < (int64_t(1) << 24) && h.head_stride < (int64_t(1) << 24);
  };
  a.near_k = near(d.k) && near(d.v);
  a.near_q = near(d.q) && 16 % a.group == 0;
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
