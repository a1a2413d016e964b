// attend_grad.hip -- the backward pass of attention, which computes the
// probabilities again from the products and lse.
//
// With P = exp(scale Q K^T - lse) and delta = rowsum(dO o O):
// dV = P^T dO, dP = dO V^T, dS = P o (dP - delta), dQ = scale dS K,
// dK = scale dS^T Q.  One kernel holds keys and walks over the query rows (dK,
// dV), one holds query rows and walks over the keys (dQ), so that every sum has
// one order and no atomics: 14 D operations per pair in place of 10 D.
#include <hip/hip_runtime.h>

#include "attend.h"
#include "policy_launch.h"

namespace policy {

AttendArgs attend_args(const sched_attention_desc& d);

namespace {

constexpr int kThreads = 256;
constexpr int kTileOfBlock = 128;  // keys or query rows that a block holds, 32 of each wave
constexpr int kQueries = 32;       // rows of a tile that the kernel of dK and dV walks over
constexpr int kKeys = 32;          // keys of a tile that the kernel of dQ walks over

// delta of every query row and head; 16 lanes a row.
template <class T>
__global__ __launch_bounds__(kThreads) void delta_kernel(AttendArgs a, int64_t first) {
  const int64_t i = first + int64_t(blockIdx.x) * (kThreads / 16) + int(threadIdx.x) / 16;
  if (i >= int64_t(a.q_rows) * a.q_heads) return;
  const int64_t row = i / a.q_heads;
  const int head = int(i % a.q_heads), d = int(threadIdx.x) % 16 * 8;
  const auto x = piece(head_row<T>(a.out, row, head), d, a.dim, true);
  const auto y = piece(head_row<T>(a.d_out, row, head), d, a.dim, true);
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += float(x[e]) * float(y[e]);
#pragma unroll
  for (int k = 8; k; k >>= 1) sum += __shfl_xor(sum, k);
  if (threadIdx.x % 16 == 0) a.delta[int64_t(head) * a.q_rows + row] = sum;
}

// Keys 32 wave + lane % 32 of the block's tile; lanes' columns are keys, their
// values run along the query rows.
template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void keys_kernel(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) T q_tile[kQueries * D];
  __shared__ __attribute__((aligned(16))) T o_tile[kQueries * D];
  __shared__ float lse2[kQueries], delta[kQueries];
  const Tile tile = tile_of(a.k_offsets, a.n_seqs, a.k_rows, 1, kTileOfBlock, int(blockIdx.x));
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kTileOfBlock;
  if (tile.index < 0 || first >= s.slot) return;
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
  const int kv = int(blockIdx.y), j = first + 32 * wave + lane % 32;
  const bool on = j < s.keys;
  const int64_t key = int64_t(s.k0) + (on ? j : 0);
  typename Frag<T>::type k[D / 16], v[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    k[i] = piece(head_row<T>(a.k, key, kv), 16 * i + 8 * (lane / 32), a.dim, on);
    v[i] = piece(head_row<T>(a.v, key, kv), 16 * i + 8 * (lane / 32), a.dim, on);
  }
  const float c = a.scale * kLog2e;
  const Rows<T, D> qs = {q_tile}, os = {o_tile};
  Acc dk[D / 32] = {}, dv[D / 32] = {};
  const int rows = first < s.keys ? s.queries * a.group : 0, ahead = s.keys - s.queries;
  // The first query that sees the block's first key.
  const int begin =
      a.causal && rows > 0 ? max(0, first - ahead) * a.group / kQueries * kQueries : 0;
  for (int r0 = begin; r0 < rows; r0 += kQueries) {
    __syncthreads();
    for (int i = int(threadIdx.x); i < kQueries * (D / 8); i += kThreads) {
      const int row = i / (D / 8), d = i % (D / 8) * 8;
      const bool in = r0 + row < rows;
      const QueryRow at = query_row(a, kv, in ? r0 + row : 0);
      const auto qp = piece(head_row<T>(a.q, s.q0 + at.query, at.head), d, a.dim, in);
      const auto op = piece(head_row<T>(a.d_out, s.q0 + at.query, at.head), d, a.dim, in);
      qs.put(row, d / 8, qp);
      os.put(row, d / 8, op);
      if (d == 0) {
        const int64_t n = int64_t(at.head) * a.q_rows + s.q0 + at.query;
        lse2[row] = in ? a.lse[n] * kLog2e : INFINITY;  // powers of rows that are not there are 0
        delta[row] = in ? a.delta[n] : 0.f;
      }
    }
    __syncthreads();
    Acc x = {}, y = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      x = product(qs.along(0, i), k[i], x);
      y = product(os.along(0, i), v[i], y);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = c_row(i);
      const bool seen = on && (!a.causal || j <= (r0 + r) / a.group + ahead);
      x[i] = seen ? pow2(__builtin_fmaf(x[i], c, -lse2[r])) : 0.f;
      y[i] = x[i] * (y[i] - delta[r]);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const auto pb = narrow<T>(x, p), db = narrow<T>(y, p);
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        dv[d] = product(os.across(16 * p, d), pb, dv[d]);
        dk[d] = product(qs.across(16 * p, d), db, dk[d]);
      }
    }
  }
  if (j >= s.slot) return;
  store_column<T, D>(head_row<T>(a.d_k, int64_t(s.k0) + j, kv), dk, a.dim, on ? a.scale : 0.f);
  store_column<T, D>(head_row<T>(a.d_v, int64_t(s.k0) + j, kv), dv, a.dim, on ? 1.f : 0.f);
}

// Query rows 32 wave + lane % 32 of the block's tile; lanes' columns are query
// rows, their values run along the keys.
template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void queries_kernel(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) T k_tile[kKeys * D];
  __shared__ __attribute__((aligned(16))) T v_tile[kKeys * D];
  const Tile tile = tile_of(a.q_offsets, a.n_seqs, a.q_rows, a.group, kTileOfBlock, int(blockIdx.x));
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kTileOfBlock, rows = s.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
  const int kv = int(blockIdx.y), r = first + 32 * wave + lane % 32;
  const bool on = r < rows;
  const QueryRow me = query_row(a, kv, on ? r : 0);
  const int ahead = s.keys - s.queries;
  const int last = !on ? -1 : a.causal ? min(s.keys - 1, me.query + ahead) : s.keys - 1;
  const int last_row = min(first + kTileOfBlock, rows) - 1;
  const int end = a.causal ? min(s.keys, last_row / a.group + ahead + 1) : s.keys;
  typename Frag<T>::type q[D / 16], o[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const int d = 16 * i + 8 * (lane / 32);
    q[i] = piece(head_row<T>(a.q, s.q0 + me.query, me.head), d, a.dim, on);
    o[i] = piece(head_row<T>(a.d_out, s.q0 + me.query, me.head), d, a.dim, on);
  }
  const int64_t n = int64_t(me.head) * a.q_rows + s.q0 + me.query;
  const float c = a.scale * kLog2e, lse2 = on ? a.lse[n] * kLog2e : INFINITY;
  const float delta = on ? a.delta[n] : 0.f;
  const Rows<T, D> ks = {k_tile}, vs = {v_tile};
  Acc dq[D / 32] = {};
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
    Acc x = {}, y = {};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      x = product(ks.along(0, i), q[i], x);
      y = product(vs.along(0, i), o[i], y);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = j0 + c_row(i) <= last ? pow2(__builtin_fmaf(x[i], c, -lse2)) : 0.f;
      y[i] = p * (y[i] - delta);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const auto db = narrow<T>(y, p);
#pragma unroll
      for (int d = 0; d < D / 32; ++d) dq[d] = product(ks.across(16 * p, d), db, dq[d]);
    }
  }
  if (on) store_column<T, D>(head_row<T>(a.d_q, s.q0 + me.query, me.head), dq, a.dim, a.scale);
}

template <class T, int D>
hipError_t attend_grad(const AttendArgs& a, int kv_heads, hipStream_t s) {
  const int64_t rows = int64_t(a.q_rows) * a.q_heads, blocks = (rows + 15) / 16;
  hipError_t e = hipSuccess;
  for (int64_t b = 0; b < blocks && e == hipSuccess; b += kMostBlocks) {
    hipLaunchKernelGGL(delta_kernel<T>, dim3(unsigned(blocks - b < kMostBlocks ? blocks - b : kMostBlocks)),
                       dim3(kThreads), 0, s, a, b * 16);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  if (a.k_rows > 0) {
    const int64_t tiles = tile_count(a.k_rows, a.n_seqs, kTileOfBlock);
    hipLaunchKernelGGL((keys_kernel<T, D>), dim3(unsigned(tiles), unsigned(kv_heads)),
                       dim3(kThreads), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.q_rows > 0) {
    const int64_t tiles = tile_count(int64_t(a.q_rows) * a.group, a.n_seqs, kTileOfBlock);
    hipLaunchKernelGGL((queries_kernel<T, D>), dim3(unsigned(tiles), unsigned(kv_heads)),
                       dim3(kThreads), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

HeadsView view(const sched_heads& h) {
  return {static_cast<char*>(h.data), h.row_stride, h.head_stride};
}

}  // namespace

size_t attention_grad_bytes(const sched_attention_desc& d) {
  return size_t(d.q_rows) * size_t(d.q_heads) * 4;
}

hipError_t launch_attention_grad(const sched_attention_desc& d, const sched_heads& d_out,
                                 const sched_heads& d_q, const sched_heads& d_k,
                                 const sched_heads& d_v, void* ws, hipStream_t s) {
  if (d.n_seqs == 0) return hipSuccess;
  AttendArgs a = attend_args(d);
  a.d_out = view(d_out);
  a.d_q = view(d_q);
  a.d_k = view(d_k);
  a.d_v = view(d_v);
  a.delta = static_cast<float*>(ws);
  const bool wide = d.head_dim > 64;
  if (d.dtype == SCHED_F16)
    return wide ? attend_grad<f16, 128>(a, d.kv_heads, s) : attend_grad<f16, 64>(a, d.kv_heads, s);
  return wide ? attend_grad<bf16, 128>(a, d.kv_heads, s) : attend_grad<bf16, 64>(a, d.kv_heads, s);
}

}  // namespace policy
