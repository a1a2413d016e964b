// attend_grad.hip -- the backward pass of attention, which computes the
// probabilities again from the products and lse.
//
// With P = exp(scale Q K^T - lse) and delta = rowsum(dO o O):
// dV = P^T dO, dP = dO V^T, dS = P o (dP - delta), dQ = scale dS K,
// dK = scale dS^T Q.  One kernel holds keys and walks over the query rows (dK,
// dV), one holds query rows and walks over the keys (dQ), so that every sum has
// one order and no atomics: 14 D operations per pair in place of 10 D.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_grad_sweep.h"
#include "policy_launch.h"

namespace policy {

AttendArgs attend_args(const sched_attention_desc& d);

namespace {

// --- dK and dV ----------------------------------------------------------------

// A block holds 64 keys; waves 0 and 1 take the even 32 rows of each tile with
// keys 0 .. 31 and 32 .. 63, waves 2 and 3 the odd 32; their sums meet at the end.
template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void keys_kernel(AttendArgs a, KeyParts p, int tiles) {
  __shared__ __attribute__((aligned(16))) T q_even[kTile * D], o_even[kTile * D];
  __shared__ __attribute__((aligned(16))) T q_odd[kTile * D], o_odd[kTile * D];
  constexpr int kRest = KeySweep<T, D>::kHeld < D / 16 ? kKeysOfBlock * 64 : 8;
  __shared__ __attribute__((aligned(16))) T v_rest[kRest];
  __shared__ __attribute__((aligned(16))) Stats s_even, s_odd;
  const Work work = work_of(int(blockIdx.x), tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return;
  const Tile tile = key_tile(a, kKeysOfBlock, work.tile);
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kKeysOfBlock;
  if (tile.index < 0 || first >= s.slot) return;
  const int lane = int(threadIdx.x) % kWave, wave = wave_id();
  const int kv = work.kv, part = wave / 2 * 32, wave_row = wave % 2 * 32;
  const int wave_key = first + wave_row;
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const Rows<T, 64> rest = {v_rest, Places<64>()};
  const int rows = first < s.keys ? s.queries * a.group : 0, ahead = s.keys - s.queries;
  // The first row that sees a key.
  auto seen_from = [&](int key) { return a.causal ? max(0, key - ahead) * a.group : 0; };
  const int j = wave_key + lane % 32;
  const bool on = j < s.keys;
  const int from = on ? seen_from(j) : rows;
  KeySweep<T, D> w;
  {
    const int64_t key = int64_t(s.k0) + (on ? j : 0);
    const T *k_row = head_row<T>(a.k, key, kv), *v_row = head_row<T>(a.v, key, kv);
    const int h = lane / 32, row = wave_row + lane % 32;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      w.k[i] = piece(k_row, 16 * i + 8 * h, a.dim, on);
      const auto v = piece(v_row, 16 * i + 8 * h, a.dim, on);
      if (i < KeySweep<T, D>::kHeld)
        w.v[i] = v;
      else if (part == 0)
        *reinterpret_cast<typename Frag<T>::type*>(
            v_rest + row * 64 + ((2 * (i - KeySweep<T, D>::kHeld) + h) ^ turn_of<64>(row)) * 8) = v;
    }
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) w.dk[i] = w.dv[i] = Acc(0.f);
  w.up = kLargest;
  int begin = rows > 0 ? seen_from(first) / kTile * kTile : 0;
  const int all = wave_key + 31 < s.keys ? seen_from(wave_key + 31) : rows;
  const int any = wave_key < s.keys ? seen_from(wave_key) : rows;
  const RowTiles<T, D> tiles_of(a);
  // From the last rows, which see every key, to the first: blocks that run side
  // by side read the same rows at the same time.
  int end = rows > 0 ? (rows - 1) / kTile * kTile : -1;
  if (p.parts > 1) {  // this block's share of the row tiles
    const int share = (max(end - begin + kTile, 0) / kTile + p.parts - 1) / p.parts;
    end -= int(blockIdx.y) * share * kTile;
    begin = max(begin, end - (share - 1) * kTile);
  }
  RowTile t = row_tile(a, max(end, 0));
  auto step = [&](int r0, const T* q_tile, const T* o_tile, const Stats& stats) {
    const int r = r0 + part;
    if (r + 31 < any || r >= rows) return;
    w.add(q_tile, o_tile, stats, rest, wave_row, part,
          [&] { return RowSpan{from - r0, rows - 1 - r0}; }, r >= all && r + 31 < rows, c, places);
  };
  if (end >= begin) tiles_of.fetch(a, s, kv, rows, t, q_even, o_even, &s_even);
  for (int r0 = end; r0 >= begin; r0 -= 2 * kTile) {
    tiles_barrier();  // the tile is there, and nobody reads the other buffer any more
    retreat(a, t);
    if (t.r0 >= begin) tiles_of.fetch(a, s, kv, rows, t, q_odd, o_odd, &s_odd);
    step(r0, q_even, o_even, s_even);
    if (r0 - kTile < begin) break;
    tiles_barrier();
    retreat(a, t);
    if (t.r0 >= begin) tiles_of.fetch(a, s, kv, rows, t, q_even, o_even, &s_even);
    step(r0 - kTile, q_odd, o_odd, s_odd);
  }
  // Waves 2 and 3 hand their sums to waves 0 and 1.
  static_assert(sizeof(q_even) == size_t(D) / 32 * 16 * kWave * sizeof(float), "a wave's sums");
  float* const buf_k = reinterpret_cast<float*>(wave % 2 ? q_odd : q_even);
  float* const buf_v = reinterpret_cast<float*>(wave % 2 ? o_odd : o_even);
  tiles_barrier();
  if (kShort<T>) {
    shift(w.dk, -w.up - int(kLiftGrad<T>));
    shift(w.dv, -int(kLiftGrad<T>));
  }
  if (wave >= 2) w.hand(buf_k, buf_v);
  tiles_barrier();
  if (wave >= 2 || j >= s.slot) return;
  w.take(buf_k, buf_v);
  if (!on) {  // also where a row that was NaN has met the tile's zeros
#pragma unroll
    for (int i = 0; i < D / 32; ++i) w.dk[i] = w.dv[i] = Acc(0.f);
  }
  if (p.parts > 1) {
    const int64_t at = key_part<D>(a, int(blockIdx.y), kv, int64_t(s.k0) + j);
    store_column<float, D>(p.dk + at, w.dk, D, a.scale);
    store_column<float, D>(p.dv + at, w.dv, D, 1.f);
    return;
  }
  store_column<T, D>(head_row<T>(a.d_k, int64_t(s.k0) + j, kv), w.dk, a.dim, a.scale);
  store_column<T, D>(head_row<T>(a.d_v, int64_t(s.k0) + j, kv), w.dv, a.dim, 1.f);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void add_parts_kernel(AttendArgs a, KeyParts p, int tiles) {
  typedef float Four __attribute__((ext_vector_type(4)));
  typedef T four __attribute__((ext_vector_type(4)));
  const Work work = work_of(int(blockIdx.x), tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return;
  const Tile tile = key_tile(a, kKeysOfBlock, work.tile);
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kKeysOfBlock;
  if (tile.index < 0 || first >= s.slot) return;
  const int d = int(threadIdx.x) % (D / 4) * 4;
  for (int j = first + int(threadIdx.x) / (D / 4); j < min(first + kKeysOfBlock, s.slot);
       j += kThreads / (D / 4)) {
    const int64_t row = int64_t(s.k0) + j;
    Four x = Four(0.f), y = Four(0.f);
    for (int i = 0; i < p.parts; ++i) {
      const int64_t at = key_part<D>(a, i, work.kv, row) + d;
      x += *reinterpret_cast<const Four*>(p.dk + at);
      y += *reinterpret_cast<const Four*>(p.dv + at);
    }
    if (d >= a.dim) continue;
    four u, v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      u[e] = T(x[e]);
      v[e] = T(y[e]);
    }
    *reinterpret_cast<four*>(head_row<T>(a.d_k, row, work.kv) + d) = u;
    *reinterpret_cast<four*>(head_row<T>(a.d_v, row, work.kv) + d) = v;
  }
}

// As many parts as fill the 512 places that the card has for the kernel's blocks,
// none with less than 8 tiles of a mean sequence's rows.  The whole pass over
// 2,000 tokens, 4, 8 and 16 heads of one key head: 141, 157 and 200 us so, 268,
// 461 and 939 in one part; 1,024 tokens, 32/4 heads: 110 and 249.
int key_parts_of(const sched_attention_desc& d) {
  if (d.n_seqs == 0 || d.k_rows == 0) return 1;
  const int64_t blocks = tile_count(d.k_rows, d.n_seqs, kKeysOfBlock) * d.kv_heads;
  const int64_t rows = d.q_rows * (d.q_heads / d.kv_heads) / d.n_seqs;
  return int(std::max<int64_t>(1, std::min(512 / blocks, rows / (8 * kTile))));
}
size_t stats_bytes(const sched_attention_desc& d) {
  return (size_t(d.q_rows) * size_t(d.q_heads) * 8 + 255) & ~size_t(255);
}
size_t key_part_count(const sched_attention_desc& d) {  // values of dK, or of dV
  const int parts = key_parts_of(d);
  if (parts == 1) return 0;
  return size_t(parts) * size_t(d.k_rows) * size_t(d.kv_heads) * (d.head_dim > 64 ? 128 : 64);
}

// --- dQ -----------------------------------------------------------------------

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void queries_kernel(AttendArgs a, RowParts p, int tiles) {
  __shared__ __attribute__((aligned(16))) T k_even[kTile * D], v_even[kTile * D];
  __shared__ __attribute__((aligned(16))) T k_odd[kTile * D], v_odd[kTile * D];
  const Work work = work_of(int(blockIdx.x), tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return;
  const Tile tile = query_tile(a, kRowsOfBlock, work.tile, tiles);
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kRowsOfBlock, rows = s.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const int lane = int(threadIdx.x) % kWave, wave = wave_id();
  const int kv = work.kv, r = first + 32 * wave + lane % 32;
  const bool on = r < rows;
  const QueryRow me = query_row(a, kv, on ? r : 0);
  const int ahead = s.keys - s.queries;
  const int last = !on || !a.causal ? s.keys - 1 : min(s.keys - 1, me.query + ahead);
  const int last_row = min(first + kRowsOfBlock, rows) - 1;
  int begin = 0, end = a.causal ? min(s.keys, last_row / a.group + ahead + 1) : s.keys;
  if (p.parts > 1) {  // this block's share of the tiles
    const int share = ((max(end, 0) + kTile - 1) / kTile + p.parts - 1) / p.parts * kTile;
    begin = min(int(blockIdx.y) * share, max(end, 0));
    end = min(begin + share, end);
  }
  const int wave_first = min(first + 32 * wave, rows - 1);
  const int wave_last = min(wave_first + 31, rows - 1);
  const int all = !a.causal ? s.keys - 1 : min(s.keys - 1, wave_first / a.group + ahead);
  const int any = !a.causal ? s.keys - 1 : min(s.keys - 1, wave_last / a.group + ahead);

  RowSweep<T, D> w;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const int d = 16 * i + 8 * (lane / 32);
    w.q[i] = piece(head_row<T>(a.q, s.q0 + me.query, me.head), d, a.dim, on);
    w.o[i] = piece(head_row<T>(a.d_out, s.q0 + me.query, me.head), d, a.dim, on);
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) w.dq[i] = Acc(0.f);
  // The row's statistics, which the kernel of dK and dV reads too.
  const int64_t n = int64_t(me.head) * a.q_rows + s.q0 + me.query;
  const T* const out_row = head_row<T>(a.out, s.q0 + me.query, me.head);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const auto x = piece(out_row, 16 * i + 8 * (lane / 32), a.dim, on);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += float(x[e]) * float(w.o[i][e]);
  }
  w.delta = -(sum + __shfl_xor(sum, 32));
  const float lse = on ? a.lse[n] : -INFINITY;
  w.lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;  // powers of rows that see nothing are 0
  const bool first_part = lane < 32 && on && blockIdx.y == 0;  // the part of the first tile
  if (first_part) a.lse2[n] = w.lse2 - kLiftGrad<T>;
  w.up = kShort<T> ? kLargest : 0;
  w.lse2 -= float(w.up);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const KeyTiles<T, D, kTile, kThreads> tiles_of(a, s, kv);
  if (begin < end) tiles_of.fetch(begin, k_even, v_even, a.dim);
  for (int j0 = begin; j0 < end; j0 += 2 * kTile) {
    tiles_barrier();
    if (j0 + kTile < end) tiles_of.fetch(j0 + kTile, k_odd, v_odd, a.dim);
    if (any < kTile && j0 <= any) w.exact_delta(k_even, v_even, last, c, places);
    if (j0 <= any) w.add(k_even, v_even, j0, UpTo{last}, j0 + kTile - 1 <= all, c, places);
    if (j0 + kTile >= end) break;
    tiles_barrier();
    if (j0 + 2 * kTile < end) tiles_of.fetch(j0 + 2 * kTile, k_even, v_even, a.dim);
    if (j0 + kTile <= any)
      w.add(k_odd, v_odd, j0 + kTile, UpTo{last}, j0 + 2 * kTile - 1 <= all, c, places);
  }
  if (!on) return;
  if (kShort<T>) shift(w.dq, -w.up);
  if (last < 0) {  // a row that sees nothing, whatever it holds
#pragma unroll
    for (int i = 0; i < D / 32; ++i) w.dq[i] = Acc(0.f);
  }
  if (p.parts > 1)
    store_column<float, D>(p.dq + row_part<D>(a, int(blockIdx.y), s.q0 + me.query, me.head), w.dq, D,
                           a.scale);
  else
    store_column<T, D>(head_row<T>(a.d_q, s.q0 + me.query, me.head), w.dq, a.dim, a.scale);
  if (first_part) a.delta[n] = w.delta;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void add_row_parts_kernel(AttendArgs a, RowParts p,
                                                                 int tiles) {
  typedef float Four __attribute__((ext_vector_type(4)));
  typedef T four __attribute__((ext_vector_type(4)));
  const Work work = work_of(int(blockIdx.x), tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return;
  const Tile tile = query_tile(a, kRowsOfBlock, work.tile, tiles);
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * kRowsOfBlock, rows = s.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const int d = int(threadIdx.x) % (D / 4) * 4;
  if (d >= a.dim) return;
  for (int r = first + int(threadIdx.x) / (D / 4); r < min(first + kRowsOfBlock, rows);
       r += kThreads / (D / 4)) {
    const QueryRow me = query_row(a, work.kv, r);
    const int64_t row = int64_t(s.q0) + me.query;
    Four x = Four(0.f);
    for (int i = 0; i < p.parts; ++i)
      x += *reinterpret_cast<const Four*>(p.dq + row_part<D>(a, i, row, me.head) + d);
    four u;
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = T(x[e]);
    *reinterpret_cast<four*>(head_row<T>(a.d_q, row, me.head) + d) = u;
  }
}

// As above, none with less than 12 tiles of a mean sequence's keys.  The whole
// pass over 8,192 tokens of one head: 184 us so, 344 in one part; 4,000 tokens, 8
// heads of 2 key heads: 246 and 274; with parts of 8 tiles 1,100 tokens, 2 heads of
// one, would lose 44 to 46.
int row_parts_of(const sched_attention_desc& d) {
  if (d.n_seqs == 0 || d.q_rows == 0) return 1;
  const int64_t blocks =
      tile_count(d.q_rows * (d.q_heads / d.kv_heads), d.n_seqs, kRowsOfBlock) * d.kv_heads;
  return int(std::max<int64_t>(1, std::min(512 / blocks, d.k_rows / d.n_seqs / (12 * kTile))));
}
size_t row_part_count(const sched_attention_desc& d) {
  const int parts = row_parts_of(d);
  if (parts == 1) return 0;
  return size_t(parts) * size_t(d.q_rows) * size_t(d.q_heads) * (d.head_dim > 64 ? 128 : 64);
}

template <class T, int D>
hipError_t attend_grad(const AttendArgs& a, const KeyParts& p, const RowParts& r, int kv_heads,
                       hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.q_rows > 0) {  // first: it leaves the rows' statistics
    const int64_t tiles = tile_count(int64_t(a.q_rows) * a.group, a.n_seqs, kRowsOfBlock);
    const dim3 grid(unsigned(work_blocks(tiles, kv_heads)), unsigned(r.parts));
    hipLaunchKernelGGL((queries_kernel<T, D>), grid, dim3(kThreads), 0, s, a, r, int(tiles));
    e = hipGetLastError();
    if (r.parts > 1 && e == hipSuccess) {
      hipLaunchKernelGGL((add_row_parts_kernel<T, D>), dim3(grid.x), dim3(kThreads), 0, s, a, r,
                         int(tiles));
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
  }
  if (a.k_rows > 0) {
    const int64_t tiles = tile_count(a.k_rows, a.n_seqs, kKeysOfBlock);
    const dim3 grid(unsigned(work_blocks(tiles, kv_heads)), unsigned(p.parts));
    hipLaunchKernelGGL((keys_kernel<T, D>), grid, dim3(kThreads), 0, s, a, p, int(tiles));
    e = hipGetLastError();
    if (p.parts > 1 && e == hipSuccess) {
      hipLaunchKernelGGL((add_parts_kernel<T, D>), dim3(grid.x), dim3(kThreads), 0, s, a, p,
                         int(tiles));
      e = hipGetLastError();
    }
  }
  return e;
}

HeadsView view(const sched_heads& h) {
  return {static_cast<char*>(h.data), h.row_stride, h.head_stride};
}

}  // namespace

size_t attention_grad_bytes(const sched_attention_desc& d) {
  // The parts of dQ have been added when those of dK and dV are written.
  return stats_bytes(d) + std::max(row_part_count(d), 2 * key_part_count(d)) * sizeof(float);
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
  a.lse2 = static_cast<float*>(ws);
  a.near_q = a.near_q && d_out.row_stride < (int64_t(1) << 24) &&
             d_out.head_stride < (int64_t(1) << 24);
  a.delta = a.lse2 + size_t(d.q_rows) * size_t(d.q_heads);
  const bool wide = d.head_dim > 64;
  float* const parts = reinterpret_cast<float*>(static_cast<char*>(ws) + stats_bytes(d));
  const KeyParts p = {parts, parts + key_part_count(d), key_parts_of(d)};
  const RowParts r = {parts, row_parts_of(d)};
  if (d.dtype == SCHED_F16)
    return wide ? attend_grad<f16, 128>(a, p, r, d.kv_heads, s)
                : attend_grad<f16, 64>(a, p, r, d.kv_heads, s);
  return wide ? attend_grad<bf16, 128>(a, p, r, d.kv_heads, s)
              : attend_grad<bf16, 64>(a, p, r, d.kv_heads, s);
}

}  // namespace policy
