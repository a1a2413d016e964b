// attend.hip -- attention of packed sequences.
//
// For a query row with scores s_j = scale q . k_j over the keys it sees:
// out = sum_j exp(s_j - lse) v_j, lse = log sum_j exp s_j, in one pass over the
// keys: the running maximum and sum of powers rescale what has been added
// when the maximum moves.  4 D operations per pair of a query row and a key.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_sweep.h"
#include "policy_launch.h"

namespace policy {
namespace {

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void attend_kernel(AttendArgs a, int tiles) {
  __shared__ __attribute__((aligned(16))) T k_even[kKeys * D], v_even[kKeys * D];
  __shared__ __attribute__((aligned(16))) T k_odd[kKeys * D], v_odd[kKeys * D];
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
  // Keys that a row sees: j <= last; those that all or any rows of the wave see.
  const int ahead = s.keys - s.queries;
  const int last = !on || !a.causal ? s.keys - 1 : min(s.keys - 1, me.query + ahead);
  const int last_row = min(first + kRowsOfBlock, rows) - 1;
  const int end = a.causal ? min(s.keys, last_row / a.group + ahead + 1) : s.keys;
  const int wave_first = min(first + 32 * wave, rows - 1);
  const int wave_last = min(wave_first + 31, rows - 1);
  const int all = !a.causal ? s.keys - 1 : min(s.keys - 1, wave_first / a.group + ahead);
  const int any = !a.causal ? s.keys - 1 : min(s.keys - 1, wave_last / a.group + ahead);

  Sweep<T, D, kKeys / 32> w;
  w.start(head_row<T>(a.q, s.q0 + me.query, me.head), a.dim, on);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const KeyTiles<T, D, kKeys, kThreads> tiles_of(a, s, kv);
  if (end > 0) tiles_of.fetch(0, k_even, v_even, a.dim);
  for (int j0 = 0; j0 < end; j0 += 2 * kKeys) {
    tiles_barrier();  // the tile is there, and nobody reads the other buffer any more
    if (j0 + kKeys < end) tiles_of.fetch(j0 + kKeys, k_odd, v_odd, a.dim);
    if (j0 <= any) w.add(k_even, v_even, 0, j0, UpTo{last}, j0 + kKeys - 1 <= all, c, places);
    if (j0 + kKeys >= end) break;
    tiles_barrier();
    if (j0 + 2 * kKeys < end) tiles_of.fetch(j0 + 2 * kKeys, k_even, v_even, a.dim);
    if (j0 + kKeys <= any)
      w.add(k_odd, v_odd, 0, j0 + kKeys, UpTo{last}, j0 + 2 * kKeys - 1 <= all, c, places);
  }
  const float sum = w.sum + __shfl_xor(w.sum, 32);
  if (!on) return;
  store_column<T, D>(head_row<T>(a.out, s.q0 + me.query, me.head), w.o, a.dim,
                     sum == 0.f ? 0.f : 1.f / sum);  // a sum of NaN stays one
  if (lane < 32)
    a.lse[int64_t(me.head) * a.q_rows + s.q0 + me.query] =
        sum == 0.f ? -INFINITY : __builtin_fmaf(w.reference(c), kLn2, ln(sum));
}

// --- few query rows -----------------------------------------------------------
//
// Where the query rows alone would leave the card idle, a sequence's keys are
// read by `splits` blocks, each for up to 32 rows (a single token's heads of one
// key head), and two waves of a block take 32 of each tile's 64 keys.  Their
// sums, in 32 bits and each with a reference of its own, are joined after them.
// Bound by the keys' and values' bytes.

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void split_kernel(AttendArgs a, Split p, int tiles) {
  __shared__ __attribute__((aligned(16))) T k_even[kKeys * D], v_even[kKeys * D];
  __shared__ __attribute__((aligned(16))) T k_odd[kKeys * D], v_odd[kKeys * D];
  const int kv = int(blockIdx.x) / tiles, split = int(blockIdx.y);
  const Tile tile = tile_of(a.q_offsets, a.n_seqs, a.q_rows, a.group, 32, int(blockIdx.x) % tiles);
  const Seq s = sequence(a, tile.seq);
  const int first = tile.index * 32, rows = s.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const int lane = int(threadIdx.x) % kWave, wave = wave_id();
  const bool on = first + lane % 32 < rows;
  const QueryRow me = query_row(a, kv, on ? first + lane % 32 : 0);
  const int ahead = s.keys - s.queries;
  const int last = !on || !a.causal ? s.keys - 1 : min(s.keys - 1, me.query + ahead);
  const int last_row = min(first + 32, rows) - 1;
  const int seen = a.causal ? min(s.keys, last_row / a.group + ahead + 1) : s.keys;
  const int all = a.causal ? min(s.keys - 1, first / a.group + ahead) : s.keys - 1;
  // This split's share of the keys that are seen, in whole tiles.
  const int share = ((max(seen, 0) + kKeys - 1) / kKeys + p.parts / 2 - 1) / (p.parts / 2) * kKeys;
  const int begin = min(split * share, max(seen, 0)), end = min(begin + share, seen);

  Sweep<T, D, 1> w;
  w.start(head_row<T>(a.q, s.q0 + me.query, me.head), a.dim, on);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const KeyTiles<T, D, kKeys, kThreads> tiles_of(a, s, kv);
  const int row = wave * 32;  // of the tile; waves 2 and 3 bring tiles only
  auto step = [&](int j0, const T* k_tile, const T* v_tile) {
    if (wave < 2 && j0 + row < end)
      w.add(k_tile, v_tile, row, j0 + row, UpTo{last}, j0 + row + 31 <= min(all, end - 1), c,
            places);
  };
  if (begin < end) tiles_of.fetch(begin, k_even, v_even, a.dim);
  for (int j0 = begin; j0 < end; j0 += 2 * kKeys) {
    tiles_barrier();
    if (j0 + kKeys < end) tiles_of.fetch(j0 + kKeys, k_odd, v_odd, a.dim);
    step(j0, k_even, v_even);
    if (j0 + kKeys >= end) break;
    tiles_barrier();
    if (j0 + 2 * kKeys < end) tiles_of.fetch(j0 + 2 * kKeys, k_even, v_even, a.dim);
    step(j0 + kKeys, k_odd, v_odd);
  }
  if (wave >= 2 || !on) return;
  const float sum = w.sum + __shfl_xor(w.sum, 32);
  const int64_t part = part_of(a, p, s.q0 + me.query, me.head, 2 * split + wave);
  store_column<float, D>(p.sums + part * D, w.o, D, 1.f);
  if (lane < 32) {
    p.weights[2 * part] = w.reference(c);
    p.weights[2 * part + 1] = sum;
  }
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendArgs a, Split p, int64_t first) {
  const int64_t i = first + int64_t(blockIdx.x) * (kThreads / kWave) + int(threadIdx.x) / kWave;
  if (i < int64_t(a.q_rows) * a.q_heads) join_row<T, D>(a, p, i);
}

// Blocks that a sequence's keys are shared by: 1 where there are 64 blocks of
// query rows (64 of them, 1,000 keys: 33 us so, 36 shared; 40 of them, 16,384
// keys: 320 us so, 153 shared) unless sequences have a wave's rows at most; else
// as many as give the card 4096 blocks, none of them with less than 256 keys of
// a sequence of the mean length.
int splits_of(const sched_attention_desc& d) {
  if (d.n_seqs == 0 || d.q_rows == 0) return 1;
  const int64_t rows = d.q_rows * (d.q_heads / d.kv_heads);
  if (rows / d.n_seqs > 32 && (rows / kRowsOfBlock + d.n_seqs) * d.kv_heads >= 64) return 1;
  const int64_t blocks = tile_count(rows, d.n_seqs, 32) * d.kv_heads;
  const int64_t want = (4096 + blocks - 1) / blocks, most = d.k_rows / d.n_seqs / 256;
  return int(std::max<int64_t>(1, std::min<int64_t>({want, most, 256})));
}

size_t part_count(const sched_attention_desc& d, int splits) {
  return size_t(d.q_rows) * size_t(d.q_heads) * size_t(2 * splits);
}

template <class T, int D>
hipError_t attend(const AttendArgs& a, int kv_heads, int splits, void* ws, size_t parts,
                  hipStream_t s) {
  if (splits == 1) {
    const int64_t tiles = tile_count(int64_t(a.q_rows) * a.group, a.n_seqs, kRowsOfBlock);
    hipLaunchKernelGGL((attend_kernel<T, D>), dim3(unsigned(work_blocks(tiles, kv_heads))),
                       dim3(kThreads), 0, s, a, int(tiles));
    return hipGetLastError();
  }
  const Split p = {static_cast<float*>(ws), static_cast<float*>(ws) + parts * D, 2 * splits};
  const int64_t tiles = tile_count(int64_t(a.q_rows) * a.group, a.n_seqs, 32);
  hipLaunchKernelGGL((split_kernel<T, D>), dim3(unsigned(tiles * kv_heads), unsigned(splits)),
                     dim3(kThreads), 0, s, a, p, int(tiles));
  hipError_t e = hipGetLastError();
  const int64_t blocks = (int64_t(a.q_rows) * a.q_heads + 3) / 4;
  for (int64_t b = 0; b < blocks && e == hipSuccess; b += kMostBlocks) {
    hipLaunchKernelGGL((join_kernel<T, D>), dim3(unsigned(std::min(blocks - b, kMostBlocks))),
                       dim3(kThreads), 0, s, a, p, b * 4);
    e = hipGetLastError();
  }
  return e;
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
  // Several long sequences (8 of 1,500 rows, 16 heads: backward 412 -> 326 us,
  // forward 108 -> 100; 40 of 400: forward 61 -> 70, so short ones do not), as many
  // as a wave has lanes: more fill the card in any order (64 of 300 to 2,500 rows, 8
  // heads of 2: forward and backward 466 and 1,500 us, 65 of them 428 and 1,485).
  a.ranked = d.n_seqs > 1 && d.n_seqs <= kWave && d.q_rows / d.n_seqs >= 1024;
  a.causal = d.causal;
  a.scale = d.scale;
  return a;
}

size_t attention_bytes(const sched_attention_desc& d) {
  const int splits = splits_of(d);
  const size_t each = size_t(d.head_dim > 64 ? 128 : 64) + 2;
  return splits == 1 ? 0 : part_count(d, splits) * each * sizeof(float);
}

hipError_t launch_attention(const sched_attention_desc& d, void* ws, hipStream_t s) {
  if (d.n_seqs == 0 || d.q_rows == 0) return hipSuccess;
  const AttendArgs a = attend_args(d);
  const int splits = splits_of(d);
  const size_t parts = part_count(d, splits);
  const bool wide = d.head_dim > 64;
  if (d.dtype == SCHED_F16)
    return wide ? attend<f16, 128>(a, d.kv_heads, splits, ws, parts, s)
                : attend<f16, 64>(a, d.kv_heads, splits, ws, parts, s);
  return wide ? attend<bf16, 128>(a, d.kv_heads, splits, ws, parts, s)
              : attend<bf16, 64>(a, d.kv_heads, splits, ws, parts, s);
}

}  // namespace policy
