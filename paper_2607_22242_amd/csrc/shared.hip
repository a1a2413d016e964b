// shared.hip -- attention of groups of sequences that share a prefix.
//
// out = sum_j exp(s_j - lse) v_j over the prefix keys of a row's group and its own
// sequence's keys up to its own place: one pass with a running maximum and sum.
// 4 D operations per pair of a query row and a key.  With many query rows a block
// takes 128 of a group (of several sequences and heads of one key head) and walks
// over both kinds of keys; with few the keys are shared by blocks.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_shared.h"
#include "attend_sweep.h"
#include "policy_launch.h"

namespace policy {
namespace {

// One turn of a block over its rows: all of them (nth < 0), which is done unless a
// sequence that holds what is no number has reached another's rows (true: nothing is
// written), or those of its nth sequence (true: there is one).
template <class T, int D>
__device__ __forceinline__ bool rows_turn(const SharedArgs& s, int block, int tiles,
                                          Buffers<T, D>& lds, int nth) {
  const AttendArgs& a = s.a;
  const bool by_one = nth >= 0;
  const Work work = work_of(block, tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return false;
  const int lane = int(threadIdx.x) % kWave;
  RowsOf<kRowsOfBlock> r(s, work, tiles, 32 * wave_id() + lane % 32);
  if (!r.there) return false;
  r.find(s);
  const int alone = r.first_seq + nth;
  if (by_one) {
    if (alone > r.last_seq) return false;
    tiles_barrier();  // nobody reads the last turn's tiles any more
  }
  const Seen seen(r.mine);
  Sweep<T, D, kKeys / 32> w;
  w.start(head_row<T>(a.q, r.query, r.me.head), a.dim, r.on);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const KeyTiles<T, D, kKeys, kThreads> prefix(s.p_k, s.p_v, r.g.p0, r.g.keys, s.near_p, a.dim,
                                               work.kv);
  Walk<T, D> walk(s, work.kv, by_one ? alone : r.first_seq, by_one ? alone : r.last_seq,
                  by_one ? r.last_key_of(s, alone) : r.last_key);
  over_keys<T, D>(
      prefix, a.dim, 0, r.g.keys, walk, true, lds,
      [&](int j0, const T* k, const T* v) {
        w.add(k, v, 0, j0, UpTo{r.g.keys - 1}, j0 + kKeys <= r.g.keys, c, places);
      },
      [&](const Step& t, const T* k, const T* v) {
        if (seen.any(t)) w.add(k, v, 0, t.key0, seen.keys(t), seen.all(t), c, places);
      });
  if (!by_one && r.first_seq < r.last_seq && __syncthreads_or(r.on && no_number(w.o))) return true;
  const float sum = w.sum + __shfl_xor(w.sum, 32);
  if (!r.on || (by_one && r.seq != alone)) return by_one;
  store_column<T, D>(head_row<T>(a.out, r.query, r.me.head), w.o, a.dim,
                     sum == 0.f ? 0.f : 1.f / sum);  // a sum of NaN stays one
  if (lane < 32)
    a.lse[int64_t(r.me.head) * a.q_rows + r.query] =
        sum == 0.f ? -INFINITY : __builtin_fmaf(w.reference(c), kLn2, ln(sum));
  return by_one;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void shared_kernel(SharedArgs s, int tiles) {
  __shared__ __attribute__((aligned(16))) Buffers<T, D> lds;
  int block = int(blockIdx.x);
  for (int nth = -1;; ++nth) {
    asm volatile("" : "+s"(block));  // a turn keeps nothing in registers for the next
    if (!rows_turn<T, D>(s, block, tiles, lds, nth)) return;
  }
}

// --- few query rows -----------------------------------------------------------
//
// Blocks of two kinds: of a group's rows (32 kAcross of them) with a share of the
// prefix keys, and of a sequence's rows (32) with a share of its own keys.  A row's
// sums over all shares are joined after them.  Bound by the keys' and values' bytes
// where groups are small, by the matrix instructions of the prefix where they are
// large: blocks of both kinds run side by side.

struct Shares {
  int p_tiles, p_splits, p_parts;  // tiles of the groups' rows; shares of the prefix; parts of a row
  int o_tiles, o_splits;
};

// One block's rows against tiles of 64 keys, begin <= j < end of `tiles_of`; wave_row:
// the wave's first key of a tile, kSubs 32 of them; a wave that has none brings tiles.
template <class T, int D, int kSubs>
__device__ __forceinline__ void sweep_share(Sweep<T, D, kSubs>& w,
                                            const KeyTiles<T, D, kKeys, kThreads>& tiles_of, int begin,
                                            int end, int wave_row, int last, int all, float c, int dim,
                                            T* k_even, T* v_even, T* k_odd, T* v_odd) {
  const Places<D> places;
  auto step = [&](int j0, const T* k_tile, const T* v_tile) {
    if (wave_row < kKeys && j0 + wave_row < end)
      w.add(k_tile, v_tile, wave_row, j0 + wave_row, UpTo{min(last, end - 1)},
            j0 + wave_row + 32 * kSubs - 1 <= min(all, end - 1), c, places);
  };
  if (begin < end) tiles_of.fetch(begin, k_even, v_even, dim);
  for (int j0 = begin; j0 < end; j0 += 2 * kKeys) {
    tiles_barrier();
    if (j0 + kKeys < end) tiles_of.fetch(j0 + kKeys, k_odd, v_odd, dim);
    step(j0, k_even, v_even);
    if (j0 + kKeys >= end) break;
    tiles_barrier();
    if (j0 + 2 * kKeys < end) tiles_of.fetch(j0 + 2 * kKeys, k_even, v_even, dim);
    step(j0 + kKeys, k_odd, v_odd);
  }
}

template <class T, int D, int kSubs>
__device__ __forceinline__ void store_part(const AttendArgs& a, const Split& p,
                                           const Sweep<T, D, kSubs>& w, int64_t row, int head,
                                           int part_, bool on, float c) {
  const float sum = w.sum + __shfl_xor(w.sum, 32);
  if (!on) return;
  const int64_t part = part_of(a, p, row, head, part_);
  store_column<float, D>(p.sums + part * D, w.o, D, 1.f);
  if (int(threadIdx.x) % kWave < 32) {
    p.weights[2 * part] = w.reference(c);
    p.weights[2 * part + 1] = sum;
  }
}

// kAcross: waves side by side along the rows of a group; the other waves share a
// tile's keys.
template <class T, int D, int kAcross>
__global__ __launch_bounds__(kThreads, 2) void shares_kernel(SharedArgs s, Split p, Shares n) {
  __shared__ __attribute__((aligned(16))) T k_even[kKeys * D], v_even[kKeys * D];
  __shared__ __attribute__((aligned(16))) T k_odd[kKeys * D], v_odd[kKeys * D];
  const AttendArgs& a = s.a;
  const int kv_heads = a.q_heads / a.group, kv = int(blockIdx.x) % kv_heads;
  const int lane = int(threadIdx.x) % kWave, wave = wave_id();
  const float c = a.scale * kLog2e;
  int block = int(blockIdx.x) / kv_heads;
  if (block < n.p_tiles * n.p_splits) {
    const int split = block / n.p_tiles;
    const Tile tile = group_tile(s, 32 * kAcross, block % n.p_tiles);
    const Group g = group_at(s, tile.seq);
    const int first = tile.index * 32 * kAcross, rows = g.queries * a.group;
    if (tile.index < 0 || first >= rows) return;
    const int r = first + wave % kAcross * 32 + lane % 32;
    const bool on = r < rows;
    const QueryRow me = query_row(a, kv, on ? r : 0);
    const int share = ((g.keys + kKeys - 1) / kKeys + n.p_splits - 1) / n.p_splits * kKeys;
    const int begin = min(split * share, g.keys), end = min(begin + share, g.keys);
    constexpr int kSubs = kAcross == 4 ? 2 : 1;
    Sweep<T, D, kSubs> w;
    w.start(head_row<T>(a.q, g.q0 + me.query, me.head), a.dim, on);
    const KeyTiles<T, D, kKeys, kThreads> tiles_of(s.p_k, s.p_v, g.p0, g.keys, s.near_p, a.dim, kv);
    sweep_share<T, D, kSubs>(w, tiles_of, begin, end, wave / kAcross * 32, g.keys - 1, g.keys - 1, c,
                             a.dim, k_even, v_even, k_odd, v_odd);
    if (wave / kAcross < 2)
      store_part<T, D, kSubs>(a, p, w, g.q0 + me.query, me.head,
                              kAcross == 4 ? split : 2 * split + wave / kAcross, on, c);
    return;
  }
  block -= n.p_tiles * n.p_splits;
  const int split = block / n.o_tiles;
  const Tile tile = tile_of(a.q_offsets, a.n_seqs, a.q_rows, a.group, 32, block % n.o_tiles);
  const Seq q = sequence(a, tile.seq);
  const int first = tile.index * 32, rows = q.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const bool on = first + lane % 32 < rows;
  const QueryRow me = query_row(a, kv, on ? first + lane % 32 : 0);
  const int ahead = q.keys - q.queries;
  const int last = !on || !a.causal ? q.keys - 1 : min(q.keys - 1, me.query + ahead);
  const int last_row = min(first + 32, rows) - 1;
  const int seen = max(0, a.causal ? min(q.keys, last_row / a.group + ahead + 1) : q.keys);
  const int all = a.causal ? min(q.keys - 1, first / a.group + ahead) : q.keys - 1;
  const int share = ((seen + kKeys - 1) / kKeys + n.o_splits - 1) / n.o_splits * kKeys;
  const int begin = min(split * share, seen), end = min(begin + share, seen);
  Sweep<T, D, 1> w;
  w.start(head_row<T>(a.q, q.q0 + me.query, me.head), a.dim, on);
  const KeyTiles<T, D, kKeys, kThreads> tiles_of(a, q, kv);
  sweep_share<T, D, 1>(w, tiles_of, begin, end, wave * 32, last, all, c, a.dim, k_even, v_even, k_odd,
                       v_odd);
  if (wave < 2)
    store_part<T, D, 1>(a, p, w, q.q0 + me.query, me.head, n.p_parts + 2 * split + wave, on, c);
}

// Rows of the groups' sequences only: others have no parts.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void join_shares_kernel(SharedArgs s, Split p, int64_t first) {
  const int64_t i = first + int64_t(blockIdx.x) * (kThreads / kWave) + int(threadIdx.x) / kWave;
  const int64_t row = i / s.a.q_heads;
  if (row >= first_query(s, 0) && row < first_query(s, s.n_groups)) join_row<T, D>(s.a, p, i);
}

struct Plan {
  bool split;
  int across;
  Shares n;
  int parts;
};

Plan plan_of(const sched_shared_desc& x) {
  const sched_attention_desc& d = x.own;
  Plan p = {};
  const int64_t group = d.q_heads / d.kv_heads, rows = d.q_rows * group;
  if (x.n_groups == 0 || d.n_seqs == 0 || rows == 0) return p;
  // Sequences with a wave's rows at most over caches, and whatever leaves the card idle.
  const int64_t blocks = tile_count(rows, x.n_groups, kRowsOfBlock) * d.kv_heads;
  p.split = (d.k_lengths && rows / d.n_seqs <= 32) || blocks < 128;
  if (!p.split) return p;
  const int64_t of_group = rows / x.n_groups;
  p.across = of_group > 64 ? 4 : of_group > 32 ? 2 : 1;
  p.n.p_tiles = int(tile_count(rows, x.n_groups, 32 * p.across));
  p.n.o_tiles = int(tile_count(rows, d.n_seqs, 32));
  auto splits = [&](int64_t tiles, int64_t keys, int64_t most_blocks) {
    const int64_t want = (most_blocks + tiles * d.kv_heads - 1) / (tiles * d.kv_heads);
    return int(std::max<int64_t>(1, std::min<int64_t>({want, keys / 256, 256})));
  };
  p.n.p_splits = splits(p.n.p_tiles, x.prefix_rows / x.n_groups, 1024);
  p.n.o_splits = splits(p.n.o_tiles, d.k_rows / d.n_seqs, 1024);
  p.n.p_parts = p.n.p_splits * (p.across == 4 ? 1 : 2);
  p.parts = p.n.p_parts + 2 * p.n.o_splits;
  return p;
}

size_t part_count(const sched_shared_desc& x, const Plan& p) {
  return size_t(x.own.q_rows) * size_t(x.own.q_heads) * size_t(p.parts);
}

template <class T, int D>
hipError_t shared(const SharedArgs& s, const Plan& n, void* ws, size_t parts, hipStream_t stream) {
  const int kv_heads = s.a.q_heads / s.a.group;
  if (!n.split) {
    const int64_t tiles = tile_count(int64_t(s.a.q_rows) * s.a.group, s.n_groups, kRowsOfBlock);
    hipLaunchKernelGGL((shared_kernel<T, D>), dim3(unsigned(work_blocks(tiles, kv_heads))),
                       dim3(kThreads), 0, stream, s, int(tiles));
    return hipGetLastError();
  }
  const Split p = {static_cast<float*>(ws), static_cast<float*>(ws) + parts * D, n.parts};
  const int64_t blocks =
      (int64_t(n.n.p_tiles) * n.n.p_splits + int64_t(n.n.o_tiles) * n.n.o_splits) * kv_heads;
  const dim3 grid = dim3(unsigned(blocks));
  if (n.across == 4)
    hipLaunchKernelGGL((shares_kernel<T, D, 4>), grid, dim3(kThreads), 0, stream, s, p, n.n);
  else if (n.across == 2)
    hipLaunchKernelGGL((shares_kernel<T, D, 2>), grid, dim3(kThreads), 0, stream, s, p, n.n);
  else
    hipLaunchKernelGGL((shares_kernel<T, D, 1>), grid, dim3(kThreads), 0, stream, s, p, n.n);
  hipError_t e = hipGetLastError();
  const int64_t joins = (int64_t(s.a.q_rows) * s.a.q_heads + 3) / 4;
  for (int64_t b = 0; b < joins && e == hipSuccess; b += kMostBlocks) {
    hipLaunchKernelGGL((join_shares_kernel<T, D>), dim3(unsigned(std::min(joins - b, kMostBlocks))),
                       dim3(kThreads), 0, stream, s, p, b * 4);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

SharedArgs shared_args(const sched_shared_desc& x) {
  SharedArgs s = {};
  s.a = attend_args(x.own);
  s.p_k = heads_view(x.prefix_k);
  s.p_v = heads_view(x.prefix_v);
  s.p_offsets = x.prefix_offsets;
  s.p_lengths = x.prefix_lengths;
  s.groups = x.group_offsets;
  s.n_groups = x.n_groups;
  s.p_rows = int32_t(x.prefix_rows);
  s.near_p = x.prefix_k.row_stride < (int64_t(1) << 24) && x.prefix_v.row_stride < (int64_t(1) << 24);
  return s;
}

size_t shared_bytes(const sched_shared_desc& x) {
  const Plan p = plan_of(x);
  const size_t each = size_t(x.own.head_dim > 64 ? 128 : 64) + 2;
  return p.split ? part_count(x, p) * each * sizeof(float) : 0;
}

hipError_t launch_shared(const sched_shared_desc& x, void* ws, hipStream_t stream) {
  const Plan p = plan_of(x);
  if (x.n_groups == 0 || x.own.n_seqs == 0 || x.own.q_rows == 0) return hipSuccess;
  const SharedArgs s = shared_args(x);
  const size_t parts = part_count(x, p);
  const bool wide = x.own.head_dim > 64;
  if (x.own.dtype == SCHED_F16)
    return wide ? shared<f16, 128>(s, p, ws, parts, stream) : shared<f16, 64>(s, p, ws, parts, stream);
  return wide ? shared<bf16, 128>(s, p, ws, parts, stream) : shared<bf16, 64>(s, p, ws, parts, stream);
}

}  // namespace policy
