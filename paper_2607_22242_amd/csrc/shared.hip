// shared.hip -- attention of groups of sequences that share a prefix.
//
// out = sum_j exp(s_j - lse) v_j over the prefix keys of a row's group and its own
// sequence's keys up to its own place: one pass with a running maximum and sum.
// 4 D operations per pair of a query row and a key.  With many query rows a block
// takes 128 of a group (of several sequences and heads of one key head) and walks
// over both kinds of keys, so that a prefix key is read once for 128 rows: bound by
// matrix instructions and the exponentials between them, at the clock that the card's
// power leaves (16 answers of 512 tokens to a prompt of 8,192, 32 heads of 128, bf16:
// 1,119 us, 1,013 TFLOP/s; halving what is read from LDS would save 5 % of it).  With
// few the keys are shared by blocks: bound by the bytes of the keys and values.
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
template <class T, int D, bool kFine>
__device__ __forceinline__ bool rows_turn(const SharedArgs& s, int block, int tiles,
                                          const Buffers<T>& lds, int nth) {
  const AttendArgs& a = s.a;
  const bool by_one = nth >= 0;
  const Work work = work_of(block, tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return false;
  const int lane = int(threadIdx.x) % kWave;
  RowsOf<kRowsOfBlock> r(s, work, tiles, 32 * wave_id() + lane % 32);
  if (!r.there) return false;
  const KeyTiles<T, D, kKeys, kThreads> prefix(s.p_k, s.p_v, r.g.p0, r.g.keys, s.near_p, a.dim,
                                               work.kv);
  Sweep<T, D, kKeys / 32, kFine> w;
  if (by_one) tiles_barrier();  // nobody reads the last turn's tiles any more
  if (r.g.keys > 0) prefix.fetch(0, lds.k_even, lds.v_even, a.dim);
  w.start(head_row<T>(a.q, r.query, r.me.head), a.dim, r.on);
  r.find(s);
  const int alone = r.first_seq + nth;
  if (by_one && alone > r.last_seq) return false;
  const Seen seen(r.mine);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  Walk<T, D> walk(s, work.kv, by_one ? alone : r.first_seq, by_one ? alone : r.last_seq,
                  by_one ? r.first_key_of(s, alone) : r.first_key,
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

template <class T, int D, bool kFine>
__global__ __launch_bounds__(kThreads, 2) void shared_kernel(SharedArgs s, int tiles) {
  __shared__ __attribute__((aligned(16))) T k_even[64 * D], v_even[64 * D];
  __shared__ __attribute__((aligned(16))) T k_odd[64 * D], v_odd[64 * D];
  const Buffers<T> lds = {k_even, v_even, k_odd, v_odd};
  int block = int(blockIdx.x);
  for (int nth = -1;; ++nth) {
    asm volatile("" : "+s"(block));  // a turn keeps nothing in registers for the next
    if (!rows_turn<T, D, kFine>(s, block, tiles, lds, nth)) return;
  }
}

// --- few query rows -----------------------------------------------------------
//
// Work is shared along the keys, and a row's sums over all shares are joined after
// them.  Blocks are of two kinds, mixed, so that what waits for memory runs beside what
// waits for the matrix instructions:
// together: up to 128 rows of a group with a share of the prefix keys, as above.
// apart: each wave takes 32 rows of a sequence (a single token's heads of one key
// head) with a share of its own keys, and reads them in tiles of 32 through LDS of its
// own, waiting for no other wave: eight waves on a unit keep the memory busy while some
// of them compute (512 sequences of 400 keys, 8 key heads: 5.3 TB/s).

constexpr int kStream = 32;  // keys of a wave's tile
constexpr int kWaves = kThreads / kWave;

struct Shares {
  int p_tiles, p_splits;  // together: tiles of 128 rows of the groups, shares of the prefix
  int o_tiles, o_splits;  // apart: tiles of 32 rows of the sequences, shares of their own keys
  int units, spread;      // of kv_heads blocks each, of both kinds; the first `spread` have
                          // those of the prefix, evenly
};

// Tiles of one wave, as KeyTiles has them.
template <class T, int D>
struct StreamTiles {
  static constexpr int kStep = kWave / (D / 8), kRounds = kStream / kStep;  // rows of a round
  const char *k, *v;  // the sequence's first row
  int64_t k_row, v_row;
  int keys, near, dim, row, turned;  // turned: this thread's piece of its row

  __device__ __forceinline__ StreamTiles(const HeadsView& ks, const HeadsView& vs, int k0, int keys_,
                                         int near_, int dim_, int kv)
      : k(reinterpret_cast<const char*>(head_row<T>(ks, k0, kv))),
        v(reinterpret_cast<const char*>(head_row<T>(vs, k0, kv))), k_row(ks.row * 2),
        v_row(vs.row * 2), keys(keys_), near(near_), dim(dim_),
        row(int(threadIdx.x) % kWave / (D / 8)),
        turned(int(threadIdx.x) % (D / 8) ^ turn_of<D>(int(threadIdx.x) % kWave / (D / 8))) {}

  // Rows j0 .. to LDS, in kRounds loads; those behind the last key repeat it.
  __device__ __forceinline__ void fetch_keys(int j0, T* tile) const { fetch(k, k_row, j0, tile); }
  __device__ __forceinline__ void fetch_values(int j0, T* tile) const { fetch(v, v_row, j0, tile); }

 private:
  __device__ __forceinline__ void fetch(const char* from, int64_t stride, int j0, T* tile) const {
    const bool whole = near && j0 + kStream <= keys;
#pragma unroll
    for (int p = 0; p < kRounds; ++p) {
      const uint32_t d = uint32_t(min(8 * (turned ^ turn_of<D>(p * kStep)), dim - 8)) * 2;
      T* const to = tile + p * kWave * 8;
      if (whole) {
        to_lds(from + (j0 + p * kStep) * stride, uint32_t(row) * uint32_t(stride) + d, to);
      } else {
        const int64_t r = min(j0 + p * kStep + row, keys - 1);
        to_lds(from + r * stride + d, 0, to);
      }
    }
  }
};

// A wave waits until no more than kLoads of its loads are under way, and until what it
// reads in LDS is read: the loads that follow may write there.
template <int kLoads>
__device__ __forceinline__ void wait_for_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
}
__device__ __forceinline__ void wait_for_reads() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

template <class T, int D, int kSubs, bool kFine>
__device__ __forceinline__ void store_part(const AttendArgs& a, const Split& p,
                                           const Sweep<T, D, kSubs, kFine>& w, int64_t row, int head,
                                           int part, bool on, float c) {
  const float sum = w.sum + __shfl_xor(w.sum, 32);
  if (!on) return;
  const int64_t at = part_of(a, p, row, head, part);
  store_column<float, D>(p.sums + at * D, w.o, D, 1.f);
  if (int(threadIdx.x) % kWave < 32) {
    p.weights[2 * at] = w.reference(c);
    p.weights[2 * at + 1] = sum;
  }
}

// Keys of a share of the prefix, in whole tiles: the longest prefix' keys over
// `splits`, so that shares are equal work; shorter ones have fewer of them.
__device__ __forceinline__ int prefix_share(const SharedArgs& s, int splits) {
  int most = 0;
  for (int g = int(threadIdx.x) % kWave; g < s.n_groups; g += kWave) {
    const int slot = offset_at(s.p_offsets, g + 1, s.p_rows) - offset_at(s.p_offsets, g, s.p_rows);
    most = max(most, s.p_lengths ? min(slot, s.p_lengths[g]) : slot);
  }
  return ((wave_most(most) + kKeys - 1) / kKeys + splits - 1) / splits * kKeys;
}

template <class T, int D, bool kFine>
__device__ __forceinline__ void share_together(const SharedArgs& s, const Split& p, const Shares& n,
                                               int unit, int kv, const Buffers<T>& lds) {
  const AttendArgs& a = s.a;
  const int split = unit / n.p_tiles, lane = int(threadIdx.x) % kWave;
  const GroupTile tile = group_tile<false>(s, kRowsOfBlock, unit % n.p_tiles);
  const Group& g = tile.g;
  const int first = tile.index * kRowsOfBlock, rows = g.queries * a.group;
  if (tile.index < 0 || first >= rows) return;
  const int r = first + wave_id() * 32 + lane % 32;
  const bool on = r < rows;
  const QueryRow me = query_row(a, kv, on ? r : 0);
  const int share = prefix_share(s, n.p_splits);
  const int begin = min(split * share, g.keys), end = min(begin + share, g.keys);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  Sweep<T, D, kKeys / 32, kFine> w;
  w.start(head_row<T>(a.q, g.q0 + me.query, me.head), a.dim, on);
  const KeyTiles<T, D, kKeys, kThreads> tiles_of(s.p_k, s.p_v, g.p0, g.keys, s.near_p, a.dim, kv);
  const bool any = first + wave_id() * 32 < rows;  // other waves bring tiles only
  auto add = [&](int j0, const T* k_tile, const T* v_tile) {
    if (any) w.add(k_tile, v_tile, 0, j0, UpTo{g.keys - 1}, j0 + kKeys <= g.keys, c, places);
  };
  if (begin < end) tiles_of.fetch(begin, lds.k_even, lds.v_even, a.dim);
  for (int j0 = begin; j0 < end; j0 += 2 * kKeys) {
    tiles_barrier();
    if (j0 + kKeys < end) tiles_of.fetch(j0 + kKeys, lds.k_odd, lds.v_odd, a.dim);
    add(j0, lds.k_even, lds.v_even);
    if (j0 + kKeys >= end) break;
    tiles_barrier();
    if (j0 + 2 * kKeys < end) tiles_of.fetch(j0 + 2 * kKeys, lds.k_even, lds.v_even, a.dim);
    add(j0 + kKeys, lds.k_odd, lds.v_odd);
  }
  store_part<T, D>(a, p, w, g.q0 + me.query, me.head, split, on, c);
}

template <class T, int D, bool kFine>
__device__ __forceinline__ void share_apart(const SharedArgs& s, const Split& p, const Shares& n,
                                            int unit, int kv, T* k_tile, T* v_tile) {
  const AttendArgs& a = s.a;
  const int lane = int(threadIdx.x) % kWave;
  const int split = unit / n.o_tiles;
  if (split >= n.o_splits) return;
  const Tile tile = tile_of(a.q_offsets, a.n_seqs, a.q_rows, a.group, 32, unit % n.o_tiles);
  const Seq q = sequence(a, tile.seq);
  const int first = tile.index * 32, rows = q.queries * a.group;
  if (first < 0 || first >= rows) return;
  // The lane's row sees the keys up to `last`, all rows those up to `all`, some row
  // those before `seen`.
  const int ahead = q.keys - q.queries, last_row = min(first + 32, rows) - 1;
  const int seen = max(0, a.causal ? min(q.keys, last_row / a.group + ahead + 1) : q.keys);
  const int all = a.causal ? min(q.keys - 1, first / a.group + ahead) : q.keys - 1;
  const int last =
      a.causal ? min(q.keys - 1, min(first + lane % 32, rows - 1) / a.group + ahead) : q.keys - 1;
  const int share = ((seen + kStream - 1) / kStream + n.o_splits - 1) / n.o_splits * kStream;
  const int begin = min(split * share, seen), end = min(begin + share, seen);
  const StreamTiles<T, D> tiles(a.k, a.v, q.k0, q.keys, a.near_k, a.dim, kv);
  if (begin < end) {
    tiles.fetch_keys(begin, k_tile);
    tiles.fetch_values(begin, v_tile);
  }
  const bool on = first + lane % 32 < rows;
  const QueryRow me = query_row(a, kv, on ? first + lane % 32 : first);
  Sweep<T, D, 1, kFine> w;
  w.start(head_row<T>(a.q, q.q0 + me.query, me.head), a.dim, on);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  constexpr int kLoads = StreamTiles<T, D>::kRounds;
  for (int j0 = begin; j0 < end; j0 += kStream) {
    const bool more = j0 + kStream < end;
    const Rows<T, D> ks = {k_tile, places.fresh()}, vs = {v_tile, ks.places};
    Acc x[1];
    wait_for_loads<kLoads>();  // the keys are there, the values may be under way
    w.scores(ks, 0, x);
    if (more) {
      wait_for_reads();
      tiles.fetch_keys(j0 + kStream, k_tile);
      wait_for_loads<kLoads>();  // the values are there
    } else {
      wait_for_loads<0>();
    }
    w.weigh(vs, 0, x, j0, UpTo{min(last, end - 1)}, j0 + kStream - 1 <= min(all, end - 1), c);
    if (more) {
      wait_for_reads();
      tiles.fetch_values(j0 + kStream, v_tile);
    }
  }
  store_part<T, D>(a, p, w, q.q0 + me.query, me.head, n.p_splits + split, on, c);
}

template <class T, int D, bool kFine>
__global__ __launch_bounds__(kThreads, 2) void shares_kernel(SharedArgs s, Split p, Shares n) {
  __shared__ __attribute__((aligned(16))) T k_even[64 * D], v_even[64 * D];
  __shared__ __attribute__((aligned(16))) T k_odd[64 * D], v_odd[64 * D];
  const Buffers<T> lds = {k_even, v_even, k_odd, v_odd};
  const int kv_heads = s.a.q_heads / s.a.group;
  const int unit = int(blockIdx.x) / kv_heads, kv = int(blockIdx.x) % kv_heads;
  const int p_units = n.p_tiles * n.p_splits;
  const int together = int(int64_t(min(unit, n.spread)) * p_units / n.spread);
  if (unit < n.spread && int(int64_t(unit + 1) * p_units / n.spread) > together) {
    share_together<T, D, kFine>(s, p, n, together, kv, lds);
    return;
  }
  const int wave = wave_id();
  const int64_t apart = (int64_t(unit - together) * kv_heads + kv) * kWaves + wave;
  const int its = int(apart / kv_heads), its_kv = int(apart % kv_heads);
  // Keys and values in arrays that the compiler tells apart (Buffers).
  const int at = wave % 2 * kStream * D;
  if (wave < 2) share_apart<T, D, kFine>(s, p, n, its, its_kv, k_even + at, v_even + at);
  else share_apart<T, D, kFine>(s, p, n, its, its_kv, k_odd + at, v_odd + at);
}

// Joins the parts of rows of the groups' sequences (others have none): a wave per row
// and head, D / 4 lanes a part, four elements each.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void join_shares_kernel(SharedArgs s, Split p, int64_t first) {
  typedef float Four __attribute__((ext_vector_type(4)));
  typedef T four __attribute__((ext_vector_type(4)));
  constexpr int kLanes = D / 4, kSides = kWave / kLanes, kAhead = 8;  // parts on their way at once
  const AttendArgs& a = s.a;
  const int lane = int(threadIdx.x) % kWave, side = lane / kLanes;
  const int64_t i = (first + int64_t(blockIdx.x)) * kWaves + wave_id();
  const int64_t row = i / a.q_heads;
  const int head = int(i - row * a.q_heads);
  if (row < first_query(s, 0) || row >= first_query(s, s.n_groups)) return;
  const float* const weights = p.weights + i * p.parts * 2;
  const float* const sums = p.sums + i * p.parts * D + lane % kLanes * 4;
  float most = -INFINITY;
  for (int k = lane; k < p.parts; k += kWave)
    if (weights[2 * k + 1] != 0.f) most = fmaxf(most, weights[2 * k]);
  most = wave_max(most);
  Four o = Four(0.f);
  float sum = 0.f;
  for (int k0 = 0; k0 < p.parts; k0 += kWave) {
    // A part's factor and sum, by the lane that has it.
    float f = 0.f, part = 0.f;
    if (k0 + lane < p.parts && weights[2 * (k0 + lane) + 1] != 0.f) {
      f = pow2(weights[2 * (k0 + lane)] - most);
      part = weights[2 * (k0 + lane) + 1] * f;
    }
    sum += wave_sum(part);
    for (int k = 0; k < min(kWave, p.parts - k0); k += kAhead * kSides) {
      float g[kAhead];
      Four x[kAhead];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) {
        const int at = k + n * kSides + side;
        const float its = __shfl(f, at % kWave);
        g[n] = at < kWave ? its : 0.f;
        x[n] = Four(0.f);
        if (g[n] != 0.f)  // what a part of no weight holds is not read
          x[n] = *reinterpret_cast<const Four*>(sums + int64_t(k0 + at) * D);
      }
#pragma unroll
      for (int n = 0; n < kAhead; ++n) o += g[n] * x[n];
    }
  }
#pragma unroll
  for (int d = kLanes; d < kWave; d *= 2)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], d);
  four v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = T(sum == 0.f ? 0.f : o[e] / sum);
  const int d = lane % kLanes * 4;
  if (side == 0 && d < a.dim) *reinterpret_cast<four*>(head_row<T>(a.out, row, head) + d) = v;
  if (lane == 0)
    a.lse[int64_t(head) * a.q_rows + row] =
        sum == 0.f ? -INFINITY : __builtin_fmaf(most, kLn2, ln(sum));
}

struct Plan {
  bool split;
  Shares n;
  int parts;
};

Plan plan_of(const sched_shared_desc& x) {
  const sched_attention_desc& d = x.own;
  Plan p = {};
  const int64_t group = d.q_heads / d.kv_heads, rows = d.q_rows * group;
  if (x.n_groups == 0 || d.n_seqs == 0 || rows == 0) return p;
  // Sequences with a wave's rows at most over caches, whose own keys 128 rows of several
  // sequences would share a tile's work for (8 groups of 64 single tokens: 147 us by
  // shares, 400 else), and whatever leaves the card idle (2 groups of 2 and 4 times 32
  // tokens, 32 heads, 48 and 80 blocks: 19 and 26 us by shares, 34 and 35 else; of 8 and
  // 16 times, 144 and 272 blocks: 36 and 59, 35 and 43).
  const int64_t blocks = tile_count(rows, x.n_groups, kRowsOfBlock) * d.kv_heads;
  p.split = (d.k_lengths && rows / d.n_seqs <= 32) || blocks < 128;
  if (!p.split) return p;
  // Shares of the prefix for some 448 blocks, so that the card's 512 places take own
  // keys beside them; of own keys for 2,048 waves (2 groups of 4 sequences, 64 heads, 8
  // key heads, prompts of 1,000 to 2,000, 1,000 to 4,000 own keys: 31 us, 39 with 1,024;
  // 4 sequences of 10,000 to 30,000 own keys: 88, 96); none of less than 256 and 128
  // keys on average.  A group's rows that are one wave's leave the prefix bound by
  // memory, too, and its blocks, the longest, come first (prompts of 20,000 to 32,000,
  // up to 2,000 own keys: 73 us, 80 in turn); more rows compute, and memory is kept busy
  // by own keys beside them, all but the last quarter of which go in turn with them (8
  // groups of 64 sequences: 142 us, 147.5 if all do, 155 one after the other; one group
  // of 16 with a prompt of 31,000: 58.5, 61 and 68).
  Shares& n = p.n;
  n.p_tiles = int(tile_count(rows, x.n_groups, kRowsOfBlock));
  n.o_tiles = int(tile_count(rows, d.n_seqs, 32));
  auto splits = [&](int64_t blocks, int64_t want, int64_t keys, int64_t least) {
    return int(std::max<int64_t>(
        1, std::min<int64_t>({(want + blocks - 1) / blocks, keys / least, 256})));
  };
  const int64_t of_group = (rows / x.n_groups + kRowsOfBlock - 1) / kRowsOfBlock;
  n.p_splits = splits(x.n_groups * std::max<int64_t>(of_group, 1) * d.kv_heads, 448,
                      x.prefix_rows / x.n_groups, 256);
  n.o_splits = splits(n.o_tiles * int64_t(d.kv_heads), 2048, d.k_rows / d.n_seqs, 128);
  n.units = n.p_tiles * n.p_splits + (n.o_tiles * n.o_splits + kWaves - 1) / kWaves;
  const int p_units = n.p_tiles * n.p_splits;
  n.spread = rows / x.n_groups <= 32 ? p_units : n.units - (n.units - p_units) / 4;
  p.parts = n.p_splits + n.o_splits;
  return p;
}

size_t part_count(const sched_shared_desc& x, const Plan& p) {
  return size_t(x.own.q_rows) * size_t(x.own.q_heads) * size_t(p.parts);
}

template <class T, int D, bool kFine>
hipError_t shared(const SharedArgs& s, const Plan& n, void* ws, size_t parts, hipStream_t stream) {
  const int kv_heads = s.a.q_heads / s.a.group;
  if (!n.split) {
    const int64_t tiles = tile_count(int64_t(s.a.q_rows) * s.a.group, s.n_groups, kRowsOfBlock);
    hipLaunchKernelGGL((shared_kernel<T, D, kFine>), dim3(unsigned(work_blocks(tiles, kv_heads))),
                       dim3(kThreads), 0, stream, s, int(tiles));
    return hipGetLastError();
  }
  const Split p = {static_cast<float*>(ws), static_cast<float*>(ws) + parts * D, n.parts};
  hipLaunchKernelGGL((shares_kernel<T, D, kFine>), dim3(unsigned(n.n.units) * unsigned(kv_heads)),
                     dim3(kThreads), 0, stream, s, p, n.n);
  hipError_t e = hipGetLastError();
  const int64_t joins = (int64_t(s.a.q_rows) * s.a.q_heads + kWaves - 1) / kWaves;
  for (int64_t b = 0; b < joins && e == hipSuccess; b += kMostBlocks) {
    hipLaunchKernelGGL((join_shares_kernel<T, D>), dim3(unsigned(std::min(joins - b, kMostBlocks))),
                       dim3(kThreads), 0, stream, s, p, b);
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
  auto run = [&](auto fine) {
    constexpr bool kFine = decltype(fine)::value;
    const bool wide = x.own.head_dim > 64;
    if (x.own.dtype == SCHED_F16)
      return wide ? shared<f16, 128, kFine>(s, p, ws, parts, stream)
                  : shared<f16, 64, kFine>(s, p, ws, parts, stream);
    return wide ? shared<bf16, 128, kFine>(s, p, ws, parts, stream)
                : shared<bf16, 64, kFine>(s, p, ws, parts, stream);
  };
  return is_small(x) ? run(std::true_type()) : run(std::false_type());
}

}  // namespace policy
