// shared_grad.hip -- the backward pass of attention over shared prefixes, which
// computes the probabilities again from the products and lse.
//
// With P = exp(scale Q K^T - lse) and delta = rowsum(dO o O):
// dV = P^T dO, dP = dO V^T, dS = P o (dP - delta), dQ = scale dS K,
// dK = scale dS^T Q, over both kinds of keys; a prefix key's sums run over all
// rows of its group.  One kernel holds query rows and walks over the keys (dQ),
// one holds keys, of either kind, and walks over the rows (dK, dV): no atomics,
// every sum has one order, for 14 D operations a pair in place of the 10 D of one
// kernel.  Bound as the forward pass: 16 answers of 512 tokens to a prompt of 8,192,
// 32 heads of 128, bf16: dQ 1,490 us (1,141 TFLOP/s), dK and dV 2,232 (1,016).
// Probabilities and dS are rounded to 16 bits for their products, all else is held in
// 32: errors are 1.4 to 1.5 times those of rounding the results alone, or, with second
// products (kFine), 1.0 to 1.15 times.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_shared.h"
#include "attend_grad_sweep.h"
#include "policy_launch.h"

namespace policy {
namespace {

// --- dQ -------------------------------------------------------------------------

// One turn of a block over its rows: all of them (nth < 0), which is done unless a
// sequence that holds what is no number has reached another's rows (true: nothing is
// written), or those of its nth sequence (true: there is one).
template <class T, int D, bool kFine>
__device__ __forceinline__ bool rows_turn(const SharedArgs& s, const RowParts& p, int block,
                                          int tiles, const Buffers<T>& lds, int nth) {
  const AttendArgs& a = s.a;
  const bool by_one = nth >= 0;
  const Work work = work_of(block, tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return false;
  const int lane = int(threadIdx.x) % kWave, part = int(blockIdx.y);
  RowsOf<kRowsOfBlock> r(s, work, tiles, 32 * wave_id() + lane % 32);
  if (!r.there) return false;
  // This block's share of the prefix; the last one has the own keys too.
  const int share = ((r.g.keys + kTile - 1) / kTile + p.parts - 1) / p.parts * kTile;
  const int begin = min(part * share, r.g.keys), end = min(begin + share, r.g.keys);
  const bool with_own = part == p.parts - 1;

  RowSweep<T, D, kFine> w;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const int d = 16 * i + 8 * (lane / 32);
    w.q[i] = piece(head_row<T>(a.q, r.query, r.me.head), d, a.dim, r.on);
    w.o[i] = piece(head_row<T>(a.d_out, r.query, r.me.head), d, a.dim, r.on);
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) w.dq[i] = Acc(0.f);
  r.find(s);
  const int alone = r.first_seq + nth;
  if (by_one && (alone > r.last_seq || !with_own)) return false;
  const Seen seen(r.mine);
  // The row's statistics, which the kernel of dK and dV reads too.
  const int64_t n = int64_t(r.me.head) * a.q_rows + r.query;
  const T* const out_row = head_row<T>(a.out, r.query, r.me.head);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const auto x = piece(out_row, 16 * i + 8 * (lane / 32), a.dim, r.on);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += float(x[e]) * float(w.o[i][e]);
  }
  w.delta = -(sum + __shfl_xor(sum, 32));
  const float lse = r.on ? a.lse[n] : -INFINITY;
  w.lse2 = lse == -INFINITY ? INFINITY : lse * kLog2e;  // powers of rows that see nothing are 0
  const bool mine = r.on && (!by_one || r.seq == alone);  // is the row this turn's
  const bool first_part = lane < 32 && mine && part == 0;
  if (first_part) a.lse2[n] = w.lse2 - kLiftGrad<T>;
  w.up = kShort<T> ? kLargest : 0;
  w.lse2 -= float(w.up);
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const KeyTiles<T, D, kTile, kThreads> prefix(s.p_k, s.p_v, r.g.p0, r.g.keys, s.near_p, a.dim,
                                               work.kv);
  const int first_seq = by_one ? alone : r.first_seq, last_seq = by_one ? alone : r.last_seq;
  const int first_key = by_one ? r.first_key_of(s, alone) : r.first_key;
  const int last_key = by_one ? r.last_key_of(s, alone) : r.last_key;
  if (by_one) tiles_barrier();  // nobody reads the last turn's tiles any more
  // Rows that see a tile's worth of keys at most take delta from the probabilities,
  // as sum_j P_j dP_j: from the rounded out it is off by a rounding of out, which
  // with few keys is as much as all other roundings together (errors of dQ and dK
  // against 64 bits, 5 to 30 keys: 1.65 times those of rounding once, 1.4 so).
  const bool few = r.g.keys + seen.most() <= kTile;
  if (__syncthreads_or(few && r.last_key - r.first_key < 16 * kTile)) {
    float dots = 0.f;
    if (r.g.keys > 0) {  // a tile's worth at most, or no row of the block is one of them
      prefix.fetch(0, lds.k_even, lds.v_even, a.dim);
      tiles_barrier();
      if (few) dots += w.dots(lds.k_even, lds.v_even, 0, UpTo{r.g.keys - 1}, c, places);
      tiles_barrier();
    }
    Walk<T, D> walk(s, work.kv, first_seq, last_seq, first_key, last_key);
    for (Step t = walk.next(lds.k_even, lds.v_even); t.there; t = walk.next(lds.k_even, lds.v_even)) {
      tiles_barrier();
      if (few && seen.any(t)) dots += w.dots(lds.k_even, lds.v_even, t.key0, seen.keys(t), c, places);
      tiles_barrier();
    }
    if (few) w.delta = -__builtin_ldexpf(dots + __shfl_xor(dots, 32), -w.up);
  }
  if (begin < end) prefix.fetch(begin, lds.k_even, lds.v_even, a.dim);
  Walk<T, D> walk(s, work.kv, first_seq, last_seq, first_key, last_key);
  over_keys<T, D>(
      prefix, a.dim, begin, end, walk, with_own, lds,
      [&](int j0, const T* k, const T* v) {
        w.add(k, v, j0, UpTo{r.g.keys - 1}, j0 + kTile <= r.g.keys, c, places);
      },
      [&](const Step& t, const T* k, const T* v) {
        if (seen.any(t)) w.add(k, v, t.key0, seen.keys(t), seen.all(t), c, places);
      });
  if (!by_one && with_own && r.first_seq < r.last_seq &&
      __syncthreads_or(r.on && (no_number(w.dq) || w.delta * 0.f != 0.f)))
    return true;
  if (!mine) return by_one;
  if (first_part) a.delta[n] = w.delta;
  if (kShort<T>) shift(w.dq, -w.up);
  if (r.g.keys == 0 && r.mine.hi < r.mine.lo) {  // a row that sees nothing, whatever it holds
#pragma unroll
    for (int i = 0; i < D / 32; ++i) w.dq[i] = Acc(0.f);
  }
  if (p.parts > 1)
    store_column<float, D>(p.dq + row_part<D>(a, part, r.query, r.me.head), w.dq, D, a.scale);
  else
    store_column<T, D>(head_row<T>(a.d_q, r.query, r.me.head), w.dq, a.dim, a.scale);
  return by_one;
}

// Heads of up to 64 elements leave room for three blocks on a unit, not two, if some
// registers that hardly anything asks for go to memory: over 16 answers of 300 tokens
// to each of 4 prompts of 2,000, 16 heads of 64, dQ 343 -> 308 us and dK and dV 452 ->
// 443 (f16: 366 -> 328, 490 -> 512); over 13 times 64 answers of 14 tokens, 4 heads of
// 32, 19 -> 20.6 and 22.5 -> 19.5.
template <int D, bool kFine>
constexpr int kBlocksOfUnit = D == 64 && !kFine ? 3 : 2;

template <class T, int D, bool kFine>
__global__ __launch_bounds__(kThreads, (kBlocksOfUnit<D, kFine>)) void shared_queries_kernel(
    SharedArgs s, RowParts p, int tiles) {
  __shared__ __attribute__((aligned(16))) T k_even[64 * D], v_even[64 * D];
  __shared__ __attribute__((aligned(16))) T k_odd[64 * D], v_odd[64 * D];
  const Buffers<T> lds = {k_even, v_even, k_odd, v_odd};
  int block = int(blockIdx.x);
  for (int nth = -1;; ++nth) {
    asm volatile("" : "+s"(block));  // a turn keeps nothing in registers for the next
    if (!rows_turn<T, D, kFine>(s, p, block, tiles, lds, nth)) return;
  }
}

// Adds the parts of the groups' rows: four elements of a head a thread.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void add_shared_rows_kernel(SharedArgs s, RowParts p,
                                                                   int64_t first) {
  typedef float Four __attribute__((ext_vector_type(4)));
  typedef T four __attribute__((ext_vector_type(4)));
  const AttendArgs& a = s.a;
  const int64_t i = (first + int64_t(blockIdx.x)) * kThreads + int(threadIdx.x);
  const int d = int(i % (D / 4)) * 4, head = int(i / (D / 4) % a.q_heads);
  const int64_t row = i / (D / 4) / a.q_heads;
  if (d >= a.dim || row < first_query(s, 0) || row >= first_query(s, s.n_groups)) return;
  Four x = Four(0.f);
  for (int n = 0; n < p.parts; ++n)
    x += *reinterpret_cast<const Four*>(p.dq + row_part<D>(a, n, row, head) + d);
  four u;
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] = T(x[e]);
  *reinterpret_cast<four*>(head_row<T>(a.d_q, row, head) + d) = u;
}

// --- dK and dV --------------------------------------------------------------------

// Where prefix keys are few a block's rows are shared by `parts` blocks.
struct PrefixParts {
  float *dk, *dv;  // parts x kv_heads x prefix rows x D
  int parts;
};
template <int D>
__device__ __forceinline__ int64_t prefix_part(const SharedArgs& s, int part, int kv, int64_t row) {
  return ((int64_t(part) * (s.a.q_heads / s.a.group) + kv) * s.p_rows + row) * D;
}

// A block holds 64 keys; waves 0 and 1 take the even 32 rows of each tile with
// keys 0 .. 31 and 32 .. 63, waves 2 and 3 the odd 32; their sums meet at the end.
// The first p_blocks blocks hold prefix keys; the others hold own keys, of one
// sequence or several.
// Turns are those of rows_turn, over the sequences of own keys.
template <class T>
struct KeyBuffers {  // arrays in LDS
  T *q_even, *o_even, *q_odd, *o_odd, *v_rest;
  Stats *s_even, *s_odd;
  int *from, *upto;  // rows that see a key
  int* seq;          // its sequence; -1: not in use, -2: another block's
};
template <class T, int D, bool kPrefix, bool kFine>
__device__ __forceinline__ bool keys_turn(const SharedArgs& s, const PrefixParts& p, int block,
                                          int blocks, int tiles, const KeyBuffers<T>& lds, int nth) {
  const AttendArgs& a = s.a;
  const bool by_one = !kPrefix && nth >= 0;
  const int part_of_rows = kPrefix ? block / blocks : 0;
  const Work work = work_of(block - part_of_rows * blocks, tiles, a.q_heads / a.group);
  if (work.tile >= tiles) return false;
  const int lane = int(threadIdx.x) % kWave, wave = wave_id();
  const int kv = work.kv, part = wave / 2 * 32, wave_row = wave % 2 * 32;
  const HeadsView &ks = kPrefix ? s.p_k : a.k, &vs = kPrefix ? s.p_v : a.v;

  // The lane's key and the rows that see it: of its sequence's (its group's) `count`
  // rows, which begin at query `query`, those from `seen` on.  What only the ends of
  // the loop below ask for lies in LDS: registers are short.
  int first, key, query, seen, count;
  int in_use = 0, owned = 0;  // prefix: rows before them are, in use and at all
  bool held, on;  // is the row this block's; is it a key in use
  // The block's rows, which begin at query q0; none before row block_from sees a key.
  int q0, rows, block_from;
  int seq = 0, low_seq = 0, high_seq = 0;  // own keys: the lane's sequence, the block's
  if (kPrefix) {
    const GroupTile tile = group_tile<true>(s, kKeysOfBlock, work.tile);
    const Group& g = tile.g;
    const int at = tile.index * kKeysOfBlock, j = at + wave_row + lane % 32;
    if (tile.index < 0 || at >= g.slot) return false;
    first = g.p0 + at;
    in_use = g.p0 + g.keys;
    owned = g.p0 + g.slot;
    key = g.p0 + j;
    held = j < g.slot;
    on = j < g.keys;
    query = q0 = g.q0;
    count = rows = at < g.keys ? g.queries * a.group : 0;
    seen = block_from = 0;
  } else {
    const int first_seq = uniform(first_sequence(s, 0));
    const int seqs = uniform(first_sequence(s, s.n_groups)) - first_seq;
    if (seqs <= 0) return false;
    const int behind = uniform(offset_at(a.k_offsets, first_seq + seqs, a.k_rows));
    first = uniform(offset_at(a.k_offsets, first_seq, a.k_rows)) + work.tile * kKeysOfBlock;
    if (first >= behind) return false;
    const int last = min(first + kKeysOfBlock, behind) - 1;
    key = first + wave_row + lane % 32;
    held = key <= last;
    const Held its = sequences_of(a.k_offsets, a.k_rows, first_seq, seqs, first, last, min(key, last));
    seq = its.mine;
    low_seq = uniform(its.low);
    high_seq = uniform(its.high);
    const Seq q = lane_sequence(a, seq), head = sequence(a, low_seq), tail = sequence(a, high_seq);
    // The first query of a sequence that sees key j of it; `queries` if none does.
    auto seen_from = [&](const Seq& x, int j) {
      return a.causal ? min(max(0, j - (x.keys - x.queries)), x.queries) : 0;
    };
    on = held && key - q.k0 < q.keys;
    query = q.q0;
    count = q.queries * a.group;
    seen = seen_from(q, key - q.k0) * a.group;
    q0 = head.q0;
    rows = max(0, tail.q0 + tail.queries - q0) * a.group;
    block_from = seen_from(head, first - head.k0) * a.group;
  }
  const float c = a.scale * kLog2e;
  const Places<D> places;
  const int alone = low_seq + nth;
  if (by_one) {
    if (alone > high_seq) return false;
    const Seq q = sequence(a, alone);
    q0 = q.q0;
    rows = q.queries * a.group;
    block_from = 0;
    tiles_barrier();  // nobody reads the last turn's tiles any more
  }
  const Rows<T, 64> rest = {lds.v_rest, Places<64>()};
  KeySweep<T, D, kFine> w;
  {
    const int64_t row = on ? key : 0;
    const T *k_row = head_row<T>(ks, row, kv), *v_row = head_row<T>(vs, row, kv);
    const int h = lane / 32, at = wave_row + lane % 32;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      w.k[i] = piece(k_row, 16 * i + 8 * h, a.dim, on);
      const auto v = piece(v_row, 16 * i + 8 * h, a.dim, on);
      if (i < KeySweep<T, D>::kHeld)
        w.v[i] = v;
      else if (part == 0)
        *reinterpret_cast<typename Frag<T>::type*>(
            lds.v_rest + at * 64 + ((2 * (i - KeySweep<T, D>::kHeld) + h) ^ turn_of<64>(at)) * 8) = v;
    }
  }
  const RowTiles<T, D> tiles_of(a);
  // Rows that all, or any, of the wave's keys are seen by.
  int all_from, all_upto, any_from, any_upto;
  {
    const bool counts = on && (!by_one || seq == alone);
    const int from = counts ? (query - q0) * a.group + seen : rows;
    const int upto = counts ? (query - q0) * a.group + count - 1 : -1;
    all_from = wave_most(from);
    all_upto = wave_least(upto);
    any_from = wave_least(from);
    any_upto = wave_most(upto);
    const int at = wave_row + lane % 32;
    if (!kPrefix && part == 0) {  // read behind the next barrier
      lds.from[at] = from;
      lds.upto[at] = upto;
      lds.seq[at] = !held ? -2 : !on ? -1 : seq;
      if (by_one && held && !on && seq != alone) lds.seq[at] = -2;
    }
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) w.dk[i] = w.dv[i] = Acc(0.f);
  w.up = kLargest;
  const Seq base = {q0, 0, 0, 0, 0};
  // From the last rows to the first: blocks that run side by side read the same
  // rows at the same time.
  int begin = block_from / kTile * kTile;
  int end = block_from < rows ? (rows - 1) / kTile * kTile : -1;
  if (kPrefix && p.parts > 1) {  // this block's share of the row tiles
    const int share = (max(end - begin + kTile, 0) / kTile + p.parts - 1) / p.parts;
    end -= part_of_rows * share * kTile;
    begin = max(begin, end - (share - 1) * kTile);
  }
  RowTile t = row_tile(a, max(end, 0));
  auto step = [&](int r0, const T* q_tile, const T* o_tile, const Stats& stats) {
    const int r = r0 + part;
    if (r + 31 < any_from || r > any_upto) return;
    w.add(q_tile, o_tile, stats, rest, wave_row, part,
          [&] {
            int at = int(threadIdx.x) % 32 + wave_row;
            asm volatile("" : "+v"(at));  // formed where it is used, not held in a register
            if (kPrefix) return RowSpan{(first + at < in_use ? 0 : rows) - r0, rows - 1 - r0};
            return RowSpan{lds.from[at] - r0, lds.upto[at] - r0};
          },
          r >= all_from && r + 31 <= all_upto, c, places);
  };
  if (end >= begin) tiles_of.fetch(a, base, kv, rows, t, lds.q_even, lds.o_even, lds.s_even);
  for (int r0 = end; r0 >= begin; r0 -= 2 * kTile) {
    tiles_barrier();  // the tile is there, and nobody reads the other buffer any more
    retreat(a, t);
    if (t.r0 >= begin) tiles_of.fetch(a, base, kv, rows, t, lds.q_odd, lds.o_odd, lds.s_odd);
    step(r0, lds.q_even, lds.o_even, *lds.s_even);
    if (r0 - kTile < begin) break;
    tiles_barrier();
    retreat(a, t);
    if (t.r0 >= begin) tiles_of.fetch(a, base, kv, rows, t, lds.q_even, lds.o_even, lds.s_even);
    step(r0 - kTile, lds.q_odd, lds.o_odd, *lds.s_odd);
  }
  // Waves 2 and 3 hand their sums to waves 0 and 1.
  static_assert(kTile * D * sizeof(T) == size_t(D) / 32 * 16 * kWave * sizeof(float), "a wave's sums");
  float* const buf_k = reinterpret_cast<float*>(wave % 2 ? lds.q_odd : lds.q_even);
  float* const buf_v = reinterpret_cast<float*>(wave % 2 ? lds.o_odd : lds.o_even);
  tiles_barrier();
  if (kShort<T>) {
    shift(w.dk, -w.up - int(kLiftGrad<T>));
    shift(w.dv, -int(kLiftGrad<T>));
  }
  if (wave >= 2) w.hand(buf_k, buf_v);
  tiles_barrier();
  if (wave < 2) w.take(buf_k, buf_v);
  int lane_again = int(threadIdx.x) % 32;
  asm volatile("" : "+v"(lane_again));
  const int row = first + wave_row + lane_again;
  const int its = !kPrefix ? lds.seq[wave_row + lane_again] : row < in_use ? 0 : row < owned ? -1 : -2;
  if (!kPrefix && !by_one && low_seq < high_seq &&
      __syncthreads_or(wave < 2 && its >= 0 && (no_number(w.dk) || no_number(w.dv))))
    return true;
  if (wave >= 2 || its == -2 || (by_one && its >= 0 && its != alone)) return by_one;
  if (its < 0) {  // also where a row that was NaN has met the tile's zeros
#pragma unroll
    for (int i = 0; i < D / 32; ++i) w.dk[i] = w.dv[i] = Acc(0.f);
  }
  if (kPrefix && p.parts > 1) {
    const int64_t at = prefix_part<D>(s, part_of_rows, kv, row);
    store_column<float, D>(p.dk + at, w.dk, D, a.scale);
    store_column<float, D>(p.dv + at, w.dv, D, 1.f);
  } else {
    store_column<T, D>(head_row<T>(kPrefix ? s.d_p_k : a.d_k, row, kv), w.dk, a.dim, a.scale);
    store_column<T, D>(head_row<T>(kPrefix ? s.d_p_v : a.d_v, row, kv), w.dv, a.dim, 1.f);
  }
  return by_one;
}

template <class T, int D, bool kFinePrefix, bool kFine>
__global__ __launch_bounds__(kThreads, (kBlocksOfUnit<D, kFinePrefix || kFine>)) void shared_keys_kernel(
    SharedArgs s, PrefixParts p, int p_tiles, int p_blocks, int tiles) {
  __shared__ __attribute__((aligned(16))) T q_even[kTile * D], o_even[kTile * D];
  __shared__ __attribute__((aligned(16))) T q_odd[kTile * D], o_odd[kTile * D];
  constexpr int kRest = KeySweep<T, D>::kHeld < D / 16 ? kKeysOfBlock * 64 : 8;
  __shared__ __attribute__((aligned(16))) T v_rest[kRest];
  __shared__ __attribute__((aligned(16))) Stats s_even, s_odd;
  __shared__ int from[kKeysOfBlock], upto[kKeysOfBlock], seq[kKeysOfBlock];
  const KeyBuffers<T> lds = {q_even, o_even, q_odd, o_odd, v_rest, &s_even, &s_odd, from, upto, seq};
  int block = int(blockIdx.x);
  if (block < p_blocks * p.parts) {
    keys_turn<T, D, true, kFinePrefix>(s, p, block, p_blocks, p_tiles, lds, -1);
    return;
  }
  block -= p_blocks * p.parts;
  for (int nth = -1;; ++nth) {
    asm volatile("" : "+s"(block));
    if (!keys_turn<T, D, false, kFine>(s, p, block, 1, tiles, lds, nth)) return;
  }
}

// Adds the parts of the prefixes' rows: four elements of a head a thread.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void add_prefix_kernel(SharedArgs s, PrefixParts p,
                                                              int64_t first) {
  typedef float Four __attribute__((ext_vector_type(4)));
  typedef T four __attribute__((ext_vector_type(4)));
  const int64_t i = (first + int64_t(blockIdx.x)) * kThreads + int(threadIdx.x);
  const int d = int(i % (D / 4)) * 4;
  const int64_t row = i / (D / 4) % s.p_rows;
  const int kv = int(i / (D / 4) / s.p_rows);
  if (kv >= s.a.q_heads / s.a.group || d >= s.a.dim || row < offset_at(s.p_offsets, 0, s.p_rows) ||
      row >= offset_at(s.p_offsets, s.n_groups, s.p_rows))
    return;
  Four x = Four(0.f), y = Four(0.f);
  for (int n = 0; n < p.parts; ++n) {
    const int64_t at = prefix_part<D>(s, n, kv, row) + d;
    x += *reinterpret_cast<const Four*>(p.dk + at);
    y += *reinterpret_cast<const Four*>(p.dv + at);
  }
  four u, v;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    u[e] = T(x[e]);
    v[e] = T(y[e]);
  }
  *reinterpret_cast<four*>(head_row<T>(s.d_p_k, row, kv) + d) = u;
  *reinterpret_cast<four*>(head_row<T>(s.d_p_v, row, kv) + d) = v;
}

// --- launches -----------------------------------------------------------------------

struct Plan {
  bool fine_rows, fine_prefix, fine_own;  // second products (kFine): for dQ; for dK and dV
  int row_parts, prefix_parts;
  size_t stats, row_values, prefix_values;  // bytes; values of dQ, and of dK or dV
};

Plan plan_of(const sched_shared_desc& x) {
  const sched_attention_desc& d = x.own;
  Plan p = {false, false, false, 1, 1, 0, 0, 0};
  if (x.n_groups == 0) return p;
  const size_t width = d.head_dim > 64 ? 128 : 64;
  const int64_t rows = d.q_rows * (d.q_heads / d.kv_heads);
  // Also for dQ where a rounded delta is much of what is left of a difference: of heads
  // of up to 48 elements (16: 1.15 times as far off as one rounding, 1.52 without; 32: 1.47
  // without; 32 answers of 20 to 100 tokens to each of 4 prompts of 300, 16 heads of 48: 51
  // us, 43 without), and where rows see few keys (13 times 64 answers of 14 tokens, 71 + 14 keys:
  // 1.06, 1.49 without, in 22 us, 20.4 without); for prefixes of a tile, and own keys
  // whose sums have few terms, parts of a call that count little, whose errors are
  // those of few numbers.  All of it takes the answers' 60 us to 68: 2^22 pairs are not
  // a small call's.
  const bool small = is_small(x);
  p.fine_rows = small || d.head_dim <= 48 || mean_keys(x) <= 128;
  p.fine_prefix = small || x.prefix_rows / x.n_groups <= kKeysOfBlock;
  p.fine_own = small || rows <= 16 * int64_t(d.n_seqs);
  p.stats = (size_t(d.q_rows) * size_t(d.q_heads) * 8 + 255) & ~size_t(255);
  // As many parts as fill the 512 places that the card has for a kernel's blocks,
  // none with less than 12 tiles of keys or 8 of rows of a mean group (13 times 64
  // answers of 14 tokens to prompts of 71: 61 us with three parts of the prefixes' rows,
  // 71 with one).  Where blocks fill the card parts only add their sums' bytes (8 prompts
  // of 1,650, 4 key heads: 934 us with one part, 972 with two).
  if (rows > 0) {
    const int64_t blocks = tile_count(rows, x.n_groups, kRowsOfBlock) * d.kv_heads;
    p.row_parts = int(std::max<int64_t>(
        1, std::min(512 / blocks, x.prefix_rows / x.n_groups / (12 * kTile))));
    if (p.row_parts > 1)
      p.row_values = size_t(p.row_parts) * size_t(d.q_rows) * size_t(d.q_heads) * width;
  }
  if (x.prefix_rows > 0) {
    const int64_t blocks = tile_count(x.prefix_rows, x.n_groups, kKeysOfBlock) * d.kv_heads;
    p.prefix_parts =
        int(std::max<int64_t>(1, std::min(512 / blocks, rows / x.n_groups / (8 * kTile))));
    if (p.prefix_parts > 1)
      p.prefix_values = size_t(p.prefix_parts) * size_t(x.prefix_rows) * size_t(d.kv_heads) * width;
  }
  return p;
}

template <class T, int D>
hipError_t shared_grad(const SharedArgs& s, const Plan& n, float* parts, hipStream_t stream) {
  const int kv_heads = s.a.q_heads / s.a.group;
  hipError_t e = hipSuccess;
  if (s.a.q_rows > 0 && s.a.n_seqs > 0) {  // first: it leaves the rows' statistics
    const RowParts r = {parts, n.row_parts};
    const int64_t tiles = tile_count(int64_t(s.a.q_rows) * s.a.group, s.n_groups, kRowsOfBlock);
    const dim3 grid(unsigned(work_blocks(tiles, kv_heads)), unsigned(r.parts));
    const auto kernel = n.fine_rows ? shared_queries_kernel<T, D, true> : shared_queries_kernel<T, D, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, s, r, int(tiles));
    e = hipGetLastError();
    const int64_t adds = (int64_t(s.a.q_rows) * s.a.q_heads * (D / 4) + kThreads - 1) / kThreads;
    for (int64_t b = 0; r.parts > 1 && b < adds && e == hipSuccess; b += kMostBlocks) {
      hipLaunchKernelGGL((add_shared_rows_kernel<T, D>), dim3(unsigned(std::min(adds - b, kMostBlocks))),
                         dim3(kThreads), 0, stream, s, r, b);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
  }
  const PrefixParts p = {parts, parts + n.prefix_values, n.prefix_parts};
  const int64_t p_tiles = s.p_rows > 0 ? tile_count(s.p_rows, s.n_groups, kKeysOfBlock) : 0;
  const int64_t o_tiles = s.a.n_seqs > 0 ? (int64_t(s.a.k_rows) + kKeysOfBlock - 1) / kKeysOfBlock : 0;
  const int64_t p_blocks = work_blocks(p_tiles, kv_heads), o_blocks = work_blocks(o_tiles, kv_heads);
  if (p_blocks + o_blocks == 0) return hipSuccess;
  const auto kernel = n.fine_prefix ? n.fine_own ? shared_keys_kernel<T, D, true, true>
                                                 : shared_keys_kernel<T, D, true, false>
                      : n.fine_own  ? shared_keys_kernel<T, D, false, true>
                                    : shared_keys_kernel<T, D, false, false>;
  hipLaunchKernelGGL(kernel, dim3(unsigned(p_blocks * p.parts + o_blocks)), dim3(kThreads), 0, stream,
                     s, p, int(p_tiles), int(p_blocks), int(o_tiles));
  e = hipGetLastError();
  const int64_t adds = (int64_t(s.p_rows) * kv_heads * (D / 4) + kThreads - 1) / kThreads;
  for (int64_t b = 0; p.parts > 1 && b < adds && e == hipSuccess; b += kMostBlocks) {
    hipLaunchKernelGGL((add_prefix_kernel<T, D>), dim3(unsigned(std::min(adds - b, kMostBlocks))),
                       dim3(kThreads), 0, stream, s, p, b);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

size_t shared_grad_bytes(const sched_shared_desc& x) {
  const Plan p = plan_of(x);
  // The parts of dQ have been added when those of dK and dV are written.
  return p.stats + std::max(p.row_values, 2 * p.prefix_values) * sizeof(float);
}

hipError_t launch_shared_grad(const sched_shared_desc& x, const sched_shared_grads& g, void* ws,
                              hipStream_t stream) {
  if (x.n_groups == 0) return hipSuccess;
  const Plan p = plan_of(x);
  SharedArgs s = shared_args(x);
  s.a.d_out = heads_view(g.d_out);
  s.a.d_q = heads_view(g.d_q);
  s.a.d_k = heads_view(g.d_k);
  s.a.d_v = heads_view(g.d_v);
  s.d_p_k = heads_view(g.d_prefix_k);
  s.d_p_v = heads_view(g.d_prefix_v);
  s.a.lse2 = static_cast<float*>(ws);
  s.a.delta = s.a.lse2 + size_t(x.own.q_rows) * size_t(x.own.q_heads);
  s.a.near_q = s.a.near_q && g.d_out.row_stride < (int64_t(1) << 24) &&
               g.d_out.head_stride < (int64_t(1) << 24);
  float* const parts = reinterpret_cast<float*>(static_cast<char*>(ws) + p.stats);
  const bool wide = x.own.head_dim > 64;
  if (x.own.dtype == SCHED_F16)
    return wide ? shared_grad<f16, 128>(s, p, parts, stream) : shared_grad<f16, 64>(s, p, parts, stream);
  return wide ? shared_grad<bf16, 128>(s, p, parts, stream) : shared_grad<bf16, 64>(s, p, parts, stream);
}

}  // namespace policy
