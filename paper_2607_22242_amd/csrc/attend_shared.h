// attend_shared.h -- attention of groups of sequences that share a prefix: what
// its forward and backward kernels have in common.
//
// A query row sees all of its group's prefix keys and, of its own sequence's
// keys, those up to its own place.  The query rows of a group's sequences lie
// one behind the other, so that a block takes rows of several sequences and
// meets every prefix key once for all of them.
#pragma once
#include <algorithm>
#include <type_traits>

#include "attend.h"

namespace policy {

struct SharedArgs {
  AttendArgs a;  // the sequences and their own keys
  HeadsView p_k, p_v, d_p_k, d_p_v;
  const int32_t *p_offsets, *p_lengths, *groups;
  int32_t n_groups, p_rows, near_p;
};

// A group: its sequences, their query rows, and the prefix (slot: the key rows
// that it owns, keys: those in use).
struct Group {
  int seq, seqs, q0, queries, p0, keys, slot;
};
__device__ __forceinline__ int first_sequence(const SharedArgs& s, int g) {
  return offset_at(s.groups, g, s.a.n_seqs);
}
__device__ __forceinline__ int first_query(const SharedArgs& s, int g) {
  return offset_at(s.a.q_offsets, first_sequence(s, g), s.a.q_rows);
}
__device__ __forceinline__ Group group_at(const SharedArgs& s, int g) {
  Group x;
  x.seq = uniform(first_sequence(s, g));
  x.seqs = max(0, uniform(first_sequence(s, g + 1)) - x.seq);
  x.p0 = uniform(offset_at(s.p_offsets, g, s.p_rows));
  x.slot = max(0, uniform(offset_at(s.p_offsets, g + 1, s.p_rows)) - x.p0);
  x.keys = s.p_lengths ? min(x.slot, max(0, uniform(s.p_lengths[g]))) : x.slot;
  x.q0 = uniform(offset_at(s.a.q_offsets, x.seq, s.a.q_rows));
  x.queries = max(0, uniform(offset_at(s.a.q_offsets, x.seq + x.seqs, s.a.q_rows)) - x.q0);
  return x;
}

// The tile of a number, and its group: tiles of `tile` query rows of the groups, or
// (kPrefix) of their prefix rows, numbered as tile_of has it.  Up to 63 groups are
// asked for all that there is to know of them at once: loads that wait for one another
// are most of a small call's time.
struct GroupTile {
  int index;
  Group g;
};
template <bool kPrefix>
__device__ __forceinline__ GroupTile group_tile(const SharedArgs& s, int tile, int number) {
  if (s.n_groups >= kWave) {
    const Tile t =
        kPrefix ? tile_of(s.p_offsets, s.n_groups, s.p_rows, 1, tile, number)
                : tile_of([&](int g) { return first_query(s, g) * s.a.group / tile + g; }, s.n_groups,
                          number);
    return {t.index, group_at(s, t.seq)};
  }
  const int lane = int(threadIdx.x) % kWave, at = min(lane, s.n_groups);
  const int length = s.p_lengths && lane < s.n_groups ? s.p_lengths[lane] : 0x7fffffff;
  const int p0 = offset_at(s.p_offsets, at, s.p_rows), seq = first_sequence(s, at);
  const int q0 = offset_at(s.a.q_offsets, seq, s.a.q_rows);
  const int begin = (kPrefix ? p0 / tile : q0 * s.a.group / tile) + at;
  const uint64_t before = __ballot(lane < s.n_groups && begin <= number);
  const int g = before ? 63 - __builtin_clzll(before) : 0;
  auto of = [](int x, int from) { return __builtin_amdgcn_readlane(x, from); };
  Group x;
  x.seq = of(seq, g);
  x.seqs = max(0, of(seq, g + 1) - x.seq);
  x.p0 = of(p0, g);
  x.slot = max(0, of(p0, g + 1) - x.p0);
  x.keys = min(x.slot, max(0, of(length, g)));
  x.q0 = of(q0, g);
  x.queries = max(0, of(q0, g + 1) - x.q0);
  return {number - of(begin, g), x};
}

// The sequences, among `n` from `first` on, that hold a block's lowest and highest
// row and this lane's: the last that begins at or before it.
struct Held {
  int low, high, mine;
};
__device__ __forceinline__ Held sequences_of(const int32_t* offsets, int rows, int first, int n,
                                             int low, int high, int row) {
  const int lane = int(threadIdx.x) % kWave;
  int at = first, left = n;  // sequences from `at` on
  if (n > kWave) {
    at += tile_of([&](int i) { return offset_at(offsets, first + i, rows); }, n, low).seq;
    left = first + n - at;
  }
  const int begin = lane < left ? offset_at(offsets, at + lane, rows) : 0x7fffffff;
  const uint64_t behind = __ballot(begin > high);
  if (left > kWave && !behind) {  // many empty ones
    return {at, at + uniform(sequence_of(offsets + at, left, high)),
            at + sequence_of(offsets + at, left, row)};
  }
  const uint64_t before = __ballot(begin <= low);
  int mine = 0;
#pragma unroll
  for (int d = kWave / 2; d; d >>= 1)
    if (__shfl(begin, mine + d) <= row) mine += d;
  return {at + (before ? 63 - __builtin_clzll(before) : 0),
          at + (behind ? max(__builtin_ctzll(behind) - 1, 0) : kWave - 1), at + mine};
}

// Own keys that a query row sees, counted in all key rows.
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span own_keys(const AttendArgs& a, const Seq& q, int query) {
  const int last = a.causal ? min(q.keys - 1, query - q.q0 + q.keys - q.queries) : q.keys - 1;
  return {q.k0, q.k0 + last};
}

__device__ __forceinline__ int wave_least(int x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = min(x, __shfl_xor(x, d));
  return uniform(x);
}
__device__ __forceinline__ int wave_most(int x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = max(x, __shfl_xor(x, d));
  return uniform(x);
}

// The tiles of 64 own keys that a block's rows meet: of the sequences seq ..
// last_seq, from first_key on and of the last one up to last_key.  Without k_lengths
// the sequences' keys lie one behind the other and count as one, and nothing more has
// to be known of them; else a sequence is walked after the other.
struct Step {
  int key0, last;  // the tile's first key, and the last that counts, of all key rows
  int there;
};
template <class T, int D>
struct Walk {
  const SharedArgs& s;
  KeyTiles<T, D, 64, 256> own;
  int kv, seq, last_seq, last_key, base, place;  // place: of the next tile, from base

  __device__ __forceinline__ Walk(const SharedArgs& s_, int kv_, int first_seq, int last_seq_,
                                  int first_key, int last_key_)
      : s(s_), own(s_.a.k, s_.a.v, 0, 0, s_.a.near_k, s_.a.dim, kv_), kv(kv_), seq(first_seq - 1),
        last_seq(last_seq_), last_key(last_key_), base(0), place(0) {
    if (s.a.k_lengths) return;
    seq = last_seq;
    go_to(first_key, last_key + 1);
  }

  __device__ __forceinline__ void go_to(int from, int behind) {
    base = from;
    place = 0;
    own.keys = behind - base;
    own.k = reinterpret_cast<const char*>(head_row<T>(s.a.k, base, kv));
    own.v = reinterpret_cast<const char*>(head_row<T>(s.a.v, base, kv));
  }
  // Own keys of the next sequence that has any.
  __device__ __forceinline__ bool enter() {
    while (++seq <= last_seq) {
      const Seq q = sequence(s.a, seq);
      int behind = q.k0 + q.keys;
      if (seq == last_seq) behind = min(behind, last_key + 1);
      if (q.queries == 0 || behind <= q.k0) continue;
      go_to(q.k0, behind);
      return true;
    }
    return false;
  }
  // The next tile, on its way to LDS.
  __device__ __forceinline__ Step next(T* k_tile, T* v_tile) {
    if (place >= own.keys && !enter()) return {0, 0, 0};
    const int j0 = place;
    own.fetch(j0, k_tile, v_tile, s.a.dim);
    place += 64;
    return {base + j0, base + own.keys - 1, 1};
  }
};

// The tiles of a block: arrays of their own in LDS.  (As members of one, what is read
// of a tile would wait for the next one's loads, too: the compiler tells arrays apart,
// not their parts.)
template <class T>
struct Buffers {
  T *k_even, *v_even, *k_odd, *v_odd;
};

// A block's rows over the prefix keys begin <= j < end (their first tile is under way
// in the even arrays) and then the own keys of the walk (with_own), each tile under way
// while the one before it is worked on.
// on_prefix(j0, k, v), on_own(step, k, v): what is done with a tile.
template <class T, int D, class OnPrefix, class OnOwn>
__device__ __forceinline__ void over_keys(const KeyTiles<T, D, 64, 256>& prefix, int dim, int begin,
                                          int end, Walk<T, D>& walk, bool with_own,
                                          const Buffers<T>& lds, const OnPrefix& on_prefix,
                                          const OnOwn& on_own) {
  Step step = {0, 0, 0};
  bool odd = false;  // where the first own tile is
  auto first_own = [&](T* k, T* v) {
    if (with_own) step = walk.next(k, v);
  };
  if (begin < end) {
    for (int j0 = begin;; j0 += 128) {
      tiles_barrier();  // the tile is there, and nobody reads the other buffer any more
      const bool more = j0 + 64 < end;
      if (more) prefix.fetch(j0 + 64, lds.k_odd, lds.v_odd, dim);
      else first_own(lds.k_odd, lds.v_odd);
      on_prefix(j0, lds.k_even, lds.v_even);
      if (!more) {
        odd = true;
        break;
      }
      tiles_barrier();
      const bool again = j0 + 128 < end;
      if (again) prefix.fetch(j0 + 128, lds.k_even, lds.v_even, dim);
      else first_own(lds.k_even, lds.v_even);
      on_prefix(j0 + 64, lds.k_odd, lds.v_odd);
      if (!again) break;
    }
  } else {
    first_own(lds.k_even, lds.v_even);
  }
  while (step.there) {
    if (!odd) {
      tiles_barrier();
      const Step next = walk.next(lds.k_odd, lds.v_odd);
      on_own(step, lds.k_even, lds.v_even);
      if (!next.there) break;
      step = next;
    }
    odd = false;
    tiles_barrier();
    const Step next = walk.next(lds.k_even, lds.v_even);
    on_own(step, lds.k_odd, lds.v_odd);
    step = next;
  }
}

// Keys from one to another.
struct Within {
  int lo, hi;
  __device__ __forceinline__ bool operator()(int j) const { return j >= lo && j <= hi; }
};

// What a wave's rows see of the own keys, and of a tile of them.
struct Seen {
  Span mine;
  int all_lo, all_hi, any_lo, any_hi;

  __device__ __forceinline__ explicit Seen(const Span& x)
      : mine(x), all_lo(wave_most(x.lo)), all_hi(wave_least(x.hi)), any_lo(wave_least(x.lo)),
        any_hi(wave_most(x.hi)) {}
  // The most own keys that a row of the wave sees.
  __device__ __forceinline__ int most() const { return wave_most(max(0, mine.hi - mine.lo + 1)); }
  __device__ __forceinline__ bool any(const Step& t) const {
    return t.key0 <= any_hi && t.key0 + 63 >= any_lo;
  }
  __device__ __forceinline__ bool all(const Step& t) const {
    return t.key0 + 63 <= min(t.last, all_hi) && t.key0 >= all_lo;
  }
  __device__ __forceinline__ Within keys(const Step& t) const {
    return {mine.lo, min(mine.hi, t.last)};
  }
};

// Where a block's query rows lie, and what this lane's row sees; rows behind the
// last are copies of it that nobody writes.
template <int kRows>
struct RowsOf {
  Group g;
  int first, rows;  // first of the tile, rows of the group
  bool there, on;
  QueryRow me;      // query within the group
  int query, first_seq, last_seq, seq, first_key, last_key;  // keys of the tile's first and last row
  Span mine;

  __device__ __forceinline__ RowsOf(const SharedArgs& s, const Work& work, int tiles, int lane_row) {
    const GroupTile tile = group_tile<false>(s, kRows, tiles - 1 - work.tile);
    g = tile.g;
    first = tile.index * kRows;
    rows = g.queries * s.a.group;
    there = tile.index >= 0 && first < rows;
    on = there && first + lane_row < rows;
    me = query_row(s.a, work.kv, there ? min(first + lane_row, rows - 1) : 0);
    query = g.q0 + me.query;
  }
  // The rows' sequences (where there are rows).
  __device__ __forceinline__ void find(const SharedArgs& s) {
    const int low = g.q0 + first / s.a.group;
    const int high = g.q0 + (min(first + kRows, rows) - 1) / s.a.group;
    const Held held = sequences_of(s.a.q_offsets, s.a.q_rows, g.seq, g.seqs, low, high, query);
    first_seq = uniform(held.low);
    last_seq = uniform(held.high);
    seq = held.mine;
    const Seq q = lane_sequence(s.a, seq), tail = lane_sequence(s.a, last_seq);
    first_key = uniform(offset_at(s.a.k_offsets, first_seq, s.a.k_rows));
    mine = own_keys(s.a, q, query);
    // Sequences before the last one end within the tile: all their keys count.
    const int last = own_keys(s.a, tail, high).hi;
    last_key = uniform(last_seq > first_seq ? max(last, tail.k0 - 1) : last);
  }
  // The first and the last key that rows of the tile see of one of its sequences.
  __device__ __forceinline__ int first_key_of(const SharedArgs& s, int b) const {
    return uniform(offset_at(s.a.k_offsets, b, s.a.k_rows));
  }
  __device__ __forceinline__ int last_key_of(const SharedArgs& s, int b) const {
    if (b == last_seq) return last_key;
    const Seq q = sequence(s.a, b);
    return q.k0 + q.keys - 1;
  }
};

// A key that is masked for a row has weight zero, and zero times what is no number is
// none: a sequence that holds one reaches the others of its tile.  It shows in their
// sums, and is rare; a block that finds it takes its sequences one by one.
template <int N>
__device__ __forceinline__ bool no_number(const Acc (&x)[N]) {
  float sum = 0.f;
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += x[d][i] * 0.f;
  return sum != 0.f;  // infinities, too, give NaN here
}

inline HeadsView heads_view(const sched_heads& h) {
  return {static_cast<char*>(h.data), h.row_stride, h.head_stride};
}

// Keys that a row sees, as many as groups and sequences have on average.
inline int64_t mean_keys(const sched_shared_desc& x) {
  return x.prefix_rows / std::max(x.n_groups, 1) + x.own.k_rows / std::max(x.own.n_seqs, 1);
}
// Calls of up to 2^21 pairs of a row and a key wait for chains of loads and not for
// products: theirs take what the rounding of probabilities and dS to 16 bits has left of
// them in a second product (kFine), and results are as exact as one rounding of them, not
// 1.3 to 1.5 times as far off (64 single tokens of 8 heads: 11.4 us, 10.1 without; all
// of an update of 2^22 pairs: 68, 60).
inline bool is_small(const sched_shared_desc& x) {
  return x.own.q_rows * x.own.q_heads <= (int64_t(1) << 21) / (mean_keys(x) + 1);
}

AttendArgs attend_args(const sched_attention_desc& d);
SharedArgs shared_args(const sched_shared_desc& d);

}  // namespace policy
