// attend_shared.h -- attention of groups of sequences that share a prefix: what
// its forward and backward kernels have in common.
//
// A query row sees all of its group's prefix keys and, of its own sequence's
// keys, those up to its own place.  The query rows of a group's sequences lie
// one behind the other, so that a block takes rows of several sequences and
// meets every prefix key once for all of them.
#pragma once
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

// Tiles of `tile` query rows of the groups, numbered as tile_of has it.
__device__ __forceinline__ Tile group_tile(const SharedArgs& s, int tile, int number) {
  return tile_of([&](int g) { return first_query(s, g) * s.a.group / tile + g; }, s.n_groups, number);
}

// The sequence, among `n` from `first` on, that holds a lane's row: the last that
// begins at or before it.  low and high: the wave's lowest and highest row.
__device__ __forceinline__ int lane_sequence_of(const int32_t* offsets, int rows, int first, int n,
                                                int low, int high, int row) {
  const int lane = int(threadIdx.x) % kWave;
  const int at = first + tile_of([&](int i) { return offset_at(offsets, first + i, rows); }, n, low).seq;
  const int left = first + n - at;  // sequences from it on
  const int begin = lane < left ? offset_at(offsets, at + lane, rows) : 0x7fffffff;
  if (left > kWave && __shfl(begin, kWave - 1) <= high)  // many empty ones
    return at + sequence_of(offsets + at, left, row);
  int seq = 0;
#pragma unroll
  for (int d = kWave / 2; d; d >>= 1)
    if (__shfl(begin, seq + d) <= row) seq += d;
  return at + seq;
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

// The tiles of 64 keys that a block's rows meet: those of the prefix from `begin`
// to `end`, then the own keys of the sequences seq .. last_seq, of the last one
// those up to last_key.  Without k_lengths the sequences' keys lie one behind the
// other and count as one; else a sequence is walked after the other.
struct Step {
  int own, key0, last;  // is it of the own keys; the tile's first key, the last that counts
  int there;
};
template <class T, int D>
struct Walk {
  typedef KeyTiles<T, D, 64, 256> Tiles;
  const SharedArgs& s;
  const Tiles prefix;
  Tiles own;
  int kv, end, seq, last_seq, last_key, base, place;  // place: of the next tile, from base

  __device__ __forceinline__ Walk(const SharedArgs& s_, const Group& g, int kv_, int begin, int end_,
                                  int first_seq, int last_seq_, int last_key_)
      : s(s_), prefix(s_.p_k, s_.p_v, g.p0, g.keys, s_.near_p, s_.a.dim, kv_),
        own(s_.a.k, s_.a.v, 0, 0, s_.a.near_k, s_.a.dim, kv_), kv(kv_), end(end_),
        seq(first_seq - 1), last_seq(last_seq_), last_key(last_key_), base(0), place(begin) {}

  // Own keys of the next sequence that has any.
  __device__ __forceinline__ bool enter() {
    while (++seq <= last_seq) {
      const Seq q = sequence(s.a, seq);
      int behind = q.k0 + q.keys;
      if (s.a.k_lengths) {
        if (seq == last_seq) behind = min(behind, last_key + 1);
        if (q.queries == 0) continue;
      } else {
        behind = last_key + 1;
        seq = last_seq;
      }
      if (behind <= q.k0) continue;
      base = q.k0;
      own.keys = behind - base;
      own.k = reinterpret_cast<const char*>(head_row<T>(s.a.k, base, kv));
      own.v = reinterpret_cast<const char*>(head_row<T>(s.a.v, base, kv));
      return true;
    }
    return false;
  }
  // The next tile, on its way to LDS.
  __device__ __forceinline__ Step next(T* k_tile, T* v_tile) {
    if (end > 0) {
      if (place < end) {
        const int j0 = place;
        prefix.fetch(j0, k_tile, v_tile, s.a.dim);
        place += 64;
        return {0, j0, prefix.keys - 1, 1};
      }
      end = 0;
      place = 0;
      own.keys = 0;
    }
    if (place >= own.keys) {
      place = 0;
      if (!enter()) return {0, 0, 0, 0};
    }
    const int j0 = place;
    own.fetch(j0, k_tile, v_tile, s.a.dim);
    place += 64;
    return {1, base + j0, base + own.keys - 1, 1};
  }
};

// Keys from one to another.
struct Within {
  int lo, hi;
  __device__ __forceinline__ bool operator()(int j) const { return j >= lo && j <= hi; }
};

// What a wave's rows see of the own keys.
struct Seen {
  Span mine;
  int all_lo, all_hi, any_lo, any_hi;

  __device__ __forceinline__ explicit Seen(const Span& x)
      : mine(x), all_lo(wave_most(x.lo)), all_hi(wave_least(x.hi)), any_lo(wave_least(x.lo)),
        any_hi(wave_most(x.hi)) {}
  __device__ __forceinline__ bool any(const Step& t) const {
    return !t.own || (t.key0 <= any_hi && t.key0 + 63 >= any_lo);
  }
  __device__ __forceinline__ bool all(const Step& t) const {
    return t.key0 + 63 <= t.last && (!t.own || (t.key0 >= all_lo && t.key0 + 63 <= all_hi));
  }
  __device__ __forceinline__ Within keys(const Step& t) const {
    return {t.own ? mine.lo : 0, t.own ? min(mine.hi, t.last) : t.last};
  }
};

// Where a block's 128 query rows lie, and what this lane's row sees; rows behind
// the last are copies of it that nobody writes.
template <int kRows>
struct RowsOf {
  Group g;
  int first, rows, row;  // first of the tile, rows of the group, this lane's row
  bool there, on;
  QueryRow me;           // query within the group
  int query, seq, first_seq, last_seq, last_key;
  Span mine;

  __device__ __forceinline__ RowsOf(const SharedArgs& s, int kv, int number, int lane_row) {
    const Tile tile = group_tile(s, kRows, number);
    g = group_at(s, tile.seq);
    first = tile.index * kRows;
    rows = g.queries * s.a.group;
    there = tile.index >= 0 && first < rows;
    if (!there) return;
    on = first + lane_row < rows;
    row = min(first + lane_row, rows - 1);
    me = query_row(s.a, kv, row);
    query = g.q0 + me.query;
    const int low = g.q0 + first / s.a.group;
    const int high = g.q0 + (min(first + kRows, rows) - 1) / s.a.group;
    seq = lane_sequence_of(s.a.q_offsets, s.a.q_rows, g.seq, g.seqs, low, high, query);
    mine = own_keys(s.a, lane_sequence(s.a, seq), query);
    // Of the tile's first and last row, which another wave may hold.
    first_seq = uniform(lane_sequence_of(s.a.q_offsets, s.a.q_rows, g.seq, g.seqs, low, low, low));
    last_seq = uniform(lane_sequence_of(s.a.q_offsets, s.a.q_rows, g.seq, g.seqs, high, high, high));
    const Seq q = sequence(s.a, last_seq);
    const Span last = own_keys(s.a, q, high);
    // Sequences before the last one end within the tile: all their keys count.
    last_key = last_seq > first_seq ? max(last.hi, q.k0 - 1) : last.hi;
  }
};

inline HeadsView heads_view(const sched_heads& h) {
  return {static_cast<char*>(h.data), h.row_stride, h.head_stride};
}

AttendArgs attend_args(const sched_attention_desc& d);
SharedArgs shared_args(const sched_shared_desc& d);

}  // namespace policy
