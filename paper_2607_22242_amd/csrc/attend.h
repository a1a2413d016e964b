// attend.h -- what the attention kernels share: products of 32 x 32 tiles,
// tiles in LDS, and where a block's rows lie in the packed tensors.
//
// One product of 16-bit operands takes A (32 x 16) and B (16 x 32) to C (32 x
// 32): lane l holds row (A) or column (B) l % 32 of the operands, elements
// 8 (l / 32) .. + 7 along the contraction, and of C column l % 32, rows
// 8 (i / 4) + 4 (l / 32) + i % 4 for i = 0 .. 15.
//
// Scores are computed so that a lane's column is what its statistics belong to
// and its 16 values run along the axis that the next product contracts.  That
// product's B is then the lane's own values, eight at a time, if its A lists
// the contraction in the same order: lane half h has 16 s + 4 h + {0 .. 3} and
// 16 s + 8 + 4 h + {0 .. 3} in step s.  Nothing moves between lanes.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "sched_policy.h"
#include "tensors.h"

namespace policy {

typedef float Acc __attribute__((ext_vector_type(16)));

template <class T>
struct Frag {
  typedef T type __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ Acc product(Frag<bf16>::type a, Frag<bf16>::type b, Acc c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ Acc product(Frag<f16>::type a, Frag<f16>::type b, Acc c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Probabilities and dS are rounded to the operands' 16 bits for their products:
// in 32 bits those would run at a sixteenth of the rate.  The error of a result
// against 64 bits is 1.4 times that of one rounding of it (f16 and bf16, 2,048 and
// 4,096 tokens).  f16 is normal from 2^-14 to 2^16 only, with steps of 2^-24 below:
// there both are multiplied with powers of two, which results are divided by.
// kLift: of the forward pass' powers, 2^8 at most: what is lost of 65,536 keys
// stays below 2^-16 of the largest value.  kLiftGrad: of the backward pass'
// probabilities, 1 at most.  dS takes the factor that its values ask for (fit), 3 to
// 8 % of the backward pass' time.
template <class T>
constexpr bool kShort = std::is_same<T, f16>::value;
template <class T>
constexpr float kLift = kShort<T> ? 7.f : 0.f;
template <class T>
constexpr float kLiftGrad = kShort<T> ? 14.f : 0.f;

struct HeadsView {
  char* data;
  int64_t row, head;  // strides in elements
};

struct AttendArgs {
  HeadsView q, k, v, out, d_out, d_q, d_k, d_v;
  float* lse;
  // q_heads x q_rows each: lse log2(e) (+inf in place of -inf), -rowsum(dO o O).
  float *lse2, *delta;
  const int32_t *q_offsets, *k_offsets, *k_lengths;
  int32_t n_seqs, q_rows, k_rows, q_heads, group, dim, causal;
  uint32_t per_group;  // ceil(2^32 / group), in 32 bits: quotients of small numbers
  // Rows of a tile lie within 2^31 bytes, and those that one thread brings are
  // at equal distances (groups of 1, 2, 4, 8 or 16): addresses are a sum for
  // the block and a distance for the lane.
  int32_t near_k, near_q;
  int32_t ranked;  // tiles go by their work (ranked_tile)
  float scale;
};

template <class T>
__device__ __forceinline__ T* head_row(const HeadsView& x, int64_t row, int head) {
  return reinterpret_cast<T*>(x.data) + row * x.row + int64_t(head) * x.head;
}

// A value that all lanes of a wave share, held once for the wave.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int wave_id() { return uniform(int(threadIdx.x) / kWave); }

// A sequence: where its queries and keys begin, and how many there are; slot
// counts the key rows that it owns, keys those in use.
struct Seq {
  int q0, k0, queries, keys, slot;
};
__device__ __forceinline__ Seq lane_sequence(const AttendArgs& a, int b) {
  Seq s;
  s.q0 = offset_at(a.q_offsets, b, a.q_rows);
  s.k0 = offset_at(a.k_offsets, b, a.k_rows);
  s.queries = max(0, offset_at(a.q_offsets, b + 1, a.q_rows) - s.q0);
  s.slot = max(0, offset_at(a.k_offsets, b + 1, a.k_rows) - s.k0);
  s.keys = a.k_lengths ? min(s.slot, max(0, a.k_lengths[b])) : s.slot;
  return s;
}
__device__ __forceinline__ Seq sequence(const AttendArgs& a, int b) {
  const Seq s = lane_sequence(a, b);
  return {uniform(s.q0), uniform(s.k0), uniform(s.queries), uniform(s.keys), uniform(s.slot)};
}

// Tiles of `tile` rows without a list of them: sequence b begins at tile
// number offset / tile + b, which leaves it as many numbers as it has tiles or
// one more.  Returns the sequence of a number and the tile within it, which may
// lie behind the sequence's last or, before the first sequence, be negative.
struct Tile {
  int seq, index;
};
__device__ __forceinline__ Tile tile_of(const int32_t* offsets, int n_seqs, int rows, int group,
                                        int tile, int number) {
  // The last sequence that begins at or before the number, 64 of them asked at once.
  const int lane = int(threadIdx.x) % kWave;
  int lo = 0, left = n_seqs, base = 0;  // of `left` sequences from lo on
  for (;;) {
    const int step = (left + kWave - 1) / kWave, at = lo + lane * step;
    int begin = 0;
    if (lane * step < left) begin = offset_at(offsets, at, rows) * group / tile + at;
    const uint64_t before = __ballot(lane * step < left && begin <= number);
    // The first one counts even where it begins behind the number.
    const int last = before ? 63 - __builtin_clzll(before) : 0;
    base = __shfl(begin, last);
    lo = uniform(lo + last * step);
    if (step == 1) break;
    left = uniform(min(step, left - last * step));
  }
  return {lo, number - uniform(base)};
}

// Tiles of up to 64 sequences from the one with most work to the one with least,
// so that no long one begins when the others end.  Along a causal sequence the
// work falls by one level a tile from the tile that sees (or, of keys, is seen
// by) most; otherwise all tiles of a sequence have the same.  Returns the tile
// of a rank, counted within its sequence from the one with most work; index -1
// behind the last.  Every lane brings a sequence: its tiles and its top level.
__device__ __forceinline__ int wave_total(int x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return uniform(x);
}
__device__ __forceinline__ Tile ranked_tile(int tiles, int top, bool falls, int rank) {
  // Tiles of this lane's sequence at a level or above.
  auto above = [&](int level) {
    return top < level ? 0 : falls ? min(tiles, top - level + 1) : tiles;
  };
  int hi = tiles > 0 ? top : -(1 << 30);
  int lo = tiles > 0 ? (falls ? top - tiles + 1 : top) : 1 << 30;
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    hi = max(hi, __shfl_xor(hi, d));
    lo = min(lo, __shfl_xor(lo, d));
  }
  lo = uniform(lo);
  hi = uniform(hi);
  if (lo > hi || wave_total(above(lo)) <= rank) return {0, -1};
  while (lo < hi) {  // the highest level with more than `rank` tiles at it or above
    const int mid = lo + (hi - lo + 1) / 2;
    if (wave_total(above(mid)) > rank) lo = mid;
    else hi = mid - 1;
  }
  const int here = above(lo) - above(lo + 1), behind = rank - wave_total(above(lo + 1));
  int before = here;  // of this level in earlier sequences, with this one
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int up = __shfl_up(before, d);
    if (int(threadIdx.x) % kWave >= d) before += up;
  }
  before -= here;
  const int seq = __ffsll((unsigned long long)__ballot(here > 0 && behind < before + here)) - 1;
  const int index = falls ? top - lo : behind - before;
  return {seq, uniform(__shfl(index, seq))};
}

inline int64_t tile_count(int64_t rows, int n_seqs, int tile) { return rows / tile + n_seqs; }

// Query rows of a block: the heads that share a key head are rows of their own,
// row r being query r / group and head r % group of the key head's.
struct QueryRow {
  int query, head;
};
// The tile of query rows of a rank, from most keys to least where the call ranks
// its tiles, else from the packed tensor's end (of one sequence the same).
__device__ __forceinline__ Tile query_tile(const AttendArgs& a, int tile, int rank, int count) {
  if (!a.ranked)
    return tile_of(a.q_offsets, a.n_seqs, a.q_rows, a.group, tile, count - 1 - rank);
  const int b = int(threadIdx.x) % kWave;
  int tiles = 0, top = 0;
  if (b < a.n_seqs) {
    const Seq s = lane_sequence(a, b);
    tiles = (s.queries * a.group + tile - 1) / tile;
    top = int(min(int64_t(s.keys) * a.group / tile, int64_t(1) << 29));
  }
  const Tile t = ranked_tile(tiles, top, a.causal, rank);
  return {t.seq, t.index < 0 ? -1 : a.causal ? __shfl(tiles, t.seq) - 1 - t.index : t.index};
}
// The same of keys, from most query rows to least.
__device__ __forceinline__ Tile key_tile(const AttendArgs& a, int tile, int rank) {
  if (!a.ranked) return tile_of(a.k_offsets, a.n_seqs, a.k_rows, 1, tile, rank);
  const int b = int(threadIdx.x) % kWave;
  int tiles = 0, top = 0;
  if (b < a.n_seqs) {
    const Seq s = lane_sequence(a, b);
    tiles = (s.slot + tile - 1) / tile;
    top = a.causal ? s.keys / tile : s.queries;
  }
  return ranked_tile(tiles, top, a.causal, rank);
}
__device__ __forceinline__ QueryRow query_row(const AttendArgs& a, int kv_head, int r) {
  return {r / a.group, kv_head * a.group + r % a.group};
}

// Which tile and key head a block takes.  Blocks go to the card's 8 dies in
// turn, each with a cache of its own: a die works on one key head at a time (or
// shares it with few others), whose keys and values its cache then holds.
struct Work {
  int tile, kv;
};
__device__ __forceinline__ Work work_of(int block, int tiles, int kv_heads) {
  const int die = block % 8, i = block / 8;
  if (kv_heads % 8 == 0) return {i % tiles, die + 8 * (i / tiles)};
  if (8 % kv_heads == 0) return {i * (8 / kv_heads) + die / kv_heads, die % kv_heads};
  return {block / kv_heads, block % kv_heads};
}
inline int64_t work_blocks(int64_t tiles, int kv_heads) {
  if (kv_heads % 8 != 0 && 8 % kv_heads == 0) {
    const int share = 8 / kv_heads;
    return (tiles + share - 1) / share * 8;
  }
  return tiles * kv_heads;
}

// 16 bytes of a row, zeros behind the head's last element.
template <class T>
__device__ __forceinline__ typename Frag<T>::type piece(const T* row, int d, int dim, bool on) {
  typename Frag<T>::type v = T(0);
  if (on && d < dim) v = *reinterpret_cast<const typename Frag<T>::type*>(row + d);
  return v;
}

// A tile in LDS: rows of D elements in pieces of 16 bytes, the pieces of a row
// permuted so that neither way of reading meets a bank twice: 16 rows at one
// piece (along), and 4 rows at 4 pieces next to each other (across).
template <int D>
__device__ __forceinline__ int turn_of(int row) {  // what a row's pieces are permuted by
  return D == 128 ? row % 4 * 4 + row / 4 % 4 : row / 2 % 2 * 4 + row / 4 % 4;
}

// Where a lane reads in a tile, in bytes: pieces differ by an exclusive or.
// fresh() keeps the compiler from holding every one of them in a register.
template <int D>
struct Places {
  int along, across;

  __device__ __forceinline__ Places() {
    const int l = int(threadIdx.x) % kWave, h = l / 32, row = l % 16 / 4;
    along = l % 32 * D * 2 + (h ^ turn_of<D>(l % 32)) * 16;
    const int col = l % 32 / 16 * 2 + l % 4 / 2;
    across = (4 * h + row) * D * 2 + (col ^ turn_of<D>(4 * h + row)) * 16 + l % 2 * 8;
  }
  __device__ __forceinline__ Places fresh() const {
    Places p = *this;
    asm volatile("" : "+v"(p.along), "+v"(p.across));
    return p;
  }
};

template <class T, int D>
struct Rows {
  const T* at;
  Places<D> places;

  // A or B along the rows: lane l has row l % 32 of the 32 from `row`, elements
  // 16 k + 8 (l / 32) .. + 7.
  __device__ __forceinline__ typename Frag<T>::type along(int row, int k) const {
    return *reinterpret_cast<const typename Frag<T>::type*>(
        reinterpret_cast<const char*>(at) + row * D * 2 + (places.along ^ (k << 5)));
  }
  // A across the rows: lane l has column 32 c + l % 32 of the rows row + 4 h +
  // {0..3} and row + 8 + 4 h + {0..3}, h = l / 32; row is a multiple of 16.
  // Sixteen lanes read four rows of sixteen columns, four elements each, and
  // get a column of four.
  __device__ __forceinline__ typename Frag<T>::type across(int row, int c) const {
    const int at0 = places.across ^ (c << 6);
    const auto lo = turned(row * D * 2 + at0), hi = turned((row + 8) * D * 2 + (at0 ^ 32));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }

 private:
  typedef T Four __attribute__((ext_vector_type(4)));
  __device__ __forceinline__ Four turned(int byte) const {
    typedef short Raw __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) Raw Lds;
    return __builtin_bit_cast(Four, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (Lds*)(reinterpret_cast<const char*>(at) + byte)));
  }
};

// A tile's 16 bytes per thread from memory to LDS without a register between:
// a wave fills 1024 bytes in a row, so the permutation is in what a lane reads.
// Nothing waits for it until the next tiles_barrier().
__device__ __forceinline__ void to_lds(const char* from, uint32_t lane_bytes, void* wave_at) {
  typedef __attribute__((address_space(1))) const void Global;
  typedef __attribute__((address_space(3))) void Lds;
  __builtin_amdgcn_global_load_lds((Global*)(from + lane_bytes), (Lds*)wave_at, 16, 0, 0);
}

// A barrier behind which tiles that were on their way are there: each wave waits
// for what it has brought itself (the compiler's barrier waits for LDS, and not
// in every place for loads into it), and then for the others.
__device__ __forceinline__ void tiles_barrier() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// Threads of a block over a tile of kRows rows: round p of a thread brings one
// piece of row p * kStep + row, always the same piece of its row.
template <class T, int D, int kRows, int kThreads>
struct Fill {
  static constexpr int kStep = kThreads / (D / 8), kRounds = kRows / kStep;
  int row, d;  // of this thread

  __device__ __forceinline__ Fill(int dim) {
    int t = int(threadIdx.x);
    asm volatile("" : "+v"(t));  // formed where it is used, not held in registers
    row = t / (D / 8);
    const int c = t % (D / 8) ^ turn_of<D>(row);
    d = min(8 * c, dim - 8);  // behind the head's last element: what is there twice is not used
  }
  // The lane's bytes from row 0 of the tile, rows of a head `row_stride` apart.
  __device__ __forceinline__ uint32_t bytes(int64_t row_stride) const {
    return uint32_t(row * row_stride + d) * 2;
  }
  __device__ __forceinline__ static T* at(T* tile, int p) {
    return tile + (p * kThreads + wave_id() * kWave) * 8;
  }
};

// Tiles of kRows keys and values of one sequence and key head.
template <class T, int D, int kRows, int kThreads>
struct KeyTiles {
  typedef Fill<T, D, kRows, kThreads> F;
  const char *k, *v;     // the sequence's first row
  uint32_t k_lane, v_lane;
  int64_t k_row, v_row;  // bytes
  int keys, near;

  __device__ __forceinline__ KeyTiles(const AttendArgs& a, const Seq& s, int kv)
      : k(reinterpret_cast<const char*>(head_row<T>(a.k, s.k0, kv))),
        v(reinterpret_cast<const char*>(head_row<T>(a.v, s.k0, kv))),
        k_row(a.k.row * 2), v_row(a.v.row * 2), keys(s.keys), near(a.near_k) {
    const F fill(a.dim);
    k_lane = fill.bytes(a.k.row);
    v_lane = fill.bytes(a.v.row);
  }
  // Rows j0 .. to LDS; those behind the last key repeat it, their probabilities
  // are zero.
  __device__ __forceinline__ void fetch(int j0, T* k_tile, T* v_tile, int dim) const {
    if (near && j0 + kRows <= keys) {
#pragma unroll
      for (int p = 0; p < F::kRounds; ++p) {
        to_lds(k + (j0 + p * F::kStep) * k_row, k_lane, F::at(k_tile, p));
        to_lds(v + (j0 + p * F::kStep) * v_row, v_lane, F::at(v_tile, p));
      }
      return;
    }
    const F fill(dim);
#pragma unroll
    for (int p = 0; p < F::kRounds; ++p) {
      const int row = min(j0 + fill.row + p * F::kStep, keys - 1);
      to_lds(k + row * k_row + fill.d * 2, 0, F::at(k_tile, p));
      to_lds(v + row * v_row + fill.d * 2, 0, F::at(v_tile, p));
    }
  }
};

template <class T>
__device__ __forceinline__ typename Frag<T>::type narrow(const Acc& x, int s) {
  typename Frag<T>::type v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = T(x[8 * s + e]);
  return v;
}

// Values of f16 of one row or key (a lane's and those of the lane 32 on) that pass
// 2^15 go down to 2^10, and all that come after them with them: fit() returns the
// power of two that they were divided by.  What is infinite is left out.  The first
// values come with 2^kLargest, so that every sum meets its own size: steps are
// 2^-34 of the largest value that it has had.
constexpr int kLargest = 60;
__device__ __forceinline__ bool passes(const Acc& x) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
  return m > 32768.f;
}
__device__ __forceinline__ int fit(Acc& x) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]) < INFINITY ? fabsf(x[i]) : 0.f);
  m = fmaxf(m, __shfl_xor(m, 32));
  const int e = m > 32768.f ? __builtin_amdgcn_frexp_expf(m) - 11 : 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = __builtin_ldexpf(x[i], -e);
  return e;
}
template <int N>
__device__ __forceinline__ void shift(Acc (&x)[N], int e) {
#pragma unroll
  for (int d = 0; d < N; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[d][i] = __builtin_ldexpf(x[d][i], e);
}

// Row of C that element i of lane l holds.
__device__ __forceinline__ int c_row(int i) {
  return 8 * (i / 4) + 4 * (int(threadIdx.x) % kWave / 32) + i % 4;
}

// A lane's column of C tiles (D / 32 of them, rows being the head's elements)
// times f, to a row in memory.
template <class T, int D>
__device__ __forceinline__ void store_column(T* row, const Acc (&x)[D / 32], int dim, float f) {
  typedef T four __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int d = 32 * c + c_row(i);
      if (d < dim) {
        four v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = T(x[c][i + e] * f);
        *reinterpret_cast<four*>(row + d) = v;
      }
    }
}

}  // namespace policy
