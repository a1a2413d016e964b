// embed.hip -- embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: out[i] = scale * table[t_i], a copy of rows.  Gradient: row v of the
// table gets scale * the sum of d_rows[i] over the i with t_i = v.  The pairs
// (t_i, i) are sorted by token, stable, so that every row's sum runs over one
// run of the list: no atomics on values, one order, dealt to the groups of lanes
// of a wave.  A run may hold one token or all of them; whole chunks of a run are
// summed first by waves of their own and the row adds their sums.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "policy_launch.h"
#include "tensors.h"

namespace policy {
namespace {

constexpr int kBlock = 256;
constexpr int kDigit = 9;                // bits of a digit at most
constexpr int kBins = 1 << kDigit;
constexpr int kSmall = 8192;             // tokens that one block sorts in LDS
constexpr int kSmallThreads = 1024;
constexpr int kTile = 2048;              // tokens of a block otherwise
constexpr int kTileThreads = 512;
// Tiles from whose number on their counts are scanned first; below, every block
// adds up the others' by itself, a launch less but as the square of the tiles
// (131,072 tokens, 64 of them: 54 us both ways; 2^20: 140 us so, 188 without;
// 2^22: 337 and 1,148).
constexpr uint32_t kScanned = 128;
constexpr int kMostThreads = 512;       // of a block of a row's waves

__device__ __forceinline__ uint64_t below(int lane) { return (1ull << lane) - 1; }

// --- lookup ---------------------------------------------------------------

// `lanes` threads (a power of two up to 256) take a row, in 16-byte pieces.
template <class T>
__global__ __launch_bounds__(kBlock) void embed_kernel(const T* table, int64_t vocab, int64_t dim,
                                                       int64_t stride, Tokens tokens, int64_t n,
                                                       float scale, T* out, int64_t out_stride,
                                                       int lanes, int64_t first) {
  constexpr int N = Vec<T>::kN;
  const int64_t i = first + int64_t(blockIdx.x) * (kBlock / lanes) + int(threadIdx.x) / lanes;
  if (i >= n) return;
  const int64_t t = token_in(tokens, i, vocab);
  const T* row = table + (t < 0 ? 0 : t) * stride;
  T* to = out + i * out_stride;
  for (int64_t j = int64_t(int(threadIdx.x) % lanes) * N; j < dim; j += int64_t(lanes) * N) {
    if (j + N <= dim) {
      typename Vec<T>::type v = T(0);
      if (t >= 0) {
        v = load16(row + j);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = T(float(v[k]) * scale);
      }
      store16(to + j, v);
    } else {
      for (int64_t k = j; k < dim; ++k) to[k] = t < 0 ? T(0) : T(float(row[k]) * scale);
    }
  }
}

// --- sort by token ----------------------------------------------------------

// One digit of a stable sort of the keys of a block, `kRounds` per lane: wave w
// holds keys w * 64 * kRounds .. in order, round r the r-th 64 of them.  counts
// (waves x kBins in LDS) ends as each wave's running count per digit; place()
// is called for every key with its number among the block's keys of its digit.
template <int kRounds, int kThreads>
__device__ __forceinline__ void count_digits(const uint32_t (&key)[kRounds],
                                             const bool (&on)[kRounds], int shift, int bins,
                                             uint32_t* counts) {
  for (int i = int(threadIdx.x); i < bins * (kThreads / kWave); i += kThreads) counts[i] = 0;
  __syncthreads();
  uint32_t* mine = counts + int(threadIdx.x) / kWave * bins;
#pragma unroll
  for (int r = 0; r < kRounds; ++r)
    if (on[r]) atomicAdd(&mine[(key[r] >> shift) & (bins - 1)], 1u);
  __syncthreads();
}

// Lanes of the wave with this lane's digit, of those taking part.
__device__ __forceinline__ uint64_t peers_of(uint32_t digit, bool on, int bits) {
  const uint64_t all = __ballot(on);
  uint32_t lo = uint32_t(all), hi = uint32_t(all >> 32);
  for (int b = 0; b < bits; ++b) {
    const int32_t own = int32_t(digit << (31 - b)) >> 31;  // the bit, in every place
    const uint64_t set = __ballot(own);
    lo &= ~(uint32_t(set) ^ uint32_t(own));
    hi &= ~(uint32_t(set >> 32) ^ uint32_t(own));
  }
  return uint64_t(hi) << 32 | lo;
}

// Exclusive sum over 512 or 1024 threads' values.
template <int kThreads>
__device__ __forceinline__ uint32_t block_before(uint32_t x, uint32_t* part) {
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
  uint32_t s = x;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const uint32_t up = __shfl_up(s, d);
    if (lane >= d) s += up;
  }
  if (lane == kWave - 1) part[wave] = s;
  __syncthreads();
  uint32_t before = s - x;
  for (int w = 0; w < wave; ++w) before += part[w];
  return before;
}

struct SortArgs {
  Tokens tokens;
  uint32_t n, vocab;
  int bits, passes;  // of a digit, and digits
  uint32_t *key[2], *at[2];
  uint32_t* hist;    // blocks x bins, and a row of sums
  int scanned;       // the counts have become those of earlier blocks
};

__device__ __forceinline__ uint32_t key_of(const SortArgs& a, uint32_t i) {
  const int64_t t = token_in(a.tokens, i, a.vocab);
  return t < 0 ? a.vocab : uint32_t(t);  // padding comes last
}

// All of n <= kSmall tokens in one block, in LDS.
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(SortArgs a) {
  constexpr int kRounds = kSmall / kSmallThreads, kWaves = kSmallThreads / kWave;
  __shared__ uint2 list[kSmall];
  __shared__ uint32_t counts[kWaves * kBins];
  __shared__ uint32_t part[kWaves];
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave, bins = 1 << a.bits;
  // Waves share the tokens evenly, in whole rounds.
  const uint32_t span = (a.n + kSmallThreads - 1) / kSmallThreads * kWave;
  uint32_t key[kRounds], at[kRounds];
  bool on[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint32_t i = uint32_t(wave) * span + uint32_t(r * kWave + lane);
    on[r] = uint32_t(r * kWave) < span && i < a.n;
    key[r] = on[r] ? key_of(a, i) : 0;
    at[r] = i;
  }
  for (int p = 0; p < a.passes; ++p) {
    const int shift = p * a.bits;
    count_digits<kRounds, kSmallThreads>(key, on, shift, bins, counts);
    uint32_t total = 0;
    if (int(threadIdx.x) < bins)
      for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = counts[w * bins + threadIdx.x];
        counts[w * bins + threadIdx.x] = total;
        total += c;
      }
    const uint32_t before = block_before<kSmallThreads>(total, part);
    if (int(threadIdx.x) < bins)
      for (int w = 0; w < kWaves; ++w) counts[w * bins + threadIdx.x] += before;
    __syncthreads();
    volatile uint32_t* mine = counts + wave * bins;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (uint32_t(r * kWave) >= span) continue;  // of all waves
      const uint32_t digit = (key[r] >> shift) & uint32_t(bins - 1);
      const uint64_t peers = peers_of(digit, on[r], a.bits);
      uint32_t base = 0;
      if (on[r]) base = mine[digit];
      __builtin_amdgcn_wave_barrier();
      if (on[r]) {
        list[base + uint32_t(__popcll(peers & below(lane)))] = {key[r], at[r]};
        if ((peers >> lane) == 1) mine[digit] = base + uint32_t(__popcll(peers));
      }
      __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
      if (on[r]) {
        const uint2 e = list[uint32_t(wave) * span + uint32_t(r * kWave + lane)];
        key[r] = e.x;
        at[r] = e.y;
      }
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < kRounds; ++r)
    if (on[r]) {
      const uint32_t i = uint32_t(wave) * span + uint32_t(r * kWave + lane);
      a.key[0][i] = key[r];
      a.at[0][i] = at[r];
    }
}

// Longer lists, a digit at a time: every block's count of each digit, then
// each block's keys to their places.
__global__ __launch_bounds__(kTileThreads) void sort_count_kernel(SortArgs a, int p) {
  __shared__ uint32_t counts[kBins];
  const int bins = 1 << a.bits;
  for (int i = int(threadIdx.x); i < bins; i += kTileThreads) counts[i] = 0;
  __syncthreads();
  const uint32_t first = blockIdx.x * uint32_t(kTile);
  for (uint32_t i = first + threadIdx.x; i < first + kTile && i < a.n; i += kTileThreads) {
    const uint32_t key = p == 0 ? key_of(a, i) : a.key[(p - 1) & 1][i];
    atomicAdd(&counts[(key >> (p * a.bits)) & uint32_t(bins - 1)], 1u);
  }
  __syncthreads();
  for (int i = int(threadIdx.x); i < bins; i += kTileThreads)
    a.hist[blockIdx.x * uint32_t(bins) + i] = counts[i];
}

// A block per digit: every tile's count becomes the sum of the tiles before it,
// and the last row the sum of all.
__global__ __launch_bounds__(kTileThreads) void sort_scan_kernel(SortArgs a, uint32_t tiles) {
  __shared__ uint32_t part[kTileThreads / kWave], carry;
  const uint32_t bins = 1u << a.bits;
  if (threadIdx.x == 0) carry = 0;
  for (uint32_t t0 = 0; t0 < tiles; t0 += kTileThreads) {
    const uint32_t t = t0 + threadIdx.x;
    const uint32_t x = t < tiles ? a.hist[t * bins + blockIdx.x] : 0;
    __syncthreads();  // the carry is there, and `part` has been read
    const uint32_t before = carry + block_before<kTileThreads>(x, part);
    if (t < tiles) a.hist[t * bins + blockIdx.x] = before;
    __syncthreads();
    if (threadIdx.x == kTileThreads - 1) carry = before + x;
  }
  __syncthreads();
  if (threadIdx.x == 0) a.hist[tiles * bins + blockIdx.x] = carry;
}

__global__ __launch_bounds__(kTileThreads) void sort_place_kernel(SortArgs a, int p) {
  constexpr int kRounds = kTile / kTileThreads, kWaves = kTileThreads / kWave;
  static_assert(kBins <= kTileThreads, "a thread per digit");
  __shared__ uint32_t counts[kWaves * kBins];
  __shared__ uint32_t part[kWaves];
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave, bins = 1 << a.bits;
  const int shift = p * a.bits;
  uint32_t key[kRounds], at[kRounds];
  bool on[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint32_t i = blockIdx.x * uint32_t(kTile) + uint32_t((wave * kRounds + r) * kWave + lane);
    on[r] = i < a.n;
    key[r] = !on[r] ? 0 : p == 0 ? key_of(a, i) : a.key[(p - 1) & 1][i];
    at[r] = !on[r] ? 0 : p == 0 ? i : a.at[(p - 1) & 1][i];
  }
  count_digits<kRounds, kTileThreads>(key, on, shift, bins, counts);
  // This block's first place of each digit: keys of lower digits, and of the
  // same digit in earlier blocks.
  uint32_t total = 0, earlier = 0;
  if (int(threadIdx.x) < bins && a.scanned) {
    total = a.hist[gridDim.x * uint32_t(bins) + threadIdx.x];
    earlier = a.hist[blockIdx.x * uint32_t(bins) + threadIdx.x];
  } else if (int(threadIdx.x) < bins) {
    for (uint32_t b = 0; b < gridDim.x; b += 16) {
      uint32_t c[16];  // under way at once
#pragma unroll
      for (uint32_t k = 0; k < 16; ++k)
        c[k] = a.hist[min(b + k, gridDim.x - 1) * uint32_t(bins) + threadIdx.x];
#pragma unroll
      for (uint32_t k = 0; k < 16; ++k) {
        total += b + k < gridDim.x ? c[k] : 0;
        earlier += b + k < blockIdx.x ? c[k] : 0;
      }
    }
  }
  uint32_t before = block_before<kTileThreads>(total, part) + earlier;
  if (int(threadIdx.x) < bins)
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t c = counts[w * bins + threadIdx.x];
      counts[w * bins + threadIdx.x] = before;
      before += c;
    }
  __syncthreads();
  volatile uint32_t* mine = counts + wave * bins;
  uint32_t *to_key = a.key[p & 1], *to_at = a.at[p & 1];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const uint32_t digit = (key[r] >> shift) & uint32_t(bins - 1);
    const uint64_t peers = peers_of(digit, on[r], a.bits);
    uint32_t base = 0;
    if (on[r]) base = mine[digit];
    __builtin_amdgcn_wave_barrier();
    if (on[r]) {
      const uint32_t to = base + uint32_t(__popcll(peers & below(lane)));
      to_key[to] = key[r];
      to_at[to] = at[r];
      if ((peers >> lane) == 1) mine[digit] = base + uint32_t(__popcll(peers));
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// --- sums over runs ---------------------------------------------------------

struct SumArgs {
  const void* d_rows;
  int64_t row_stride, dim, vocab;
  const uint32_t *key, *at;  // sorted
  uint32_t n, chunk;
  float* partial;            // n / chunk rows of dim
  float scale;
  void* table;
  int64_t table_stride;
  int lanes;                 // of a row's piece: a power of two up to 64
  int across, width;         // waves of a block that share a row, and pieces of each
  int per;                   // rows of the table, or places of the list, of a wave
  int64_t first;             // row of the table or place of the list that the launch starts with
};

// N values of a row from element j on, those that there are, in 16-byte pieces.
template <class T, int N>
__device__ __forceinline__ void read_piece(const T* row, int64_t j, int64_t dim, float (&x)[N]) {
  constexpr int M = Vec<T>::kN;
  if (j + N <= dim) {
#pragma unroll
    for (int k = 0; k < N; k += M) {
      const typename Vec<T>::type v = load16(row + j + k);
#pragma unroll
      for (int e = 0; e < M; ++e) x[k + e] = float(v[e]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = j + k < dim ? float(row[j + k]) : 0.f;
  }
}
template <class T, int N, bool kPast = false>
__device__ __forceinline__ void write_piece(T* row, int64_t j, int64_t dim, const float (&x)[N]) {
  constexpr int M = Vec<T>::kN;
  if (j + N <= dim) {
#pragma unroll
    for (int k = 0; k < N; k += M) {
      typename Vec<T>::type v;
#pragma unroll
      for (int e = 0; e < M; ++e) v[e] = T(x[k + e]);
      if (kPast) stream16(row + j + k, v);
      else store16(row + j + k, v);
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (j + k < dim) row[j + k] = T(x[k]);
  }
}

// kRows entries of each group of lanes, i, i + groups, .., all under way at once.
template <class T, int kRows>
__device__ __forceinline__ void add_batch(const SumArgs& a, uint32_t mine, int i, int64_t j,
                                          float (&acc)[Vec<T>::kN]) {
  constexpr int N = Vec<T>::kN;
  const T* rows = static_cast<const T*>(a.d_rows) + j;
  uint32_t at[kRows];  // by all lanes, before their ways part
#pragma unroll
  for (int k = 0; k < kRows; ++k) at[k] = __shfl(mine, i + k * (kWave / a.lanes));
  if (j + N <= a.dim) {
    typename Vec<T>::type v[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) v[k] = load16(rows + int64_t(at[k]) * a.row_stride);
#pragma unroll
    for (int k = 0; k < kRows; ++k)
#pragma unroll
      for (int q = 0; q < N; ++q) acc[q] += float(v[k][q]);
  } else {
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const T* row = rows + int64_t(at[k]) * a.row_stride;
#pragma unroll
      for (int q = 0; q < N; ++q)
        if (j + q < a.dim) acc[q] += float(row[q]);
    }
  }
}

template <class T>
__device__ __forceinline__ void add_last(const SumArgs& a, uint32_t mine, int i, int count,
                                         int64_t j, float (&acc)[Vec<T>::kN]) {
  const int64_t row = __shfl(mine, min(i, kWave - 1));
  if (i >= count) return;
  float x[Vec<T>::kN];
  read_piece(static_cast<const T*>(a.d_rows) + row * a.row_stride, j, a.dim, x);
#pragma unroll
  for (int q = 0; q < Vec<T>::kN; ++q) acc[q] += x[q];
}

// Sum of rows by a wave: 64 / lanes groups of lanes
// take an entry each, in 16-byte pieces; the groups' sums are added in one order
// at the end.
template <class T>
__device__ __forceinline__ void add_rows(const SumArgs& a, uint32_t b, uint32_t e, int64_t j,
                                         float (&acc)[Vec<T>::kN]) {
  const int lane = int(threadIdx.x) % kWave, groups = kWave / a.lanes, group = lane / a.lanes;
  for (uint32_t base = b; base < e; base += kWave) {
    const int count = int(min(e - base, uint32_t(kWave)));
    const uint32_t mine = lane < count ? a.at[base + lane] : 0;
    int i = 0;
    for (; i + 8 * groups <= count; i += 8 * groups) add_batch<T, 8>(a, mine, i + group, j, acc);
    if (i + 4 * groups <= count) {
      add_batch<T, 4>(a, mine, i + group, j, acc);
      i += 4 * groups;
    }
    if (i + 2 * groups <= count) {
      add_batch<T, 2>(a, mine, i + group, j, acc);
      i += 2 * groups;
    }
    if (i + groups <= count) {
      add_batch<T, 1>(a, mine, i + group, j, acc);
      i += groups;
    }
    if (i < count) add_last<T>(a, mine, i + group, count, j, acc);
  }
}

template <int N>
__device__ __forceinline__ void join_groups(const SumArgs& a, float (&acc)[N]) {
  for (int d = a.lanes; d < kWave; d <<= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) acc[k] += __shfl_xor(acc[k], d);
}

// The columns of a wave: `width` pieces of tile `tile`; lanes behind them (and
// behind the row) get a column that is not there.
template <class T>
__device__ __forceinline__ int64_t column(const SumArgs& a, int64_t tile) {
  const int lane = int(threadIdx.x) % kWave % a.lanes;
  return lane < a.width ? (tile * a.width + lane) * Vec<T>::kN : a.dim;
}

// Chunks of the list that hold one token only (parts of long runs).
template <class T>
__global__ __launch_bounds__(kMostThreads) void chunk_kernel(SumArgs a) {
  constexpr int N = Vec<T>::kN;
  const int wave = int(threadIdx.x) / kWave, at_once = int(blockDim.x) / kWave / a.across;
  const uint32_t c = blockIdx.x * uint32_t(at_once) + uint32_t(wave / a.across);
  if (c >= a.n / a.chunk) return;
  const uint32_t b = c * a.chunk, e = b + a.chunk, v = a.key[b];
  if (v != a.key[e - 1] || v >= uint32_t(a.vocab)) return;
  const int64_t j = column<T>(a, int64_t(blockIdx.y) * a.across + wave % a.across);
  float acc[N] = {};
  add_rows<T>(a, b, e, j, acc);
  join_groups(a, acc);
  if (int(threadIdx.x) % kWave < a.lanes)
    write_piece(a.partial + int64_t(c) * a.dim, j, a.dim, acc);
}

// First place of the sorted list whose token is at least v, by a wave: 64 probes
// at once.
__device__ __forceinline__ uint32_t place_of(const uint32_t* key, uint32_t n, uint32_t v) {
  const uint32_t lane = threadIdx.x % kWave;
  uint32_t lo = 0, hi = n;  // the place is in [lo, hi]
  while (hi - lo > kWave) {
    const uint32_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const uint32_t less = uint32_t(__popcll(__ballot(at < hi && key[at] < v)));
    if (less == 0) return lo;
    hi = min(hi, lo + less * step);
    lo += (less - 1) * step + 1;
  }
  return lo + uint32_t(__popcll(__ballot(lo + lane < hi && key[lo + lane] < v)));
}

// Row v of the table from the run [s, e): the entries before the first whole
// chunk, the chunks' sums, the entries behind the last.
template <class T, class O, bool kAdd>
__device__ __forceinline__ void table_row(const SumArgs& a, int64_t v, uint32_t s, uint32_t e,
                                          int64_t j) {
  constexpr int N = Vec<T>::kN, kAhead = 8;
  const int lane = int(threadIdx.x) % kWave, group = lane / a.lanes, groups = kWave / a.lanes;
  O* to = static_cast<O*>(a.table) + v * a.table_stride;
  float x[N] = {}, acc[N] = {};
  if (kAdd) read_piece(to, j, a.dim, x);
  const uint32_t c0 = (s + a.chunk - 1) / a.chunk, c1 = e / a.chunk;
  if (c1 > c0) {
    add_rows<T>(a, s, c0 * a.chunk, j, acc);
    for (uint32_t c = c0 + uint32_t(group); c < c1; c += uint32_t(groups * kAhead)) {
      float y[kAhead][N];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const uint32_t part = min(c + uint32_t(i * groups), c1 - 1);
        read_piece(a.partial + int64_t(part) * a.dim, j, a.dim, y[i]);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] += c + uint32_t(i * groups) < c1 ? y[i][k] : 0.f;
    }
    add_rows<T>(a, c1 * a.chunk, e, j, acc);
  } else {
    add_rows<T>(a, s, e, j, acc);
  }
  join_groups(a, acc);
  if (lane < a.lanes) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] += acc[k] * a.scale;
    write_piece<O, N, !kAdd>(to, j, a.dim, x);
  }
}

// Every row of the table, a few in turn by each wave, zeros for those without a
// run.
template <class T, class O>
__global__ __launch_bounds__(kMostThreads) void table_kernel(SumArgs a) {
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
  const int at_once = int(blockDim.x) / kWave / a.across;
  const int64_t v0 = a.first + (int64_t(blockIdx.x) * at_once + wave / a.across) * a.per;
  if (v0 >= a.vocab) return;
  const int64_t j = column<T>(a, int64_t(blockIdx.y) * a.across + wave % a.across);
  const uint32_t first = place_of(a.key, a.n, uint32_t(v0));
  const uint32_t near = first + lane < a.n ? a.key[first + lane] : ~0u;
  uint32_t s = first;
  for (int r = 0; r < a.per && v0 + r < a.vocab; ++r) {
    // The run's end is among the 64 entries at hand, or it is looked for.
    const int passed = __popcll(__ballot(near <= uint32_t(v0 + r)));
    const uint32_t e = passed < kWave ? first + uint32_t(passed)
                                      : place_of(a.key, a.n, uint32_t(v0 + r + 1));
    table_row<T, O, false>(a, v0 + r, s, e, j);
    s = e;
  }
}

// The rows that have a run, added to what is there: a wave takes the runs that
// begin at a few places of the list.
template <class T, class O>
__global__ __launch_bounds__(kMostThreads) void add_kernel(SumArgs a) {
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave;
  const int at_once = int(blockDim.x) / kWave / a.across;
  const int64_t first = a.first + (int64_t(blockIdx.x) * at_once + wave / a.across) * a.per;
  if (first >= a.n) return;
  const int64_t j = column<T>(a, int64_t(blockIdx.y) * a.across + wave % a.across);
  const uint32_t i = uint32_t(first) + uint32_t(lane);
  const uint32_t near = i < a.n ? a.key[i] : ~0u;
  const bool begins = lane < a.per && near < uint32_t(a.vocab) && (i == 0 || a.key[i - 1] != near);
  for (uint64_t heads = __ballot(begins); heads; heads &= heads - 1) {
    const int at = __ffsll((unsigned long long)heads) - 1;
    const uint32_t v = uint32_t(__shfl(near, at));
    const int passed = __popcll(__ballot(near <= v));
    const uint32_t e = passed < kWave ? uint32_t(first) + uint32_t(passed)
                                      : place_of(a.key, a.n, v + 1);
    table_row<T, O, true>(a, v, uint32_t(first) + uint32_t(at), e, j);
  }
}

int lanes_for(int64_t pieces, int most) {
  int l = 1;
  while (l < most && l < pieces) l *= 2;
  return l;
}

uint32_t chunk_for(int64_t n) {
  uint32_t c = 32;
  while (n / c > 4096) c *= 2;
  return c;
}

size_t up(size_t x) { return (x + 255) & ~size_t(255); }

uint32_t tiles_for(int64_t n) { return uint32_t((n + kTile - 1) / kTile); }

template <class T>
hipError_t embed_of(const sched_matrix& table, const sched_tokens& tokens, float scale,
                    const sched_matrix& out, hipStream_t s) {
  const int lanes = lanes_for((table.cols + Vec<T>::kN - 1) / Vec<T>::kN, kBlock);
  const int64_t blocks = (tokens.n + kBlock / lanes - 1) / (kBlock / lanes);
  hipError_t e = hipSuccess;
  for (int64_t b = 0; b < blocks && e == hipSuccess; b += kMostBlocks) {
    hipLaunchKernelGGL(embed_kernel<T>, dim3(unsigned(std::min(blocks - b, kMostBlocks))),
                       dim3(kBlock), 0, s, static_cast<const T*>(table.data), table.rows,
                       table.cols, table.stride, Tokens{tokens.data, tokens.bits == 64}, tokens.n,
                       scale, static_cast<T*>(out.data), out.stride, lanes, b * (kBlock / lanes));
    e = hipGetLastError();
  }
  return e;
}

template <class T, class O>
hipError_t sums_of(const SumArgs& in, bool accumulate, hipStream_t s) {
  SumArgs a = in;
  const int64_t pieces = (a.dim + Vec<T>::kN - 1) / Vec<T>::kN;
  a.lanes = lanes_for(pieces, kWave);
  // A row's waves stand in one block, up to 8 of them, and share its pieces
  // evenly; blocks of short rows take several rows.
  const int64_t waves = (pieces + kWave - 1) / kWave, parts = (waves + 7) / 8;
  a.across = int((waves + parts - 1) / parts);
  a.width = int((pieces + parts * a.across - 1) / (parts * a.across));
  if (a.width > 8) a.width = std::min((a.width + 7) / 8 * 8, kWave);  // whole lines
  const int at_once = std::max(1, 4 / a.across);
  const dim3 block(unsigned(kWave * a.across * at_once));
  if (const uint32_t chunks = a.n / a.chunk) {
    const unsigned blocks = (chunks + unsigned(at_once) - 1) / unsigned(at_once);
    hipLaunchKernelGGL(chunk_kernel<T>, dim3(blocks, unsigned(parts)), block, 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t all = accumulate ? int64_t(a.n) : a.vocab;
  // Few rows a wave where there are few, many (one search in the list for all)
  // where there are more than fill the card: 131072 x 4096, 65,536 tokens, 4, 8
  // and 16 rows a wave 526, 490 and 467 us; 200 x 1024, 60,000 tokens, 115, 147
  // and 183.
  a.per = 1;
  while (a.per < 16 && all * waves / (a.per * 2) >= 16384) a.per *= 2;
  const int64_t per = int64_t(at_once) * a.per;
  const int64_t blocks = (all + per - 1) / per;
  hipError_t e = hipSuccess;
  for (int64_t b = 0; b < blocks && e == hipSuccess; b += kMostBlocks) {
    a.first = b * per;
    const dim3 grid(unsigned(std::min(blocks - b, kMostBlocks)), unsigned(parts));
    if (accumulate)
      hipLaunchKernelGGL((add_kernel<T, O>), grid, block, 0, s, a);
    else
      hipLaunchKernelGGL((table_kernel<T, O>), grid, block, 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

template <class T>
hipError_t sums_to(const SumArgs& a, bool same, bool accumulate, hipStream_t s) {
  return same ? sums_of<T, T>(a, accumulate, s) : sums_of<T, float>(a, accumulate, s);
}

}  // namespace

hipError_t launch_embed(const sched_matrix& table, const sched_tokens& tokens, float scale,
                        const sched_matrix& out, hipStream_t s) {
  if (tokens.n == 0 || table.cols == 0) return hipSuccess;
  return table.dtype == SCHED_F32   ? embed_of<float>(table, tokens, scale, out, s)
         : table.dtype == SCHED_F16 ? embed_of<f16>(table, tokens, scale, out, s)
                                    : embed_of<bf16>(table, tokens, scale, out, s);
}

size_t embed_grad_bytes(int64_t n, int64_t dim) {
  const size_t lists = n <= kSmall ? 2 : 4;
  return lists * up(size_t(n) * 4) + (n <= kSmall ? 0 : up(size_t(tiles_for(n) + 1) * kBins * 4)) +
         up(size_t(n / chunk_for(n)) * size_t(dim) * 4);
}

hipError_t launch_embed_grad(const sched_matrix& d_rows, const sched_tokens& tokens, float scale,
                             bool accumulate, const sched_matrix& d_table, void* ws,
                             hipStream_t s) {
  if (d_table.rows == 0 || d_table.cols == 0) return hipSuccess;
  SortArgs a = {};
  a.tokens = {tokens.data, tokens.bits == 64};
  a.n = uint32_t(tokens.n);
  a.vocab = uint32_t(d_table.rows);
  const int width = 32 - __builtin_clz(a.vocab);  // keys are 0 .. vocab
  a.passes = (width + kDigit - 1) / kDigit;
  a.bits = (width + a.passes - 1) / a.passes;
  char* at = static_cast<char*>(ws);
  auto take = [&](size_t bytes) {
    char* p = at;
    at += up(bytes);
    return p;
  };
  int last = 0;
  a.key[0] = reinterpret_cast<uint32_t*>(take(size_t(a.n) * 4));
  a.at[0] = reinterpret_cast<uint32_t*>(take(size_t(a.n) * 4));
  hipError_t e = hipSuccess;
  if (a.n > uint32_t(kSmall)) {
    a.key[1] = reinterpret_cast<uint32_t*>(take(size_t(a.n) * 4));
    a.at[1] = reinterpret_cast<uint32_t*>(take(size_t(a.n) * 4));
    const uint32_t tiles = tiles_for(a.n);
    a.hist = reinterpret_cast<uint32_t*>(take(size_t(tiles + 1) * kBins * 4));
    // With few tiles every block adds up the counts of the others by itself.
    a.scanned = tiles > kScanned;
    for (int p = 0; p < a.passes && e == hipSuccess; ++p) {
      hipLaunchKernelGGL(sort_count_kernel, dim3(tiles), dim3(kTileThreads), 0, s, a, p);
      e = hipGetLastError();
      if (e != hipSuccess) break;
      if (a.scanned) {
        hipLaunchKernelGGL(sort_scan_kernel, dim3(1u << a.bits), dim3(kTileThreads), 0, s, a, tiles);
        e = hipGetLastError();
        if (e != hipSuccess) break;
      }
      hipLaunchKernelGGL(sort_place_kernel, dim3(tiles), dim3(kTileThreads), 0, s, a, p);
      e = hipGetLastError();
    }
    last = (a.passes - 1) & 1;
  } else if (a.n > 0) {
    hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(kSmallThreads), 0, s, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  SumArgs b = {};
  b.d_rows = d_rows.data;
  b.row_stride = d_rows.stride;
  b.dim = d_table.cols;
  b.vocab = d_table.rows;
  b.key = a.key[last];
  b.at = a.at[last];
  b.n = a.n;
  b.chunk = chunk_for(a.n);
  b.partial = reinterpret_cast<float*>(at);
  b.scale = scale;
  b.table = d_table.data;
  b.table_stride = d_table.stride;
  const bool same = d_table.dtype == d_rows.dtype;
  return d_rows.dtype == SCHED_F32   ? sums_to<float>(b, same, accumulate, s)
         : d_rows.dtype == SCHED_F16 ? sums_to<f16>(b, same, accumulate, s)
                                     : sums_to<bf16>(b, same, accumulate, s);
}

}  // namespace policy
