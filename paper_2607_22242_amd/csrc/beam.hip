// beam.hip -- beam search: the best continuations of each group's beams, and the
// beams' states following them.
//
// Logits are read once.  Every wave takes a strip of a row and keeps its `width`
// best logits (a continuation that is not among its strip's best is not among
// the group's) and what the sum of powers needs; a block per group then gives
// the strips' best their scores and takes the best of those.  Bound by the
// logits' bytes where rows are long, and by what waits for one another in a
// group's block where they are short.  16 groups of 16 beams, 131,072 logits in
// bfloat16: strips 31 us (67 MB, 2.2 TB/s: 16 vector operations a logit, 5 of them
// for its power), groups 13.  Sums of powers are held in 32 bits, relative to the
// largest logit met; scores are formed in 64, as a score that has been added up
// over many tokens is no finer than 2^-24 of itself in 32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "policy_launch.h"
#include "tensors.h"

namespace policy {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMostWidth = 128;
constexpr int kRounds = 4;                        // of a chunk: eight logits a lane each
constexpr int kChunk = kRounds * 8 * kWave;       // logits of a chunk
constexpr int kMostStrips = 64;                   // of a row
constexpr uint32_t kLeast = 0x00800000u;          // the order of the lowest finite logit
constexpr int kTokenBits = 22;                    // a row has up to 2^22 logits

// Floating-point numbers' order as that of whole numbers; zeros are one number.
// What is less than kLeast (-inf, and 0 for what is not there) is no candidate.
__device__ __forceinline__ uint32_t order_of(float x) {
  x += 0.f;
  const uint32_t u = __float_as_uint(x);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t order_of(double x) {
  x += 0.;
  const uint64_t u = uint64_t(__double_as_longlong(x));
  return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}
__device__ __forceinline__ double of_order(uint64_t k) {
  return __longlong_as_double(
      (long long)(k >> 63 ? k & ~(uint64_t(1) << 63) : ~k));
}

// Lanes of the mask before this one.
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}
// The lowest bit in which the orders of a type's numbers differ by more than their
// sign: 16-bit numbers have fewer digits.
template <class T>
constexpr int kLowest = sizeof(T) == 4 ? 0 : std::is_same<T, bf16>::value ? 16 : 13;
template <class T>
__device__ __forceinline__ uint32_t with_low_bits(uint32_t order) {
  return order >> 31 ? order : order | ((1u << kLowest<T>) - 1);
}

// What a wave's lanes have written to LDS is read by its other lanes from here on.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

struct Entry {
  uint32_t order, token;
};

// A wave's list of candidates in LDS, of as many as it can come to (room_of).
// cut() leaves the k best (greater orders, of equal ones lower tokens), in no order.
__host__ __device__ inline int reach_of(int k) { return k + (k < 48 ? k : 48); }
__host__ __device__ inline int room_of(int k) { return 8 * reach_of(k) + k + 2 * kWave; }
template <class T>
struct List {
  Entry* at;
  int n;           // entries
  uint32_t least;  // k logits of this or a greater order have been met

  // Adds an entry of each lane that has one, in the lanes' order.
  __device__ __forceinline__ void add(bool have, uint32_t order, uint32_t token) {
    const uint64_t mask = __ballot(have);
    if (!mask) return;
    if (have) at[n + lanes_before(mask)] = {order, token};
    n += __popcll(mask);
  }

  __device__ __forceinline__ void cut(int k) {
    if (n <= k) return;
    wave_order();
    const int lane = int(threadIdx.x) % kWave;
    if (n <= 2 * kWave) {
      held<2>(k);
    } else if (n <= 4 * kWave) {
      held<4>(k);
    } else if (n <= 8 * kWave) {
      held<8>(k);
    } else if (n <= 16 * kWave) {
      held<16>(k);
    } else {
      const int rounds = (n + kWave - 1) / kWave;
      leave<2>(k, rounds, [&](int i) {
        return i * kWave + lane < n ? at[i * kWave + lane] : Entry{0, ~0u};
      });
    }
  }

 private:
  // Entries in registers (2 groups of 40 beams of 12,709 logits: strips 13 us, 32 if what
  // is more than 128 entries is counted in LDS).
  template <int kHeld>
  __device__ __forceinline__ void held(int k) {
    const int lane = int(threadIdx.x) % kWave;
    Entry e[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      e[i] = {0, ~0u};
      if (i * kWave + lane < n) e[i] = at[i * kWave + lane];
    }
    leave<kHeld>(k, kHeld, [&](int i) { return e[i]; });
  }
  template <int kUnroll, class Get>
  __device__ __forceinline__ void leave(int k, int rounds, Get get) {
    auto count = [&](auto in) {
      int c = 0;
#pragma unroll kUnroll
      for (int i = 0; i < rounds; ++i) c += __popcll(__ballot(in(get(i))));
      return c;
    };
    // The greatest order that k entries have or pass, bit by bit.
    uint32_t v = 0;
    int reach = n;
#pragma unroll 1
    for (int bit = 31; bit >= kLowest<T> && reach != k; --bit) {
      const uint32_t t = v | 1u << bit;
      const int c = count([&](const Entry& x) { return x.order >= t; });
      if (c >= k) {
        v = t;
        reach = c;
      }
    }
    if (reach != k) v = with_low_bits<T>(v);  // a logit's order
    // Of those that have it the lowest tokens: the least bound that leaves k.
    uint32_t upto = ~0u;
    if (reach != k) {
      const int over = count([&](const Entry& x) { return x.order > v; });
      uint32_t below = 0;  // fewer than k - over have a lower token
#pragma unroll 1
      for (int bit = kTokenBits - 1; bit >= 0; --bit) {
        const uint32_t t = below | 1u << bit;
        if (over + count([&](const Entry& x) { return x.order == v && x.token < t; }) < k) below = t;
      }
      upto = below;
    }
    // In place: what is written lies before what is read next.
    const int all = n;
    n = 0;
#pragma unroll kUnroll
    for (int i = 0; i < rounds; ++i) {
      const int kept = n;
      n = all;  // what get() looks at
      const Entry e = get(i);
      n = kept;
      wave_order();
      add(e.order > v || (e.order == v && e.token <= upto), e.order, e.token);
      wave_order();
    }
    least = max(least, v);
  }
};

struct BeamArgs {
  const char* logits;
  int64_t stride;
  int32_t rows, cols, beams, width, strips, strip_chunks, stay, lists;  // lists: of a row
  uint32_t per_each;  // ceil(2^32 / candidates of a beam), in 32 bits: quotients of small numbers
  const float* scores;
  Tokens last;
  int64_t end_token;
  double per_temperature;     // 1 / temperature
  float factor;               // log2(e) / temperature
  Entry* entries;             // rows x lists x width; 0 orders fill what is left
  float2* sums;               // rows x strips: largest logit, sum of powers relative to it
  float* new_scores;
  int32_t* parents;
  void* tokens;
  int32_t wide_tokens;
};

__device__ __forceinline__ bool finished(const BeamArgs& a, int64_t row) {
  return a.last.data && a.end_token >= 0 && token_at(a.last, row) == a.end_token;
}
__device__ __forceinline__ bool present(const BeamArgs& a, int64_t row) {
  return fabsf(a.scores[row]) < INFINITY;
}

// Eight logits a lane of each of a chunk's rounds, as they are in memory; -inf
// behind the last.
template <class T>
struct Chunk {
  typename Vec<T>::type part[kRounds][8 / Vec<T>::kN];

  __device__ __forceinline__ void fetch(const T* row, int64_t at, int64_t end) {
    const int64_t mine = at + 8 * (int(threadIdx.x) % kWave);
    if (at + kChunk <= end) {
#pragma unroll
      for (int r = 0; r < kRounds; ++r)
#pragma unroll
        for (int i = 0; i < 8 / Vec<T>::kN; ++i)
          part[r][i] = load16(row + mine + r * 8 * kWave + i * Vec<T>::kN);
      return;
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
#pragma unroll
      for (int i = 0; i < 8 / Vec<T>::kN; ++i) {
        const int64_t first = mine + r * 8 * kWave + i * Vec<T>::kN;
        if (first + Vec<T>::kN <= end) {
          part[r][i] = load16(row + first);
        } else {
#pragma unroll
          for (int e = 0; e < Vec<T>::kN; ++e)
            part[r][i][e] = first + e < end ? row[first + e] : T(-INFINITY);
        }
      }
  }
  __device__ __forceinline__ float at(int r, int e) const {
    return float(part[r][e / Vec<T>::kN][e % Vec<T>::kN]);
  }
};

// --- strips of rows -----------------------------------------------------------

// Adds what is `bound` at least, or passes it and of what is equal to it the first
// `first`; eights: the greatest of each lane's eight.
template <class T, bool kFirst>
__device__ __forceinline__ void add_chunk(List<T>& list, const Chunk<T>& x, const float (&eights)[kRounds],
                                          float bound, uint32_t token0, int first) {
  int taken = 0;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    if (!__ballot(eights[r] >= bound)) continue;
    const uint32_t token = token0 + r * 8 * kWave + 8 * (int(threadIdx.x) % kWave);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = x.at(r, e);
      const bool in = kFirst ? v > bound : v >= bound;
      if (__ballot(in)) list.add(in, order_of(v), token + e);
    }
    if (!kFirst) continue;
    // The first of those that are equal, in the tokens' order.
    int nth = taken;
#pragma unroll
    for (int e = 0; e < 8; ++e) nth += lanes_before(__ballot(x.at(r, e) == bound));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = x.at(r, e);
      taken += __popcll(__ballot(v == bound));
      list.add(v == bound && nth < first, order_of(v), token + e);
      nth += v == bound;
    }
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void strips_kernel(BeamArgs a, int64_t first) {
  extern __shared__ Entry lists[];
  const int lane = int(threadIdx.x) % kWave, k = a.width, room = room_of(k);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
  const int64_t unit = first + int64_t(blockIdx.x) * kWaves + wave;
  if (unit >= int64_t(a.rows) * a.strips) return;
  const int64_t row = unit / a.strips;
  const int strip = int(unit % a.strips);
  if (finished(a, row) || !present(a, row)) return;  // its logits do not matter
  const T* const logits = reinterpret_cast<const T*>(a.logits) + row * a.stride;
  const int64_t begin = int64_t(strip) * a.strip_chunks * kChunk;
  const int64_t end = min(begin + int64_t(a.strip_chunks) * kChunk, int64_t(a.cols));
  List<T> list = {lists + wave * room, 0, 0};
  float most = -INFINITY, sum = 0.f;  // of this lane's logits
  Chunk<T> next;
  next.fetch(logits, begin, end);
  for (int64_t at = begin; at < end; at += kChunk) {
    const Chunk<T> x = next;
    if (at + kChunk < end) next.fetch(logits, at + kChunk, end);
    // The greatest of each lane's eights, and of all so far.
    float eights[kRounds], up = most;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      eights[r] = x.at(r, 0);
#pragma unroll
      for (int e = 1; e < 8; ++e) eights[r] = fmaxf(eights[r], x.at(r, e));
      up = fmaxf(up, eights[r]);
    }
    // Powers relative to it; NaN and +inf end in a sum of NaN.
    const float from = up == -INFINITY ? 0.f : up;
    if (__any(up > most))
      sum = most == -INFINITY ? sum : sum * pow2((most - from) * a.factor);  // 0, or NaN met before
    float sums[kRounds] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int r = 0; r < kRounds; ++r) sums[r] += pow2((x.at(r, e) - from) * a.factor);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) sum += sums[r];
    most = up;
    // What is taken: all that may be among the k best.  Where many eights have some, a
    // bound that k of them reach, and not many more, is found bit by bit; a bound
    // that more reach however far one looks is a value of many logits, of which the
    // first k are taken.
    uint32_t bound = max(list.least, kLeast - 1) + 1;  // what has been met k times does
    float least = of_order(bound);                     // not count any more
    int reach = 0;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) reach += __popcll(__ballot(eights[r] >= least));
    if (!reach) continue;
    const int most_reach = reach_of(k);
    if (reach > most_reach) {
      uint32_t top[kRounds], v = 0;
#pragma unroll
      for (int r = 0; r < kRounds; ++r) top[r] = eights[r] > -INFINITY ? order_of(eights[r]) : 0u;
#pragma unroll 1
      for (int bit = 31; bit >= kLowest<T> && reach > most_reach; --bit) {
        const uint32_t t = v | 1u << bit;
        int c = 0;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) c += __popcll(__ballot(top[r] >= t));
        if (c >= k) {
          v = t;
          reach = c;
        }
      }
      if (reach > most_reach) v = with_low_bits<T>(v);
      if (v >= bound) {
        bound = v;
        least = of_order(bound);
        if (bound > list.least) list.least = bound;  // k logits have it or pass it
      }
    }
    if (list.n + 8 * min(reach, most_reach) + k > room) list.cut(k);
    if (reach > most_reach) add_chunk<T, true>(list, x, eights, least, uint32_t(at), k);
    else add_chunk<T, false>(list, x, eights, least, uint32_t(at), k);
    if (list.n > 2 * k + kWave) list.cut(k);
  }
  list.cut(k);
  wave_order();
  Entry* const out = a.entries + unit * k;
  for (int i = lane; i < k; i += kWave) out[i] = i < list.n ? list.at[i] : Entry{0, ~0u};
  const float top = wave_max(most), from = top == -INFINITY ? 0.f : top;
  sum = wave_sum(most == -INFINITY ? sum : sum * pow2((most - from) * a.factor));
  if (lane == 0) a.sums[unit] = make_float2(from, sum);
}

// A row's lists become one, where the group's together would be too many: a wave
// each, in place.
__global__ __launch_bounds__(kThreads) void join_lists_kernel(BeamArgs a) {
  extern __shared__ Entry lists[];
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave, k = a.width;
  const int room = room_of(k);
  const int64_t row = int64_t(blockIdx.x) * kWaves + wave;
  if (row >= a.rows || finished(a, row) || !present(a, row)) return;
  List<float> list = {lists + wave * room, 0, 0};
  Entry* const in = a.entries + row * a.strips * k;
  const int n = a.strips * k;
  for (int i = 0; i < n; i += kWave) {
    Entry e = {0, ~0u};
    if (i + lane < n) e = in[i + lane];
    list.add(e.order >= max(list.least, kLeast), e.order, e.token);
    if (list.n + kWave > room) list.cut(k);
  }
  list.cut(k);
  wave_order();
  for (int i = lane; i < k; i += kWave) in[i] = i < list.n ? list.at[i] : Entry{0, ~0u};
}

// --- a group's best -------------------------------------------------------------

// Sums over a block of one number per thread's wave: waves count by ballots.
template <int kCount>
struct Counter {
  int (*room)[kCount];
  int turn;
  __device__ __forceinline__ int total(int wave_count) {
    const int wave = int(threadIdx.x) / kWave;
    turn ^= 1;  // the last total may still be read
    if (int(threadIdx.x) % kWave == 0) room[turn][wave] = wave_count;
    __syncthreads();
    int c = 0;
#pragma unroll
    for (int w = 0; w < kCount; ++w) c += room[turn][w];
    return c;
  }
  // Of the last total, what the waves before this one counted.
  __device__ __forceinline__ int before() const {
    int c = 0;
    for (int w = 0; w < int(threadIdx.x) / kWave; ++w) c += room[turn][w];
    return c;
  }
};

constexpr int kMostRanked = 256;  // candidates that are ranked one against the other
enum State : int { kNone, kLive, kFinished };

// A block takes a group.  kSmall: the group's logits themselves (kHeld kBlock at
// most); else the strips' lists.  A few blocks are all there is, so that what counts
// is how many loads wait for one another: the candidates are under way first.  Ranking
// is n^2 comparisons in 64 bits over the block's threads: of 1,024 candidates 42 us, of
// 256 some 2; hence kMostRanked.
template <class T, int kBlock, int kHeld, bool kSmall>
__global__ __launch_bounds__(kBlock) void group_kernel(BeamArgs a) {
  // Of a beam: its greatest logit, and what is added to (logit - greatest) / temperature,
  // or its score.
  __shared__ float greatest[kMostWidth];
  __shared__ double base[kMostWidth];
  __shared__ int state[kMostWidth], best_rank[kMostWidth], free_slots[kMostWidth];
  __shared__ int counts[2][kBlock / kWave];
  __shared__ uint32_t bounds[3][kBlock / kWave];
  __shared__ uint64_t masks[2][2], best_score[kMostRanked], sorted_score[kMostWidth];
  __shared__ uint32_t best_place[kMostRanked], sorted_place[kMostWidth];  // beam and token
  const int group = int(blockIdx.x), t = int(threadIdx.x), lane = t % kWave, wave = t / kWave;
  const int64_t row0 = int64_t(group) * a.beams;
  const int k = a.width;
  const T* const logits = reinterpret_cast<const T*>(a.logits);

  const int each = kSmall ? a.cols : a.lists * k, n = a.beams * each;
  auto beam_of = [&](int c) { return a.per_each ? int(__umulhi(uint32_t(c), a.per_each)) : c; };
  float x[kHeld];
  uint32_t token[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = i * kBlock + t, b = beam_of(c), r = c - b * each;
    x[i] = -INFINITY;
    token[i] = uint32_t(r);
    if (c >= n) continue;
    if (kSmall) {
      x[i] = float(logits[(row0 + b) * a.stride + r]);
    } else {  // of a beam without logits: what the memory held, which is not used
      const Entry e = a.entries[(row0 + b) * a.strips * k + r];
      x[i] = e.order >= kLeast ? of_order(e.order) : -INFINITY;
      token[i] = e.token & ((1u << kTokenBits) - 1);
    }
  }

  // Every beam's greatest logit, and its base: score - log of the sum of powers.
  const int per_row = kSmall ? a.cols : a.strips;
  int lanes = 1;
  while (lanes < per_row && lanes < kWave) lanes *= 2;
  const int at_once = kBlock / lanes;
  for (int b0 = 0; b0 < a.beams; b0 += at_once) {
    const int b = b0 + t / lanes;
    const int64_t row = row0 + min(b, a.beams - 1);
    const float score = a.scores[row];
    const bool done = finished(a, row);
    float most = -INFINITY, sum = 0.f;
    auto power = [&](float y, float from) { return pow2((y - from) * a.factor); };
    for (int i = t % lanes; i < per_row; i += lanes) {
      float y, s = 1.f;
      if (kSmall) {
        y = float(logits[row * a.stride + i]);
      } else {
        const float2 p = a.sums[row * a.strips + i];
        y = p.x;
        s = p.y;
      }
      if (kSmall ? y == -INFINITY : s == 0.f) continue;
      const float up = fmaxf(most, y);
      sum = (most == -INFINITY ? sum : sum * power(most, up)) + s * power(y, up);
      most = up;
    }
    for (int d = lanes / 2; d; d >>= 1) {
      const float y = __shfl_xor(most, d), s = __shfl_xor(sum, d), up = fmaxf(most, y);
      sum = up == -INFINITY ? sum + s
                            : (most == -INFINITY ? sum : sum * power(most, up)) +
                                  (y == -INFINITY ? s : s * power(y, up));
      most = up;
    }
    if (b < a.beams && t % lanes == 0) {
      const bool there = fabsf(score) < INFINITY;
      const bool ok = sum > 0.f && sum < INFINITY && fabsf(most) < INFINITY;
      state[b] = !there ? kNone : done ? kFinished : ok ? kLive : kNone;
      greatest[b] = most;
      base[b] = done ? double(score) : double(score) - log(double(sum));
    }
  }
  if (t < kMostWidth) best_rank[t] = kMostWidth;
  __syncthreads();

  // The candidates: score's order (0: none) and place.
  uint64_t score[kHeld];
  uint32_t place[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = i * kBlock + t, b = min(beam_of(c), a.beams - 1);
    const int is = state[b];
    const bool alone = is == kFinished;
    // The greatest is taken away first: added to it, what is far below (a score beside a
    // row of a type's lowest number) would be lost.
    const double s = base[b] + (alone ? 0. : (double(x[i]) - double(greatest[b])) * a.per_temperature);
    const bool on = c < n && (alone ? c == b * each : is == kLive) && s > -INFINITY && s < INFINITY;
    score[i] = on ? order_of(s) : 0;
    place[i] = on ? uint32_t(b) << kTokenBits | (alone ? 0u : token[i]) : ~0u;
  }

  // What may be among the k best.  Every wave finds a bound that k of its own scores
  // reach, and not many more, bit by bit; where what reaches the greatest of them is still
  // many the waves go on together, and the rest is ranked one against the other.
  Counter<kBlock / kWave> counter = {counts, 0};
  auto in_wave = [&](auto in) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i * kBlock < n) c += __popcll(__ballot(in(score[i], place[i])));
    return c;
  };
  auto count = [&](auto in) { return counter.total(in_wave(in)); };
  uint32_t least = 0;  // of the order's upper half
  const int mine = in_wave([&](uint64_t s, uint32_t) { return s > 0; });
  if (n > kMostRanked) {
    uint32_t hi = 0, lo = ~0u;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (score[i] > 0) {
        hi = max(hi, uint32_t(score[i] >> 32));
        lo = min(lo, uint32_t(score[i] >> 32));
      }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
      hi = max(hi, uint32_t(__shfl_xor(int(hi), d)));
      lo = min(lo, uint32_t(__shfl_xor(int(lo), d)));
    }
    least = mine ? lo : 0;
    if (mine > 2 * k) {
      int bit = 31 - __clz(int(hi ^ lo));  // the bits above are all scores'
      least = bit < 0 ? hi : hi >> bit >> 1 << bit << 1;
      int reach = mine;
#pragma unroll 1
      for (; bit >= 0 && reach > 2 * k; --bit) {
        const uint32_t bound = least | 1u << bit;
        const int c = in_wave([&](uint64_t s, uint32_t) { return uint32_t(s >> 32) >= bound; });
        if (c >= k) {
          least = bound;
          reach = c;
        }
      }
    }
    if (lane == 0) {
      bounds[0][wave] = mine >= k ? least : 0;
      bounds[1][wave] = mine ? lo : ~0u;
      bounds[2][wave] = hi;
    }
  }
  const int there = counter.total(mine);
  uint64_t v = 1;
  uint32_t low = ~0u, high = 0;  // of all scores
  if (n > kMostRanked) {
    least = 0;
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) {
      least = max(least, bounds[0][w]);
      low = min(low, bounds[1][w]);
      high = max(high, bounds[2][w]);
    }
    v = max(uint64_t(least) << 32, uint64_t(1));
  }
  int reach = count([&](uint64_t s, uint32_t) { return s >= v; });
  if (reach > kMostRanked) {  // the waves together, in the same way
    low = max(low, least);
    int bit = 31 - __clz(int(high ^ low));
    least = bit < 0 ? high : high >> bit >> 1 << bit << 1;
#pragma unroll 1
    for (; bit >= 0 && reach > kMostRanked; --bit) {
      const uint32_t bound = least | 1u << bit;
      const int c = count([&](uint64_t s, uint32_t) { return uint32_t(s >> 32) >= bound; });
      if (c >= k) {
        least = bound;
        reach = c;
      }
    }
    v = max(uint64_t(least) << 32, v);
    reach = count([&](uint64_t s, uint32_t) { return s >= v; });
  }
  uint32_t upto = ~0u;
  if (reach > kMostRanked) {
    // Many equal scores: exactly the k best, by score and place.
    v = 0;
    reach = there;
#pragma unroll 1
    for (int bit = 63; bit >= 0 && reach != k; --bit) {
      const uint64_t bound = v | uint64_t(1) << bit;
      const int c = count([&](uint64_t s, uint32_t) { return s >= bound; });
      if (c >= k) {
        v = bound;
        reach = c;
      }
    }
    if (reach != k) {
      const int over = count([&](uint64_t s, uint32_t) { return s > v; });
      uint32_t below = 0;
#pragma unroll 1
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t bound = below | 1u << bit;
        if (over + count([&](uint64_t s, uint32_t p) { return s == v && p < bound; }) < k)
          below = bound;
      }
      upto = below;
      reach = k;
    }
    count([&](uint64_t s, uint32_t p) { return s > v || (s == v && p <= upto); });
  }
  int at_best = counter.before();
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const bool in = score[i] > v || (score[i] == v && place[i] <= upto);
    const uint64_t mask = __ballot(in);
    if (in) {
      best_score[at_best + lanes_before(mask)] = score[i];
      best_place[at_best + lanes_before(mask)] = place[i];
    }
    at_best += __popcll(mask);
  }
  __syncthreads();
  const int got = min(there, k);
  {
    constexpr int kSides = kBlock / kMostRanked;  // threads that rank one
    const int c = t / kSides;
    const uint64_t s = best_score[c];
    const uint32_t p = best_place[c];
    int rank = 0;
    if (c < reach) {
#pragma unroll 8
      for (int i = t % kSides; i < reach; i += kSides) {
        const uint64_t other = best_score[i];
        const uint32_t at = best_place[i];
        rank += int(other > s) | (int(other == s) & int(at < p));
      }
    }
#pragma unroll
    for (int d = 1; d < kSides; d *= 2) rank += __shfl_xor(rank, d);
    if (c < reach && t % kSides == 0 && rank < k) {
      sorted_score[rank] = s;
      sorted_place[rank] = p;
    }
  }
  __syncthreads();

  // Rank t's slot.
  int slot = t;
  const uint32_t at = t < got ? sorted_place[t] : 0;
  const int beam = int(at >> kTokenBits);
  if (a.stay) {
    if (t < got) atomicMin(&best_rank[beam], t);
    __syncthreads();
    const bool kept = t < got && best_rank[beam] == t;  // the beam's best continuation
    const bool moves = t < k && !kept, open = t < k && best_rank[t] == kMostWidth;
    if (wave < 2) {
      const uint64_t a0 = __ballot(moves), a1 = __ballot(open);
      if (lane == 0) {
        masks[0][wave] = a0;
        masks[1][wave] = a1;
      }
    }
    __syncthreads();
    if (wave < 2) {  // as many ranks move as slots are left
      auto nth = [&](int which) {
        return lanes_before(masks[which][wave]) + (wave ? __popcll(masks[which][0]) : 0);
      };
      if (open) free_slots[nth(1)] = t;
      slot = kept ? beam : nth(0);
    }
    __syncthreads();
    if (moves) slot = free_slots[slot];
  }
  if (t >= k) return;
  const int64_t out = int64_t(group) * k + slot;
  int64_t next = -1;
  int parent = -1;
  float new_score = -INFINITY;
  if (t < got) {
    parent = int(row0 + beam);
    next = state[beam] == kFinished ? a.end_token : int64_t(at & ((1u << kTokenBits) - 1));
    new_score = float(of_order(sorted_score[t]));
  }
  a.new_scores[out] = new_score;
  a.parents[out] = parent;
  if (a.wide_tokens) static_cast<int64_t*>(a.tokens)[out] = next;
  else static_cast<int32_t*>(a.tokens)[out] = int32_t(next);
}

struct Plan {
  int strips, strip_chunks, lists;
  bool small;
};
constexpr int kMostHeld = 16;  // candidates of a thread of 1024

Plan plan_of(const sched_beam_desc& d) {
  Plan p = {};
  const int64_t cols = d.logits.cols, rows = d.logits.rows;
  // The group's block reads the logits itself where they are few: 13 groups of 16 beams,
  // 128 logits 13.2 us, 17.3 by strips; of 64 beams, 16 logits 14.1 and 21.5; of 32 beams,
  // 128 logits 19.0 and 16.7; of 8 beams, 400 logits, which it does not, 14.2 and 12.8.
  p.small = cols <= 4 * kWave && cols * d.beams <= 4096;
  const int64_t chunks = (cols + kChunk - 1) / kChunk;
  // Some 4096 waves, as far as rows are long enough (256 rows of 131,072, with the groups'
  // blocks: 2,048 waves take 4 % longer, 8,192 23 %).
  const int64_t want = std::min<int64_t>(
      {std::max<int64_t>(1, 4096 / std::max<int64_t>(rows, 1)), chunks, int64_t(kMostStrips)});
  p.strip_chunks = int((chunks + want - 1) / want);
  p.strips = int((chunks + p.strip_chunks - 1) / p.strip_chunks);
  p.lists = int64_t(d.beams) * p.strips * d.width > kMostHeld * 1024 ? 1 : p.strips;
  return p;
}

template <class T, int kBlock, int kHeld, bool kSmall>
hipError_t group(const BeamArgs& a, int groups, hipStream_t s) {
  hipLaunchKernelGGL((group_kernel<T, kBlock, kHeld, kSmall>), dim3(unsigned(groups)), dim3(kBlock), 0,
                     s, a);
  return hipGetLastError();
}

// Blocks of 256 threads for a group of up to 256 candidates, where there is a group for
// every unit at least or hardly anything to rank; else of 1024, four of which rank one
// candidate (13 groups of 192: 6.8 us, 8.9 with 256; of 12: 5.0 and 4.4; 1,024 groups of
// 128: 20.5 and 8.9).
bool narrow(int candidates, int groups) {
  return candidates <= 256 && (candidates <= 64 || groups > 256);
}

template <class T>
hipError_t select(BeamArgs a, const Plan& p, int groups, hipStream_t s) {
  const int64_t each = p.small ? a.cols : a.lists * a.width;
  a.per_each = uint32_t(((uint64_t(1) << 32) + each - 1) / each);
  if (p.small) {
    if (narrow(a.cols * a.beams, groups)) return group<T, 256, 1, true>(a, groups, s);
    if (a.cols * a.beams <= 1024) return group<T, 1024, 1, true>(a, groups, s);
    return group<T, 1024, 4, true>(a, groups, s);
  }
  const size_t lists = size_t(kWaves) * room_of(a.width) * sizeof(Entry);
  const int64_t blocks = (int64_t(a.rows) * a.strips + kWaves - 1) / kWaves;
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {
    hipLaunchKernelGGL((strips_kernel<T>), dim3(unsigned(std::min(blocks - b, kMostBlocks))),
                       dim3(kThreads), lists, s, a, b * kWaves);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (a.lists < a.strips) {
    hipLaunchKernelGGL(join_lists_kernel, dim3(unsigned((a.rows + kWaves - 1) / kWaves)),
                       dim3(kThreads), lists, s, a);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  const int n = a.beams * a.lists * a.width;
  if (narrow(n, groups)) return group<float, 256, 1, false>(a, groups, s);
  if (n <= 1024) return group<float, 1024, 1, false>(a, groups, s);
  if (n <= 4096) return group<float, 1024, 4, false>(a, groups, s);
  return group<float, 1024, kMostHeld, false>(a, groups, s);
}

size_t entry_bytes(const sched_beam_desc& d, const Plan& p) {
  return (size_t(d.logits.rows) * p.strips * d.width * sizeof(Entry) + 255) & ~size_t(255);
}

// --- states follow ----------------------------------------------------------------

struct StateArgs {
  char* data;
  int64_t rows, outer_stride, slot_stride, row_stride;
  const int32_t *parents, *lengths;
  uint32_t units, per_unit;  // of a row; ceil(2^32 / units)
  int32_t beams, shift;      // a block has 2^shift places
  int32_t first_slot;        // parents count from the slot so many before data's
};
typedef uint32_t Quad __attribute__((ext_vector_type(4)));
constexpr int kStateHeld = 16;  // units that a thread moves at once

// A block moves some places (units of 16 bytes or less) of all slots of a group:
// it reads every slot that is followed before it writes any, so that slots may
// follow one another in a circle without a second copy of the states.  Bound by the
// moved rows' bytes, read and written once (141 MB of 256 slots' states: 55 us, 5.1
// TB/s; 16 to a thread, all under way at once).
template <class U>
__global__ __launch_bounds__(kThreads) void reorder_kernel(StateArgs a, int64_t chunk0) {
  __shared__ int from[kMostWidth], to[kMostWidth], length[kMostWidth], moves;
  const int t = int(threadIdx.x), size = 1 << a.shift;
  const int64_t slot0 = int64_t(blockIdx.y) * a.beams;
  const int64_t begin = (chunk0 + blockIdx.x) << a.shift;  // the chunk's first place
  const int64_t row = begin >> 32 ? begin / a.units : uint32_t(begin) / a.units;
  const uint32_t unit = uint32_t(begin - row * a.units);
  char* const data = a.data + blockIdx.z * a.outer_stride + slot0 * a.slot_stride + row * a.row_stride;
  if (t == 0) moves = 0;
  __syncthreads();
  if (t < a.beams) {
    const int64_t p = int64_t(a.parents[slot0 + t]) - a.first_slot;
    if (p >= slot0 && p < slot0 + a.beams && p != slot0 + t) {
      const int64_t rows = a.lengths ? min(a.rows, int64_t(max(a.lengths[p], 0))) : a.rows;
      if (rows * a.units > begin) {
        const int m = atomicAdd(&moves, 1);  // in any order: each is a place of its own
        from[m] = int(p - slot0);
        to[m] = t;
        length[m] = int(min(rows * a.units - begin, int64_t(size)));
      }
    }
  }
  __syncthreads();
  const int work = moves << a.shift;
  if (work == 0) return;
  U held[kStateHeld];
  auto place = [&](int i, int slot) {
    // Less than 2 rows where rows have 4,096 units or more, else less than 2^13 units.
    const uint32_t at = unit + uint32_t(i & (size - 1));
    const uint32_t r = a.units >= 4096 ? at >= a.units : a.per_unit ? __umulhi(at, a.per_unit) : at;
    return reinterpret_cast<U*>(data + slot * a.slot_stride + int64_t(r) * a.row_stride) +
           (at - r * a.units);
  };
#pragma unroll
  for (int n = 0; n < kStateHeld; ++n) {
    const int i = n * kThreads + t, m = i >> a.shift;
    if (i < work && (i & (size - 1)) < length[m]) held[n] = *place(i, from[m]);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what is read is here
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kStateHeld; ++n) {
    const int i = n * kThreads + t, m = i >> a.shift;
    if (i < work && (i & (size - 1)) < length[m]) *place(i, to[m]) = held[n];
  }
}

template <class U>
hipError_t reorder(const sched_states& x, StateArgs a, hipStream_t s) {
  a.units = uint32_t(x.row_bytes / int64_t(sizeof(U)));
  a.per_unit = uint32_t(((uint64_t(1) << 32) + a.units - 1) / a.units);
  a.shift = 12;
  while ((kStateHeld * kThreads >> a.shift) < a.beams) --a.shift;
  const int64_t chunks = (int64_t(a.units) * x.rows + (1 << a.shift) - 1) >> a.shift;
  const int64_t groups = x.slots / a.beams;
  constexpr int64_t kMostY = 65535;  // of a grid's second and third side
  const int32_t* const parents = a.parents;
  const int32_t* const lengths = a.lengths;
  for (int64_t z = 0; z < x.outer; z += kMostY)
    for (int64_t y = 0; y < groups; y += kMostY)
      for (int64_t c = 0; c < chunks; c += kMostBlocks) {
        // A part's groups are counted from its first.
        a.data = static_cast<char*>(x.data) + z * x.outer_stride + y * a.beams * x.slot_stride;
        a.parents = parents + y * a.beams;
        a.lengths = lengths ? lengths + y * a.beams : nullptr;
        a.first_slot = int32_t(y * a.beams);
        const dim3 grid(unsigned(std::min(chunks - c, kMostBlocks)), unsigned(std::min(groups - y, kMostY)),
                        unsigned(std::min(x.outer - z, kMostY)));
        hipLaunchKernelGGL((reorder_kernel<U>), grid, dim3(kThreads), 0, s, a, c);
        if (const hipError_t e = hipGetLastError()) return e;
      }
  return hipSuccess;
}

}  // namespace

size_t beam_bytes(const sched_beam_desc& d) {
  if (d.logits.rows == 0) return 0;
  const Plan p = plan_of(d);
  return p.small ? 0 : entry_bytes(d, p) + size_t(d.logits.rows) * p.strips * sizeof(float2);
}

hipError_t launch_beam_select(const sched_beam_desc& d, void* ws, hipStream_t s) {
  if (d.n_groups == 0) return hipSuccess;
  const Plan p = plan_of(d);
  BeamArgs a = {};
  a.logits = static_cast<const char*>(d.logits.data);
  a.stride = d.logits.stride;
  a.rows = int32_t(d.logits.rows);
  a.cols = int32_t(d.logits.cols);
  a.beams = d.beams;
  a.width = d.width;
  a.strips = p.strips;
  a.strip_chunks = p.strip_chunks;
  a.lists = p.lists;
  a.stay = d.stay;
  a.scores = d.scores;
  a.last = {d.last.data, d.last.bits == 64};
  a.end_token = d.end_token;
  a.per_temperature = 1. / double(d.temperature);
  a.factor = float(1.4426950408889634 / double(d.temperature));
  if (!p.small) {
    a.entries = static_cast<Entry*>(ws);
    a.sums = reinterpret_cast<float2*>(static_cast<char*>(ws) + entry_bytes(d, p));
  }
  a.new_scores = d.new_scores;
  a.parents = d.parents;
  a.tokens = d.tokens;
  a.wide_tokens = d.token_bits == 64;
  if (d.logits.dtype == SCHED_F32) return select<float>(a, p, d.n_groups, s);
  if (d.logits.dtype == SCHED_F16) return select<f16>(a, p, d.n_groups, s);
  return select<bf16>(a, p, d.n_groups, s);
}

hipError_t launch_beam_reorder(const sched_states& x, const int32_t* parents, const int32_t* lengths,
                               int32_t beams, hipStream_t s) {
  if (x.outer == 0 || x.slots == 0 || x.rows == 0 || x.row_bytes == 0 || beams == 1) return hipSuccess;
  StateArgs a = {};
  a.data = static_cast<char*>(x.data);
  a.rows = x.rows;
  a.outer_stride = x.outer_stride;
  a.slot_stride = x.slot_stride;
  a.row_stride = x.row_stride;
  a.parents = parents;
  a.lengths = lengths;
  a.beams = beams;
  const uint64_t all = reinterpret_cast<uintptr_t>(x.data) | uint64_t(x.row_bytes) |
                       uint64_t(x.outer > 1 ? x.outer_stride : 0) | uint64_t(x.slot_stride) |
                       uint64_t(x.rows > 1 ? x.row_stride : 0);
  if (all % 16 == 0) return reorder<Quad>(x, a, s);
  if (all % 8 == 0) return reorder<uint64_t>(x, a, s);
  if (all % 4 == 0) return reorder<uint32_t>(x, a, s);
  if (all % 2 == 0) return reorder<uint16_t>(x, a, s);
  return reorder<uint8_t>(x, a, s);
}

}  // namespace policy
