// beam.hip -- beam search: the best continuations of each group's beams, and the
// beams' states following them.
//
// Logits are read once.  Every wave takes a strip of a row and keeps its `width`
// best logits (a continuation that is not among its strip's best is not among
// the group's) and what the sum of powers needs; a block per group then gives
// the strips' best their scores and takes the best of those.  Bound by the
// logits' bytes where rows are long.
#include <hip/hip_runtime.h>

#include <algorithm>

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
constexpr int kRoom = 10 * kMostWidth;            // of a wave's list
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

__device__ __forceinline__ int lanes_before(uint64_t mask) {
  const int lane = int(threadIdx.x) % kWave;
  return __popcll(mask & ((uint64_t(1) << lane) - 1));
}
// What a wave's lanes have written to LDS is read by its other lanes from here on.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

struct Entry {
  uint32_t order, token;
};

// A wave's list of candidates in LDS.  cut() leaves the k best (greater orders,
// of equal ones lower tokens), in no order.
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
    constexpr int kHeld = kRoom / kWave;
    const int lane = int(threadIdx.x) % kWave;
    wave_order();
    Entry e[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      e[i] = {0, ~0u};
      if (i * kWave + lane < n) e[i] = at[i * kWave + lane];
    }
    const int rounds = (n + kWave - 1) / kWave;
    auto count = [&](auto in) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (i < rounds) c += __popcll(__ballot(in(e[i])));
      return c;
    };
    // The greatest order that k entries have or pass, bit by bit.
    uint32_t v = 0;
    int reach = n;
#pragma unroll 1
    for (int bit = 31; bit >= 0 && reach != k; --bit) {
      const uint32_t t = v | 1u << bit;
      const int c = count([&](const Entry& x) { return x.order >= t; });
      if (c >= k) {
        v = t;
        reach = c;
      }
    }
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
    n = 0;
    wave_order();
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i < rounds)
        add(e[i].order > v || (e[i].order == v && e[i].token <= upto), e[i].order, e[i].token);
    wave_order();
    least = v;
  }
};

struct BeamArgs {
  const char* logits;
  int64_t stride;
  int32_t rows, cols, beams, width, strips, strip_chunks, stay, lists;  // lists: of a row
  const float* scores;
  Tokens last;
  int64_t end_token;
  float temperature, factor;  // log2(e) / temperature
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

template <class T>
__device__ __forceinline__ void eight_logits(const T* row, int64_t at, int64_t end, float (&x)[8]) {
  if (at + 8 <= end) {
#pragma unroll
    for (int i = 0; i < 8; i += Vec<T>::kN) {
      const auto v = load16(row + at + i);
#pragma unroll
      for (int e = 0; e < Vec<T>::kN; ++e) x[i + e] = float(v[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = at + e < end ? float(row[at + e]) : -INFINITY;
  }
}

// --- strips of rows -----------------------------------------------------------

template <class T>
__global__ __launch_bounds__(kThreads) void strips_kernel(BeamArgs a, int64_t first) {
  __shared__ Entry lists[kWaves][kRoom];
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave, k = a.width;
  const int64_t unit = first + int64_t(blockIdx.x) * kWaves + wave;
  if (unit >= int64_t(a.rows) * a.strips) return;
  const int64_t row = unit / a.strips;
  const int strip = int(unit % a.strips);
  if (finished(a, row) || !present(a, row)) return;  // its logits do not matter
  const T* const logits = reinterpret_cast<const T*>(a.logits) + row * a.stride;
  const int64_t begin = int64_t(strip) * a.strip_chunks * kChunk;
  const int64_t end = min(begin + int64_t(a.strip_chunks) * kChunk, int64_t(a.cols));
  List list = {lists[wave], 0, 0};
  float most = -INFINITY, sum = 0.f;  // of this lane's logits
  for (int64_t at = begin; at < end; at += kChunk) {
    float x[kRounds][8];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) eight_logits(logits, at + r * 8 * kWave + 8 * lane, end, x[r]);
    // Powers relative to the largest so far; NaN and +inf end in a sum of NaN.
    float up = most;
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) up = fmaxf(up, x[r][e]);
    const float from = up == -INFINITY ? 0.f : up;
    sum = most == -INFINITY ? sum : sum * pow2((most - from) * a.factor);  // 0, or NaN met before
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += pow2((x[r][e] - from) * a.factor);
    most = up;
    // The greatest order of each lane's eight.
    uint32_t top[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      float m = x[r][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) m = fmaxf(m, x[r][e]);
      top[r] = m > -INFINITY ? order_of(m) : 0u;
    }
    uint32_t over = max(list.least, kLeast - 1);  // candidates pass it
    int passing = 0;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) passing += __popcll(__ballot(top[r] > over));
    if (!passing) continue;
    if (list.n + 8 * passing > kRoom) list.cut(k);
    uint32_t equal = 0;  // orders of which the first k are taken too
    if (passing > k) {
      // The k-th greatest of the eights' greatest: k logits have its order or
      // pass it, and less than 8 k pass it.
      uint32_t v = 0;
#pragma unroll 1
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t t = v | 1u << bit;
        int c = 0;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) c += __popcll(__ballot(top[r] >= t));
        if (c >= k) v = t;
      }
      over = v;
      equal = v;
    }
    int taken = 0;
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (!__ballot(top[r] > over || (equal && top[r] == equal))) continue;
      const uint32_t token = uint32_t(at + r * 8 * kWave + 8 * lane);
      uint32_t order[8];
      uint64_t same[8];
      int before = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        order[e] = x[r][e] > -INFINITY ? order_of(x[r][e]) : 0u;
        list.add(order[e] > over, order[e], token + e);
        same[e] = __ballot(equal && order[e] == equal);
        before += lanes_before(same[e]);
      }
      if (!equal) continue;
      // The first of those that are equal, in the tokens' order.
      int nth = taken + before;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool mine = order[e] == equal;
        list.add(mine && nth < k, order[e], token + e);
        nth += mine;
        taken += __popcll(same[e]);
      }
    }
    if (list.n > k && (equal || list.n > 2 * k + kWave)) list.cut(k);
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
  __shared__ Entry lists[kWaves][kRoom];
  const int lane = int(threadIdx.x) % kWave, wave = int(threadIdx.x) / kWave, k = a.width;
  const int64_t row = int64_t(blockIdx.x) * kWaves + wave;
  if (row >= a.rows || finished(a, row) || !present(a, row)) return;
  List list = {lists[wave], 0, 0};
  Entry* const in = a.entries + row * a.strips * k;
  const int n = a.strips * k;
  for (int i = 0; i < n; i += kWave) {
    Entry e = {0, ~0u};
    if (i + lane < n) e = in[i + lane];
    list.add(e.order >= max(list.least, kLeast), e.order, e.token);
    if (list.n + kWave > kRoom) list.cut(k);
  }
  list.cut(k);
  wave_order();
  for (int i = lane; i < k; i += kWave) in[i] = i < list.n ? list.at[i] : Entry{0, ~0u};
}

// --- a group's best -------------------------------------------------------------

// Sums over a block of one number per thread's wave: waves count by ballots.
struct Counter {
  int (*room)[kWaves];
  int turn;
  __device__ __forceinline__ int total(int wave_count) {
    const int wave = int(threadIdx.x) / kWave;
    turn ^= 1;  // the last total may still be read
    if (int(threadIdx.x) % kWave == 0) room[turn][wave] = wave_count;
    __syncthreads();
    int c = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) c += room[turn][w];
    return c;
  }
};

struct Best {
  uint64_t score[kMostWidth];
  uint32_t place[kMostWidth];  // beam and token
};

// A block takes a group.  kSmall: the group's logits themselves (kHeld kThreads at
// most); else the strips' lists.
template <class T, int kHeld, bool kSmall>
__global__ __launch_bounds__(kThreads) void group_kernel(BeamArgs a) {
  __shared__ double base[kMostWidth];  // of a beam: what is added to logit / temperature
  __shared__ int counts[2][kWaves], found;
  __shared__ Best best, sorted;
  __shared__ int first[kMostWidth], used[kMostWidth];
  const int group = int(blockIdx.x), t = int(threadIdx.x), lane = t % kWave;
  const int64_t row0 = int64_t(group) * a.beams;
  const int k = a.width;

  // Every beam's base: score - log of the sum of powers; NaN where there is none.
  const int per_row = kSmall ? a.cols : a.strips;
  int lanes = 1;
  while (lanes < per_row && lanes < kWave) lanes *= 2;
  for (int b = t / lanes; b < (a.beams + kThreads / lanes - 1) / (kThreads / lanes) * (kThreads / lanes);
       b += kThreads / lanes) {
    const int64_t row = row0 + b;
    const bool live = b < a.beams && present(a, row) && !finished(a, row);
    float most = -INFINITY, sum = 0.f;
    auto power = [&](float x, float from) { return pow2((x - from) * a.factor); };
    if (live) {
      for (int i = t % lanes; i < per_row; i += lanes) {
        float x, s = 1.f;
        if (kSmall) x = float((reinterpret_cast<const T*>(a.logits) + row * a.stride)[i]);
        else {
          const float2 p = a.sums[row * a.strips + i];
          x = p.x;
          s = p.y;
        }
        if (kSmall ? x == -INFINITY : s == 0.f) continue;
        const float up = fmaxf(most, x);
        sum = (most == -INFINITY ? sum : sum * power(most, up)) + s * power(x, up);
        most = up;
      }
    }
    for (int d = lanes / 2; d; d >>= 1) {
      const float x = __shfl_xor(most, d), s = __shfl_xor(sum, d), up = fmaxf(most, x);
      sum = up == -INFINITY ? sum + s
                            : (most == -INFINITY ? sum : sum * power(most, up)) +
                                  (x == -INFINITY ? s : s * power(x, up));
      most = up;
    }
    if (b < a.beams && t % lanes == 0) {
      const double none = __longlong_as_double(0x7ff8000000000000LL);
      const bool ok = live && sum > 0.f && sum < INFINITY && fabsf(most) < INFINITY;
      base[b] = ok ? double(a.scores[row]) - double(most) / double(a.temperature) - log(double(sum))
                   : none;
    }
  }
  if (t == 0) found = 0;
  if (t < kMostWidth) {
    used[t] = 0;
    best.score[t] = sorted.score[t] = 0;
  }
  __syncthreads();

  // The candidates: score's order and place (beam, then token).
  uint64_t score[kHeld];
  uint32_t place[kHeld];
  const int each = kSmall ? a.cols : a.lists * k, n = a.beams * each;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = i * kThreads + t;
    score[i] = 0;
    place[i] = ~0u;
    if (c >= n) continue;
    const int b = c / each, r = c % each;
    const int64_t row = row0 + b;
    if (finished(a, row)) {  // its one candidate
      if (r == 0 && present(a, row)) {
        score[i] = order_of(double(a.scores[row]));
        place[i] = uint32_t(b) << kTokenBits;
      }
      continue;
    }
    float x = -INFINITY;
    uint32_t token = uint32_t(r);
    if (kSmall) {
      x = float((reinterpret_cast<const T*>(a.logits) + row * a.stride)[r]);
    } else if (present(a, row)) {
      const Entry e = a.entries[row * a.strips * k + r];
      if (e.order >= kLeast) {
        x = of_order(e.order);
        token = e.token;
      }
    }
    const double s = base[b] + double(x) / double(a.temperature);
    if (s > -INFINITY && s < INFINITY) {
      score[i] = order_of(s);
      place[i] = uint32_t(b) << kTokenBits | token;
    }
  }

  // The k best: the greatest order that k of them have or pass, and of those that
  // have it the first places.
  Counter counter = {counts, 0};
  auto count = [&](auto in) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i * kThreads < n) c += __popcll(__ballot(in(score[i], place[i])));
    return counter.total(c);
  };
  const int there = count([&](uint64_t s, uint32_t) { return s > 0; });
  uint64_t v = 1;
  uint32_t upto = ~0u;
  if (there > k) {
    int reach = there;
    v = 0;
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
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t bound = below | 1u << bit;
        if (over + count([&](uint64_t s, uint32_t p) { return s == v && p < bound; }) < k)
          below = bound;
      }
      upto = below;
    }
  }
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (score[i] > v || (score[i] == v && place[i] <= upto)) {
      const int at = atomicAdd(&found, 1);  // in any order: they are sorted next
      best.score[at] = score[i];
      best.place[at] = place[i];
    }
  __syncthreads();
  const int got = min(there, k);
  if (t < got) {
    int rank = 0;
    const uint64_t s = best.score[t];
    const uint32_t p = best.place[t];
    for (int i = 0; i < got; ++i)
      rank += best.score[i] > s || (best.score[i] == s && best.place[i] < p);
    sorted.score[rank] = s;
    sorted.place[rank] = p;
  }
  __syncthreads();

  int slot = t;
  if (a.stay) {
    const int beam = t < got ? int(sorted.place[t] >> kTokenBits) : -1;
    bool mine = t < got;  // the beam's best continuation
    for (int i = 0; i < min(t, got) && mine; ++i)
      mine = int(sorted.place[i] >> kTokenBits) != beam;
    if (mine) used[beam] = 1;
    if (t < k) first[t] = mine;
    __syncthreads();
    slot = beam;
    if (t < k && !mine) {
      int nth = 0;  // of those without a slot
      for (int i = 0; i < t; ++i) nth += !first[i];
      slot = 0;
      for (int free = -1;; ++slot) {
        free += !used[slot];
        if (free == nth) break;
      }
    }
  }
  if (t >= k) return;
  const int64_t out = int64_t(group) * k + slot;
  int64_t token = -1;
  int parent = -1;
  float new_score = -INFINITY;
  if (t < got) {
    const uint32_t p = sorted.place[t];
    parent = int(row0 + (p >> kTokenBits));
    token = finished(a, parent) ? a.end_token : int64_t(p & ((1u << kTokenBits) - 1));
    new_score = float(of_order(sorted.score[t]));
  }
  a.new_scores[out] = new_score;
  a.parents[out] = parent;
  if (a.wide_tokens) static_cast<int64_t*>(a.tokens)[out] = token;
  else static_cast<int32_t*>(a.tokens)[out] = int32_t(token);
}

struct Plan {
  int strips, strip_chunks, lists;
  bool small;
};
constexpr int kMostHeld = 64;  // candidates of a thread

Plan plan_of(const sched_beam_desc& d) {
  Plan p = {};
  const int64_t cols = d.logits.cols, rows = d.logits.rows;
  p.small = cols <= 4 * kWave && cols * d.beams <= 16 * kThreads;
  const int64_t chunks = (cols + kChunk - 1) / kChunk;
  // Some 4096 waves, as far as rows are long enough.
  const int64_t want = std::min<int64_t>(
      {std::max<int64_t>(1, 4096 / std::max<int64_t>(rows, 1)), chunks, int64_t(kMostStrips)});
  p.strip_chunks = int((chunks + want - 1) / want);
  p.strips = int((chunks + p.strip_chunks - 1) / p.strip_chunks);
  p.lists = int64_t(d.beams) * p.strips * d.width > kMostHeld * kThreads ? 1 : p.strips;
  return p;
}

template <class T, int kHeld, bool kSmall>
hipError_t group(const BeamArgs& a, int groups, hipStream_t s) {
  hipLaunchKernelGGL((group_kernel<T, kHeld, kSmall>), dim3(unsigned(groups)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T>
hipError_t select(const BeamArgs& a, const Plan& p, int groups, hipStream_t s) {
  if (p.small) {
    if (a.cols * a.beams <= 4 * kThreads) return group<T, 4, true>(a, groups, s);
    return group<T, 16, true>(a, groups, s);
  }
  const int64_t blocks = (int64_t(a.rows) * a.strips + kWaves - 1) / kWaves;
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {
    hipLaunchKernelGGL((strips_kernel<T>), dim3(unsigned(std::min(blocks - b, kMostBlocks))),
                       dim3(kThreads), 0, s, a, b * kWaves);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (a.lists < a.strips) {
    hipLaunchKernelGGL(join_lists_kernel, dim3(unsigned((a.rows + kWaves - 1) / kWaves)),
                       dim3(kThreads), 0, s, a);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  const int n = a.beams * a.lists * a.width;
  if (n <= 4 * kThreads) return group<float, 4, false>(a, groups, s);
  if (n <= 16 * kThreads) return group<float, 16, false>(a, groups, s);
  return group<float, kMostHeld, false>(a, groups, s);
}

size_t entry_bytes(const sched_beam_desc& d, const Plan& p) {
  return (size_t(d.logits.rows) * p.strips * d.width * sizeof(Entry) + 255) & ~size_t(255);
}

// --- states follow ----------------------------------------------------------------

struct StateArgs {
  char* data;
  int64_t units, rows;  // of a row, of a slot
  int64_t outer_stride, slot_stride, row_stride;
  const int32_t *parents, *lengths;
  int32_t beams, groups, shift;  // a block has 2^shift places
  int64_t chunks;
};
typedef uint32_t Quad __attribute__((ext_vector_type(4)));
constexpr int kStateHeld = 16;  // units that a thread moves at once

// A block moves some places (units of 16 bytes or less) of all slots of a group:
// it reads every slot that is followed before it writes any.
template <class U>
__global__ __launch_bounds__(kThreads) void reorder_kernel(StateArgs a, int64_t first) {
  __shared__ int from[kMostWidth], to[kMostWidth], length[kMostWidth], moves;
  const int64_t block = first + int64_t(blockIdx.x);
  const int64_t chunk = block % a.chunks, rest = block / a.chunks;
  const int64_t slot0 = rest % a.groups * a.beams;
  const int64_t begin = chunk << a.shift, row = begin / a.units;  // the chunk's first place
  const uint32_t units = uint32_t(a.units), unit = uint32_t(begin - row * a.units);
  char* const data = a.data + rest / a.groups * a.outer_stride + slot0 * a.slot_stride +
                     row * a.row_stride;
  const int t = int(threadIdx.x), size = 1 << a.shift;
  if (t == 0) moves = 0;
  __syncthreads();
  if (t < a.beams) {
    const int64_t p = a.parents[slot0 + t];
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
    const uint32_t at = unit + uint32_t(i & (size - 1));
    return reinterpret_cast<U*>(data + slot * a.slot_stride + int64_t(at / units) * a.row_stride) +
           at % units;
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
  a.units = x.row_bytes / int64_t(sizeof(U));
  a.shift = 12;
  while ((kStateHeld * kThreads >> a.shift) < a.beams) --a.shift;
  a.chunks = (a.units * x.rows + (1 << a.shift) - 1) >> a.shift;
  const int64_t blocks = a.chunks * a.groups * x.outer;
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {
    hipLaunchKernelGGL((reorder_kernel<U>), dim3(unsigned(std::min(blocks - b, kMostBlocks))),
                       dim3(kThreads), 0, s, a, b);
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
  a.temperature = d.temperature;
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
  a.groups = int32_t(x.slots / beams);
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
