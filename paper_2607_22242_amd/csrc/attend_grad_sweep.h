// attend_grad_sweep.h -- what the backward kernels of attention share: a wave's
// keys against tiles of query rows, and its query rows against tiles of keys.
#pragma once
#include "attend.h"

namespace policy {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;          // rows of a tile that is walked over
constexpr int kKeysOfBlock = 64;   // keys that a block holds for dK and dV
constexpr int kRowsOfBlock = 128;  // query rows that a block holds for dQ, 32 of each wave

// Keys up to one.
struct UpTo {
  int last;
  __device__ __forceinline__ bool operator()(int j) const { return j <= last; }
};

// A tile of query rows: where row 0 of it lies, counted in queries and in rows
// behind the query's first head.
struct RowTile {
  int r0, query, rest;
};
__device__ __forceinline__ RowTile row_tile(const AttendArgs& a, int r0) {
  return {r0, r0 / a.group, r0 % a.group};
}
__device__ __forceinline__ void retreat(const AttendArgs& a, RowTile& t) {
  t.r0 -= kTile;
  t.query -= kTile / a.group;
  t.rest -= kTile % a.group;
  if (t.rest < 0) {
    t.rest += a.group;
    --t.query;
  }
}

// Rows of a tile from one to another.
struct RowSpan {
  int from, upto;
};

struct Stats {
  float lse2[kTile], delta[kTile];
};

// Tiles of query rows of one sequence and the heads of one key head: Q, dO and
// the rows' statistics.
template <class T, int D>
struct RowTiles {
  typedef Fill<T, D, kTile, kThreads> F;
  uint32_t q_lane, o_lane;

  __device__ __forceinline__ RowTiles(const AttendArgs& a) {
    const F fill(a.dim);
    auto lane = [&](const HeadsView& x) {
      return uint32_t(fill.row / a.group * x.row + fill.row % a.group * x.head + fill.d) * 2;
    };
    q_lane = lane(a.q);
    o_lane = lane(a.d_out);
  }
  // Rows behind the last repeat it.
  __device__ __forceinline__ void fetch(const AttendArgs& a, const Seq& s, int kv, int rows,
                                        const RowTile& t, T* q_tile, T* o_tile,
                                        Stats* stats) const {
    const int most = t.rest + rows - 1 - t.r0;
    auto row_of = [&](int i) -> QueryRow {
      const int x = min(t.rest + i, most), y = int(__umulhi(uint32_t(x), a.per_group));
      const int q = a.per_group ? y : x;  // 0: groups of one
      return {t.query + q, kv * a.group + x - q * a.group};
    };
    if (a.near_q && t.r0 + kTile <= rows) {
      const int64_t row = int64_t(s.q0) + t.query;
      const int step = F::kStep / a.group;
#pragma unroll
      for (int p = 0; p < F::kRounds; ++p) {
        const T* q = head_row<T>(a.q, row + p * step, kv * a.group);
        const T* o = head_row<T>(a.d_out, row + p * step, kv * a.group);
        to_lds(reinterpret_cast<const char*>(q), q_lane, F::at(q_tile, p));
        to_lds(reinterpret_cast<const char*>(o), o_lane, F::at(o_tile, p));
      }
    } else {
      const F fill(a.dim);
#pragma unroll
      for (int p = 0; p < F::kRounds; ++p) {
        const QueryRow r = row_of(fill.row + p * F::kStep);
        const int64_t row = int64_t(s.q0) + r.query;
        to_lds(reinterpret_cast<const char*>(head_row<T>(a.q, row, r.head) + fill.d), 0,
               F::at(q_tile, p));
        to_lds(reinterpret_cast<const char*>(head_row<T>(a.d_out, row, r.head) + fill.d), 0,
               F::at(o_tile, p));
      }
    }
    const int wave = wave_id();
    if (wave < 2) {
      int lane = int(threadIdx.x) % kWave;
      asm volatile("" : "+v"(lane));
      const QueryRow r = row_of(lane);
      const int64_t n = int64_t(r.head) * a.q_rows + s.q0 + r.query;
      typedef __attribute__((address_space(1))) const void Global;
      typedef __attribute__((address_space(3))) void Lds;
      __builtin_amdgcn_global_load_lds((Global*)((wave ? a.delta : a.lse2) + n),
                                       (Lds*)(wave ? stats->delta : stats->lse2), 4, 0, 0);
    }
  }
};

// 32 keys of a wave (lane l has key l % 32) against the rows it is given: the
// lanes' columns are keys, their values run along the query rows.  The sums
// (D / 32 tiles each) and the keys and values take most of the 256 registers
// that leave two waves on a unit; of 128 elements the values' upper half stays
// in LDS for that.
template <class T, int D, bool kFine = false>
struct KeySweep {
  static constexpr int kHeld = D == 128 ? D / 32 : D / 16;  // pieces of the values in registers
  typename Frag<T>::type k[D / 16], v[kHeld];
  Acc dk[D / 32], dv[D / 32];
  int up;  // f16: dS is held 2^up times

  // Rows part .. part + 31 of a tile; the lane's key is seen by the rows of the tile
  // that seen() names (`whole`: all of the wave's are by all).
  template <class Seen>
  __device__ __forceinline__ void add(const T* q_tile, const T* o_tile, const Stats& stats,
                                      const Rows<T, 64>& rest, int wave_row, int part,
                                      const Seen& seen, bool whole, float c,
                                      const Places<D>& places) {
    const Rows<T, D> qs = {q_tile, places.fresh()}, os = {o_tile, qs.places};
    typedef float Four __attribute__((ext_vector_type(4)));
    const int h4 = int(threadIdx.x) % kWave / 32 * 4;
    Acc x = Acc(0.f), y;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const Four d = *reinterpret_cast<const Four*>(&stats.delta[part + 2 * i + h4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[i + e] = d[e];
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) x = product(qs.along(part, i), k[i], x);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      y = product(os.along(part, i), i < kHeld ? v[i] : rest.along(wave_row, i - kHeld), y);
    if (!whole) {
      const RowSpan s = seen();
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = part + c_row(i);
        if (r < s.from || r > s.upto) x[i] = -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const Four l = *reinterpret_cast<const Four*>(&stats.lse2[part + 2 * i + h4]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[i + e] = pow2(__builtin_fmaf(x[i + e], c, -l[e]));
        y[i + e] *= x[i + e];
        if (kShort<T>) y[i + e] = __builtin_ldexpf(y[i + e], up);
      }
    }
    if (kShort<T> && __any(passes(y))) {
      const int e = fit(y);
      up -= e;
      shift(dk, -e);
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const auto pb = narrow<T>(x, p), db = narrow<T>(y, p);
#pragma unroll
      for (int d = 0; d < D / 32; ++d) dv[d] = product(os.across(part + 16 * p, d), pb, dv[d]);
#pragma unroll
      for (int d = 0; d < D / 32; ++d) dk[d] = product(qs.across(part + 16 * p, d), db, dk[d]);
      if (kFine) {
        const auto p_rest = rest_of<T>(x, p, pb), d_rest = rest_of<T>(y, p, db);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) dv[d] = product(os.across(part + 16 * p, d), p_rest, dv[d]);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) dk[d] = product(qs.across(part + 16 * p, d), d_rest, dk[d]);
      }
    }
  }

  // A wave's sums to and from another's, through two buffers.
  __device__ __forceinline__ void hand(float* a, float* b) const {
    const int lane = int(threadIdx.x) % kWave;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        a[(d * 16 + i) * kWave + lane] = dk[d][i];
        b[(d * 16 + i) * kWave + lane] = dv[d][i];
      }
  }
  __device__ __forceinline__ void take(const float* a, const float* b) {
    const int lane = int(threadIdx.x) % kWave;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        dk[d][i] += a[(d * 16 + i) * kWave + lane];
        dv[d][i] += b[(d * 16 + i) * kWave + lane];
      }
  }
};

// Where few keys would leave the card idle, a block's rows are shared by `parts`
// blocks, whose sums, in 32 bits, are added after them in one order.
struct KeyParts {
  float *dk, *dv;  // parts x kv_heads x k_rows x D
  int parts;
};
template <int D>
__device__ __forceinline__ int64_t key_part(const AttendArgs& a, int part, int kv, int64_t row) {
  return ((int64_t(part) * (a.q_heads / a.group) + kv) * a.k_rows + row) * D;
}

// 32 query rows of a wave (lane l has row l % 32): the lanes' columns are query
// rows, their values run along the keys.
template <class T, int D, bool kFine = false>
struct RowSweep {
  typename Frag<T>::type q[D / 16], o[D / 16];
  Acc dq[D / 32];
  float lse2, delta;
  int up;  // f16: the powers, and dS, are held 2^up times, which lse2 has in it

  // Adds the keys of a tile, the first of them key j0; the lane's row sees key j if
  // sees(j) (`whole`: all rows of the wave see all).
  template <class Sees>
  __device__ __forceinline__ void add(const T* k_tile, const T* v_tile, int j0, const Sees& sees,
                                      bool whole, float c, const Places<D>& places) {
    const Rows<T, D> ks = {k_tile, places.fresh()}, vs = {v_tile, ks.places};
#pragma unroll
    for (int t = 0; t < kTile / 32; ++t) {
      Acc x = Acc(0.f), y = Acc(delta);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) x = product(ks.along(32 * t, i), q[i], x);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) y = product(vs.along(32 * t, i), o[i], y);
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!sees(j0 + 32 * t + c_row(i))) x[i] = -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] *= pow2(__builtin_fmaf(x[i], c, -lse2));
      if (kShort<T> && __any(passes(y))) {
        const int e = fit(y);
        up -= e;
        lse2 += float(e);
        shift(dq, -e);
      }
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const auto b = narrow<T>(y, p);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) dq[d] = product(ks.across(32 * t + 16 * p, d), b, dq[d]);
        if (kFine) {
          const auto rest = rest_of<T>(y, p, b);
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
            dq[d] = product(ks.across(32 * t + 16 * p, d), rest, dq[d]);
        }
      }
    }
  }

  // Sum over a tile's keys of P_j dP_j, of this lane's half of them.
  template <class Sees>
  __device__ __forceinline__ float dots(const T* k_tile, const T* v_tile, int j0, const Sees& sees,
                                        float c, const Places<D>& places) const {
    const Rows<T, D> ks = {k_tile, places.fresh()}, vs = {v_tile, ks.places};
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < kTile / 32; ++t) {
      Acc x = Acc(0.f), y = Acc(0.f);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) x = product(ks.along(32 * t, i), q[i], x);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) y = product(vs.along(32 * t, i), o[i], y);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        // What is not seen may be no number, times a power of 0 too.
        const float d = pow2(__builtin_fmaf(x[i], c, -lse2)) * y[i];
        sum += sees(j0 + 32 * t + c_row(i)) ? d : 0.f;
      }
    }
    return sum;
  }

  // delta of rows that see keys of the first tile only, from the probabilities
  // as sum_j P_j dP_j: from the rounded out it is off by a rounding of out, which
  // with few keys is as much as all other roundings together (errors of dQ and
  // dK against exact products of 16-bit operands: 1.6 to 1.8 times before, 1.4
  // so, which is what rounding dS and the result gives).
  __device__ __forceinline__ void exact_delta(const T* k_tile, const T* v_tile, int last, float c,
                                              const Places<D>& places) {
    const float sum = dots(k_tile, v_tile, 0, UpTo{last}, c, places);
    delta = -__builtin_ldexpf(sum + __shfl_xor(sum, 32), -up);
  }
};

// Where few query rows would leave the card idle, the keys of a block's rows are
// shared by `parts` blocks in the same way.
struct RowParts {
  float* dq;  // parts x q_rows x q_heads x D
  int parts;
};
template <int D>
__device__ __forceinline__ int64_t row_part(const AttendArgs& a, int part, int64_t row, int head) {
  return ((int64_t(part) * a.q_rows + row) * a.q_heads + head) * D;
}

}  // namespace
}  // namespace policy
