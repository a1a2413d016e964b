// rotate.hip -- norms of heads and their rotation by position, and the gradient.
//
// Forward: y = R(p f) (r x o w), r = (mean x^2 + eps)^-1/2.  Backward, with g =
// R(-p f) dy: dw = sum g o (r x), u = g o w, dx = r (u - (r x) mean(u o (r x))).
// Some 8 and 16 operations per element in and out: bound by memory.  65,536 tokens
// of 32 and 8 heads of 128 in bfloat16: forward 270 us (1.34 GB, 5.0 TB/s), backward
// 470 (2.01 GB, 4.3 TB/s; a copy reaches 4.9).
//
// A head is held by a power of two of lanes, eight elements each, so that its sums
// are a few shuffles.  A block takes some rows: it forms their cosines and sines
// first, once for all heads, as an angle in 64 bits costs as much as a head's other
// work, and its lane groups go over the rows' heads.  Everything is held in 32 bits;
// what is rounded to the tensors' type is the result, once.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "policy_launch.h"
#include "tensors.h"

namespace policy {
namespace {

constexpr int kThreads = 256;
constexpr int kMostRows = 8;     // of a block
constexpr int kMostPairs = 128;  // of a head

struct Side {  // heads of one tensor: row and head strides in elements
  char* data;
  int64_t row, head;
};
template <class T>
__device__ __forceinline__ T* head_at(const Side& s, int64_t row, int head) {
  return reinterpret_cast<T*>(s.data) + row * s.row + int64_t(head) * s.head;
}

struct RotateArgs {
  Side q, k, v, q_out, k_out, v_out, d_q, d_k;  // backward: the outputs' gradients in q_out, k_out
  Tokens positions, places;
  const float *q_weight, *k_weight, *frequencies;
  float* parts;  // backward: blocks x 2 x dim
  int64_t rows, out_rows;
  int32_t dim, q_heads, kv_heads, pairs, norm, per_block;
  float eps;
};

// How a head's pairs lie: next to each other; eight lanes' elements or a
// multiple of them apart, so that a lane's partners are another lane's eight;
// any other distance, through LDS.
enum Pairs { kNext, kLanes, kAny };

typedef float Eight[8];

// Eight elements of a head as they are in memory.
template <class T>
struct Raw {
  typename Vec<T>::type part[8 / Vec<T>::kN];
};
template <class T>
__device__ __forceinline__ Raw<T> fetch(const T* at, bool on) {
  Raw<T> r;
#pragma unroll
  for (int i = 0; i < 8 / Vec<T>::kN; ++i) {
    r.part[i] = T(0);
    if (on) r.part[i] = *reinterpret_cast<const typename Vec<T>::type*>(at + i * Vec<T>::kN);
  }
  return r;
}
template <class T>
__device__ __forceinline__ void widen(const Raw<T>& r, Eight& x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = float(r.part[e / Vec<T>::kN][e % Vec<T>::kN]);
}
template <class T>
__device__ __forceinline__ void put(T* at, const Raw<T>& r) {
#pragma unroll
  for (int i = 0; i < 8 / Vec<T>::kN; ++i)
    *reinterpret_cast<typename Vec<T>::type*>(at + i * Vec<T>::kN) = r.part[i];
}
template <class T>
__device__ __forceinline__ void put(T* at, const Eight& x) {
  Raw<T> r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r.part[e / Vec<T>::kN][e % Vec<T>::kN] = T(x[e]);
  put(at, r);
}

// Cosines and sines of a block's rows; pairs behind the turned ones have those
// of no angle.
struct Angles {
  float cos[kMostRows][kMostPairs], sin[kMostRows][kMostPairs];
};
__device__ __forceinline__ void form_angles(const RotateArgs& a, int64_t row0, int rows,
                                            Angles& angles) {
  const int pairs = a.dim / 2;
  for (int i = int(threadIdx.x); i < rows * pairs; i += kThreads) {
    const int r = i / pairs, j = i % pairs;
    float c = 1.f, s = 0.f;
    if (j < a.pairs) {
      // Full turns in 64 bits: what is left of them is good to 2^-22 of a turn
      // at a position of 2^31, where 32 bits would know nothing of it.
      const double turns = double(token_at(a.positions, row0 + r)) *
                           (double(a.frequencies[j]) * 0.15915494309189535);
      sincospif(2.f * float(turns - rint(turns)), &s, &c);
    }
    angles.cos[r][j] = c;
    angles.sin[r][j] = s;
  }
}

// What a wave's lanes have written to LDS is read by its other lanes from here on.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// x turned by its row's angles (kBack: back).  `own` is the group's room in LDS.
template <int kPairs, bool kBack>
__device__ __forceinline__ void turn(const RotateArgs& a, const float* cos, const float* sin,
                                     int piece, float* own, Eight& x) {
  if (kPairs == kNext) {
    const int j = min(4 * piece, a.dim / 2 - 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float c = cos[j + e], s = kBack ? -sin[j + e] : sin[j + e];
      const float u = x[2 * e], v = x[2 * e + 1];
      if (j + e < a.pairs) {  // by no angle a neighbour's infinity would still come in
        x[2 * e] = u * c - v * s;
        x[2 * e + 1] = u * s + v * c;
      }
    }
  } else if (kPairs == kLanes) {
    const int apart = a.pairs / 8;
    const bool low = piece < apart, turned = piece < 2 * apart;
    const int to = int(threadIdx.x) % kWave + (low ? apart : turned ? -apart : 0);
    const int j = turned ? 8 * (low ? piece : piece - apart) : 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float other = __shfl(x[e], to);
      const float s = low != kBack ? -sin[j + e] : sin[j + e];
      x[e] = turned ? x[e] * cos[j + e] + other * s : x[e];
    }
  } else {
    // The group's lanes are in one wave: what they write, they can read next.
#pragma unroll
    for (int e = 0; e < 8; ++e) own[8 * piece + e] = x[e];
    wave_order();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = 8 * piece + e;
      const bool low = at < a.pairs, turned = at < 2 * a.pairs;
      const int j = turned ? (low ? at : at - a.pairs) : 0;
      const float other = own[turned ? (low ? at + a.pairs : at - a.pairs) : at];
      const float s = low != kBack ? -sin[j] : sin[j];
      x[e] = turned ? x[e] * cos[j] + other * s : x[e];
    }
    wave_order();
  }
}

template <int kLanes_>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int d = kLanes_ / 2; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

__device__ __forceinline__ void weights_of(const float* w, int piece, bool on, Eight& out) {
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = w && on ? w[8 * piece + e] : 1.f;
}

// The lane groups take the heads of the block's rows in turn, one at a time: the units'
// many waves keep enough of them on their way (65,536 tokens of 32 and 8 heads of 128:
// two heads at once take 5 % longer, four 11 %, eight 22 %).
template <class T, int kPairs, int kGroup>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a) {
  constexpr int kGroups = kThreads / kGroup;
  __shared__ Angles angles;
  __shared__ float room[kPairs == kAny ? kThreads * 8 : 1];
  const int64_t row0 = int64_t(blockIdx.x) * a.per_block;
  const int rows = int(min(int64_t(a.per_block), a.rows - row0));
  const int piece = int(threadIdx.x) % kGroup, group = int(threadIdx.x) / kGroup;
  const bool on = 8 * piece < a.dim;
  const int heads = a.q_heads + a.kv_heads, all = heads + (a.v.data ? a.kv_heads : 0);
  const int items = rows * all;
  form_angles(a, row0, rows, angles);
  Eight wq, wk;
  weights_of(a.q_weight, piece, on, wq);
  weights_of(a.k_weight, piece, on, wk);
  __syncthreads();
  for (int i0 = 0; i0 < items; i0 += kGroups) {  // of all groups: lanes meet in shuffles
    const int i = i0 + group, h = i % all, r = min(i / all, kMostRows - 1);
    const int64_t row = row0 + i / all;
    const T* const at = h < a.q_heads ? head_at<T>(a.q, row, h)
                        : h < heads   ? head_at<T>(a.k, row, h - a.q_heads)
                                      : head_at<T>(a.v, row, h - heads);
    const Raw<T> raw = fetch<T>(at + 8 * piece, on && i < items);
    Eight x;
    widen(raw, x);
    if (a.norm) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
      const float f = 1.f / sqrtf(group_sum<kGroup>(sum) / float(a.dim) + a.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * f * (h < a.q_heads ? wq[e] : wk[e]);
    }
    turn<kPairs, false>(a, angles.cos[r], angles.sin[r], piece,
                        room + (kPairs == kAny ? group * kGroup * 8 : 0), x);
    if (!on || i >= items) continue;
    if (h < a.q_heads) {
      put(head_at<T>(a.q_out, row, h) + 8 * piece, x);
      continue;
    }
    int64_t to = row;
    if (a.places.data) {
      to = token_in(a.places, row, a.out_rows);
      if (to < 0) continue;
    }
    if (h < heads) put(head_at<T>(a.k_out, to, h - a.q_heads) + 8 * piece, x);
    else put(head_at<T>(a.v_out, to, h - heads) + 8 * piece, raw);
  }
}

// A head's row and number among the block's: the lane groups take them in turn.
struct Item {
  int row, head;
};

// The gradient of one tensor's heads over a block's rows; adds to `sums` what a
// lane's elements give to the weights' gradient.
template <class T, int kPairs, int kGroup, bool kKeys>
__device__ __forceinline__ void grad_heads(const RotateArgs& a, const Angles& angles, float* room,
                                           int64_t row0, int rows, const float* weight,
                                           Eight& sums) {
  constexpr int kGroups = kThreads / kGroup, kAhead = 2;
  const Side &in = kKeys ? a.k : a.q, &d_out = kKeys ? a.k_out : a.q_out,
             &d_in = kKeys ? a.d_k : a.d_q;
  const int heads = kKeys ? a.kv_heads : a.q_heads, items = rows * heads;
  const int piece = int(threadIdx.x) % kGroup, group = int(threadIdx.x) / kGroup;
  const bool on = 8 * piece < a.dim;
  Eight w;
  weights_of(weight, piece, on, w);
  for (int i0 = group; i0 < items + group; i0 += kGroups * kAhead) {
    Raw<T> raw_x[kAhead], raw_g[kAhead];
    Item item[kAhead];
    bool placed[kAhead];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const int i = i0 + n * kGroups;
      item[n] = {i / heads, i % heads};
      const int64_t row = row0 + item[n].row;
      int64_t from = row;
      if (kKeys && a.places.data && i < items) from = token_in(a.places, row, a.out_rows);
      placed[n] = i < items && from >= 0;
      raw_x[n] = fetch<T>(head_at<T>(in, row, item[n].head) + 8 * piece, on && placed[n]);
      raw_g[n] = fetch<T>(head_at<T>(d_out, from, item[n].head) + 8 * piece, on && placed[n]);
    }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const int i = i0 + n * kGroups;
      if (i - group >= items) break;
      const int r = min(item[n].row, kMostRows - 1);
      Eight x, g;
      widen(raw_x[n], x);
      widen(raw_g[n], g);
      turn<kPairs, true>(a, angles.cos[r], angles.sin[r], piece,
                         room + (kPairs == kAny ? group * kGroup * 8 : 0), g);
      if (a.norm) {
        float sum = 0.f, dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum += x[e] * x[e];
          dot += g[e] * w[e] * x[e];
        }
        const float f = 1.f / sqrtf(group_sum<kGroup>(sum) / float(a.dim) + a.eps);
        const float mean = group_sum<kGroup>(dot) * f / float(a.dim);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = x[e] * f;
          sums[e] += placed[n] ? g[e] * y : 0.f;
          g[e] = placed[n] ? f * (g[e] * w[e] - y * mean) : 0.f;
        }
      }
      if (on && i < items)
        put(head_at<T>(d_in, row0 + item[n].row, item[n].head) + 8 * piece, g);
    }
  }
}

// Blocks stay and go over the rows in turn, so that the weights' gradients are sums of
// few blocks, added behind them in one order.
template <class T, int kPairs, int kGroup>
__global__ __launch_bounds__(kThreads) void rotate_grad_kernel(RotateArgs a) {
  constexpr int kGroups = kThreads / kGroup;
  __shared__ Angles angles;
  __shared__ float room[kThreads * 8];
  Eight q_sums = {}, k_sums = {};
  const int piece = int(threadIdx.x) % kGroup, group = int(threadIdx.x) / kGroup;
  const int64_t step = int64_t(gridDim.x) * a.per_block;
  for (int64_t row0 = int64_t(blockIdx.x) * a.per_block; row0 < a.rows; row0 += step) {
    const int rows = int(min(int64_t(a.per_block), a.rows - row0));
    __syncthreads();  // nobody reads the last rows' angles any more
    form_angles(a, row0, rows, angles);
    __syncthreads();
    grad_heads<T, kPairs, kGroup, false>(a, angles, room, row0, rows, a.q_weight, q_sums);
    grad_heads<T, kPairs, kGroup, true>(a, angles, room, row0, rows, a.k_weight, k_sums);
  }
  if (!a.parts) return;
  // A block's sums of the weights' gradients, in the groups' order.
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e)
      room[(group * kGroup + piece) * 8 + e] = side ? k_sums[e] : q_sums[e];
    __syncthreads();
    for (int d = int(threadIdx.x); d < a.dim; d += kThreads) {
      float sum = 0.f;
      for (int g = 0; g < kGroups; ++g) sum += room[g * kGroup * 8 + d];
      a.parts[(int64_t(blockIdx.x) * 2 + side) * a.dim + d] = sum;
    }
  }
}

// Adds the blocks' parts: 16 columns and 64 rows of parts at a time.
__global__ __launch_bounds__(1024) void add_weights_kernel(const float* parts, int blocks, int dim,
                                                           float* d_q, float* d_k) {
  __shared__ double sums[64][17];
  const int col = int(threadIdx.x) % 16, lane = int(threadIdx.x) / 16;
  const int at = int(blockIdx.x) * 16 + col;
  double sum = 0;
  if (at < 2 * dim)
#pragma unroll 4
    for (int b = lane; b < blocks; b += 64) sum += double(parts[int64_t(b) * 2 * dim + at]);
  sums[lane][col] = sum;
  __syncthreads();
  if (lane != 0 || at >= 2 * dim) return;
  sum = 0;
  for (int i = 0; i < 64; ++i) sum += sums[i][col];
  float* const out = at < dim ? d_q : d_k;
  if (out) out[at < dim ? at : at - dim] = float(sum);
}

// Rows of a block: enough blocks for the card first (forward and backward of 1,001
// tokens: four rows take 27 % longer than one), then as many as share the angles (65,536
// tokens: four rows take 1 % longer than eight, two 6 %, one 26 %).
int rows_of_block(int64_t rows) {
  return int(std::min<int64_t>(kMostRows, std::max<int64_t>(1, rows / 1024)));
}
// Blocks of the backward pass (65,536 tokens, both passes: 512 take 22 % longer than
// 1,024, 2,048 as long).
int grad_blocks(int64_t rows) {
  const int64_t chunks = (rows + rows_of_block(rows) - 1) / rows_of_block(rows);
  return int(std::min<int64_t>(chunks, 1024));
}

template <class T, int kPairs, int kGroup>
hipError_t forward(const RotateArgs& a, hipStream_t s) {
  const int64_t blocks = (a.rows + a.per_block - 1) / a.per_block;
  RotateArgs part = a;
  for (int64_t b = 0; b < blocks; b += kMostBlocks) {  // rows' tensors move along
    const int64_t n = std::min(blocks - b, kMostBlocks), row = b * a.per_block;
    const int64_t bytes = int64_t(sizeof(T));
    auto moved = [&](const Side& x, int64_t rows) {
      return Side{x.data ? x.data + rows * x.row * bytes : nullptr, x.row, x.head};
    };
    auto tokens = [&](const Tokens& t) {
      return Tokens{t.data ? static_cast<const char*>(t.data) + row * (t.wide ? 8 : 4) : nullptr,
                    t.wide};
    };
    const bool placed = a.places.data != nullptr;
    part.q = moved(a.q, row);
    part.k = moved(a.k, row);
    part.v = moved(a.v, row);
    part.q_out = moved(a.q_out, row);
    part.k_out = placed ? a.k_out : moved(a.k_out, row);
    part.v_out = placed ? a.v_out : moved(a.v_out, row);
    part.positions = tokens(a.positions);
    part.places = tokens(a.places);
    part.rows = std::min(a.rows - row, n * a.per_block);
    hipLaunchKernelGGL((rotate_kernel<T, kPairs, kGroup>), dim3(unsigned(n)), dim3(kThreads), 0, s,
                       part);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}
template <class T, int kPairs, int kGroup>
hipError_t backward(const RotateArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((rotate_grad_kernel<T, kPairs, kGroup>), dim3(unsigned(grad_blocks(a.rows))),
                     dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <class T, int kPairs, bool kGrad>
hipError_t by_group(const RotateArgs& a, hipStream_t s) {
  if (a.dim <= 32) return kGrad ? backward<T, kPairs, 4>(a, s) : forward<T, kPairs, 4>(a, s);
  if (a.dim <= 64) return kGrad ? backward<T, kPairs, 8>(a, s) : forward<T, kPairs, 8>(a, s);
  if (a.dim <= 128) return kGrad ? backward<T, kPairs, 16>(a, s) : forward<T, kPairs, 16>(a, s);
  return kGrad ? backward<T, kPairs, 32>(a, s) : forward<T, kPairs, 32>(a, s);
}
template <class T, bool kGrad>
hipError_t by_pairs(const RotateArgs& a, bool interleaved, hipStream_t s) {
  if (interleaved) return by_group<T, kNext, kGrad>(a, s);
  if (a.pairs % 8 == 0) return by_group<T, kLanes, kGrad>(a, s);
  return by_group<T, kAny, kGrad>(a, s);
}
template <bool kGrad>
hipError_t by_type(const RotateArgs& a, const sched_norm_rotate_desc& d, hipStream_t s) {
  if (d.dtype == SCHED_F32) return by_pairs<float, kGrad>(a, d.interleaved, s);
  if (d.dtype == SCHED_F16) return by_pairs<f16, kGrad>(a, d.interleaved, s);
  return by_pairs<bf16, kGrad>(a, d.interleaved, s);
}

Side side(const sched_heads& h) {
  return {static_cast<char*>(h.data), h.row_stride, h.head_stride};
}

RotateArgs rotate_args(const sched_norm_rotate_desc& d) {
  RotateArgs a = {};
  a.q = side(d.q);
  a.k = side(d.k);
  a.positions = {d.positions.data, d.positions.bits == 64};
  a.places = {d.places.data, d.places.bits == 64};
  a.q_weight = d.q_weight;
  a.k_weight = d.k_weight;
  a.frequencies = d.frequencies;
  a.rows = d.rows;
  a.out_rows = d.out_rows;
  a.dim = d.head_dim;
  a.q_heads = d.q_heads;
  a.kv_heads = d.kv_heads;
  a.pairs = d.turned / 2;
  a.norm = d.norm;
  a.eps = d.eps;
  a.per_block = rows_of_block(d.rows);
  return a;
}

}  // namespace

hipError_t launch_norm_rotate(const sched_norm_rotate_desc& d, hipStream_t s) {
  if (d.rows == 0) return hipSuccess;
  RotateArgs a = rotate_args(d);
  a.v = side(d.v);
  a.q_out = side(d.q_out);
  a.k_out = side(d.k_out);
  a.v_out = side(d.v_out);
  return by_type<false>(a, d, s);
}

size_t norm_rotate_grad_bytes(const sched_norm_rotate_desc& d) {
  if (d.rows == 0 || !d.norm) return 0;
  return size_t(grad_blocks(d.rows)) * 2 * size_t(d.head_dim) * sizeof(float);
}

hipError_t launch_norm_rotate_grad(const sched_norm_rotate_desc& d, const sched_heads& d_q_out,
                                   const sched_heads& d_k_out, const sched_heads& d_q,
                                   const sched_heads& d_k, float* d_q_weight, float* d_k_weight,
                                   void* ws, hipStream_t s) {
  RotateArgs a = rotate_args(d);
  a.q_out = side(d_q_out);
  a.k_out = side(d_k_out);
  a.d_q = side(d_q);
  a.d_k = side(d_k);
  const bool weights = d_q_weight || d_k_weight;
  if (d.rows > 0) {
    a.parts = weights ? static_cast<float*>(ws) : nullptr;
    if (const hipError_t e = by_type<true>(a, d, s)) return e;
  }
  if (!weights) return hipSuccess;
  hipLaunchKernelGGL(add_weights_kernel, dim3(unsigned((2 * d.head_dim + 15) / 16)), dim3(1024), 0, s,
                     static_cast<const float*>(ws), d.rows > 0 ? grad_blocks(d.rows) : 0, d.head_dim,
                     d_q_weight, d_k_weight);
  return hipGetLastError();
}

}  // namespace policy
