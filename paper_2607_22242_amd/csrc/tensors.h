// tensors.h -- what the kernels of sched_policy.h share: element types, 16-byte
// pieces of rows, and reductions over a wave and a block.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace policy {

typedef _Float16 f16;
typedef __bf16 bf16;

constexpr int kWave = 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <class T>
struct Vec {
  static constexpr int kN = 16 / int(sizeof(T));
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
};

// 16 bytes at an address that is aligned to its elements only (a row of an odd
// vocabulary): one wide access all the same.
template <class T>
__device__ __forceinline__ typename Vec<T>::type load16(const T* p) {
  typename Vec<T>::type v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
template <class T>
__device__ __forceinline__ void store16(T* p, typename Vec<T>::type v) {
  __builtin_memcpy(p, &v, 16);
}

// The same past the caches, for what this launch does not read again.
template <class T>
__device__ __forceinline__ void stream16(T* p, typename Vec<T>::type v) {
  typedef typename Vec<T>::type Loose __attribute__((aligned(sizeof(T))));
  __builtin_nontemporal_store(v, reinterpret_cast<Loose*>(p));
}

// Powers and logarithms to the base 2 as the hardware has them (1 ulp).
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log_2(float x) { return __builtin_amdgcn_logf(x); }

// Natural logarithm of a positive sum with one step of Newton's: the hardware's
// logarithm errs to one side (by 9e-8 of 1 to 3 on average), the power does not,
// and what all of a loss's terms share does not average out.
__device__ __forceinline__ float ln(float s) {
  const float y = log_2(s);
  return __builtin_fmaf(y, kLn2, __builtin_fmaf(s, pow2(-y), -1.f));
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// Sum over a block of up to 16 waves, for every thread; `part` holds a value
// per wave and may be used again after the next barrier.
template <class V>
__device__ __forceinline__ V block_sum(V x, V* part) {
  const int waves = int(blockDim.x) / kWave;
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = x;
  __syncthreads();
  x = part[0];
  for (int i = 1; i < waves; ++i) x += part[i];
  return x;
}

// Token i of an array of 32- or 64-bit tokens; -1 for what is outside [0, vocab).
struct Tokens {
  const void* data;
  int32_t wide;
};
__device__ __forceinline__ int64_t token_at(const Tokens& t, int64_t i) {
  return t.wide ? static_cast<const int64_t*>(t.data)[i] : static_cast<const int32_t*>(t.data)[i];
}
__device__ __forceinline__ int64_t token_in(const Tokens& t, int64_t i, int64_t vocab) {
  const int64_t v = token_at(t, i);
  return v >= 0 && v < vocab ? v : -1;
}

// Offset i, cut to [0, n].
__device__ __forceinline__ int offset_at(const int32_t* offsets, int i, int n) {
  const int v = offsets[i];
  return v < 0 ? 0 : v > n ? n : v;
}

// The last of n sequences whose offset is at most i (offsets ascend; empty
// sequences before a row are passed over).
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (offsets[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace policy
