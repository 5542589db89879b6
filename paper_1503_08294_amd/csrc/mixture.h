// Declarations shared by the sources of the mixture of local experts: layer norm, routing and
// the experts' products.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/gsn.h"

namespace gsn {

using bf16_t = __bf16;
using f16_t = _Float16;

constexpr int kWave = 64;

// An address that a kernel may read 16 bytes at a time from: rows of `ld` elements from base.
__host__ inline bool aligned16(const void* p) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

__host__ __device__ inline size_t size_of(int32_t dtype) { return dtype == GSN_F32 ? 4 : 2; }

template <typename T>
__device__ __forceinline__ float to_float(T v) {
  return static_cast<float>(v);
}
// rounding to nearest even; the one rounding of a result to its type
template <typename T>
__device__ __forceinline__ T from_float(float v) {
  return static_cast<T>(v);
}

// N elements read or written as one access where N * sizeof(T) is 2, 4, 8 or 16 bytes
template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
  T v[N];
};

// Sum over the lanes of a wave, the same order and result in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// 1 / (1 + exp(-v)).  __expf multiplies by log2 e in binary32 before it takes the power of two, so
// its relative error grows with its argument, to some (|v| + 3) 2^-24; where the exponential is the
// smaller term of the sum (v > 0) little of that is left.  exp(-v) past the largest float gives
// 1 / inf = 0, as it should.
__device__ __forceinline__ float sigmoid(float v) {
  return __builtin_amdgcn_rcpf(1.0f + __expf(-v));
}

}  // namespace gsn
