// Element types of a caller's matrices, accesses to them that need no more than the element's own alignment, and what else the
// kernels on them share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace onmt {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <int N>
struct Const {
  static constexpr int value = N;
};

// Elements of a 16-byte access.
template <class T>
constexpr int kVec = 16 / (int)sizeof(T);

template <class T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }
template <class T>
__device__ __forceinline__ T from_float(float v) { return (T)v; }      // to nearest even

template <class T>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(kVec<T>), aligned(sizeof(T))));
};

template <class T>
__device__ __forceinline__ void load_vec(const T* p, float* v) {
  const typename VecOf<T>::type x = *(const typename VecOf<T>::type*)p;
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) v[i] = (float)x[i];
}
template <class T>
__device__ __forceinline__ void store_vec(T* p, const float* v) {
  typename VecOf<T>::type x;
#pragma unroll
  for (int i = 0; i < kVec<T>; ++i) x[i] = (T)v[i];
  *(typename VecOf<T>::type*)p = x;
}

// The largest value of each half of the wave, in its lanes.
__device__ inline float half_max(float v) {
  v = fmaxf(v, dpp_move<0x111, 0xf>(v, v));
  v = fmaxf(v, dpp_move<0x112, 0xf>(v, v));
  v = fmaxf(v, dpp_move<0x114, 0xf>(v, v));
  v = fmaxf(v, dpp_move<0x118, 0xf>(v, v));
  v = fmaxf(v, dpp_move<0x142, 0xa>(v, v));
  return (threadIdx.x & 32) ? readlane_f(v, 63) : readlane_f(v, 31);
}

}  // namespace onmt
