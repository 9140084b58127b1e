// Element types of a caller's matrices, and accesses to them that need no more than the element's own alignment.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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

}  // namespace onmt
