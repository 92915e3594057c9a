// Neighbours in memory as vectors, for kernels whose arrays start at any multiple of their element.
#pragma once

#include <hip/hip_runtime.h>

#include "nna_internal.h"

namespace nna {

typedef _Float16 f16;
typedef __bf16 bf16;

template <typename T, int N>
struct Vec {
  typedef T plain __attribute__((ext_vector_type(N)));
  typedef T any __attribute__((ext_vector_type(N), aligned(sizeof(T))));  // the address need only be a multiple of the element
};
template <typename T>
struct Vec<T, 1> {
  typedef T plain;
  typedef T any;
};

template <int N, typename T>
__device__ __forceinline__ typename Vec<T, N>::plain vec_load(const T* p) {
  return *reinterpret_cast<const typename Vec<T, N>::any*>(p);
}
template <int N, typename T>
__device__ __forceinline__ void vec_store(T* p, typename Vec<T, N>::plain v) {
  *reinterpret_cast<typename Vec<T, N>::any*>(p) = v;
}
template <int N, typename V>
__device__ __forceinline__ auto vec_at(const V& v, int i) {
  if constexpr (N == 1)
    return v;
  else
    return v[i];
}
template <int N, typename V, typename E>
__device__ __forceinline__ void vec_set(V& v, int i, E e) {
  if constexpr (N == 1)
    v = e;
  else
    v[i] = e;
}

// fn(a value of the type)
template <typename F>
hipError_t by_element(int type, F fn) {
  return type == NNA_F32 ? fn(float()) : type == NNA_BF16 ? fn(bf16()) : type == NNA_F16 ? fn(f16()) : hipErrorInvalidValue;
}

}  // namespace nna
