// load_frag.h -- loads of matrix instructions' operands straight from memory.
#pragma once

#include "gemm.h"

namespace abcd {
namespace {

// Where loads of what lies outside an array go: under a condition a load would be
// waited for by itself, at the end of its branch.
__device__ uint32_t zeros[4];

// 16 bytes from p as they are where `in`, else 0.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type load_whole(const T* p, bool in) {
  typedef typename Frag<T>::type F;
  typedef F FU __attribute__((aligned(sizeof(T))));
  return *reinterpret_cast<const FU*>(in ? p : reinterpret_cast<const T*>(zeros));
}
// The first n elements of v, and zeros.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type keep_first(typename Frag<T>::type v, int n) {
  typedef uint32_t U4 __attribute__((ext_vector_type(4)));
  U4 m;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4)
      m[i] = n > i ? ~0u : 0u;
    else
      m[i] = n >= 2 * i + 2 ? ~0u : n == 2 * i + 1 ? 0xFFFFu : 0u;
  }
  return __builtin_bit_cast(typename Frag<T>::type, __builtin_bit_cast(U4, v) & m);
}

// 16 bytes from p of which n elements are wanted (n <= 0: none), the others 0; kWhole:
// all or none. room: elements from p to the end of the array: where it reaches over 16
// bytes what lies behind the row is loaded and masked, so that only the array's last
// elements take single loads.
template <typename T, bool kWhole>
__device__ __forceinline__ typename Frag<T>::type load_frag(const T* p, int n, int64_t room) {
  if (kWhole) return load_whole(p, n > 0);
  if (n >= kPer16<T> || n <= 0 || room >= kPer16<T>) return keep_first<T>(load_whole(p, n > 0), n);
  typename Frag<T>::type v = (T)0.0f;
#pragma unroll
  for (int i = 0; i < kPer16<T> - 1; ++i) v[i] = *(i < n ? p + i : reinterpret_cast<const T*>(zeros));
  return v;
}

}  // namespace
}  // namespace abcd
