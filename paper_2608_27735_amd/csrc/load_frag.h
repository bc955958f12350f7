// load_frag.h -- loads of matrix instructions' operands straight from memory.
#pragma once

#include "gemm.h"

namespace abcd {
namespace {

// 16 bytes from p as they are where `in`, else 0.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type load_whole(const T* p, bool in) {
  typedef typename Frag<T>::type F;
  typedef F FU __attribute__((aligned(sizeof(T))));
  return *reinterpret_cast<const FU*>(in ? p : reinterpret_cast<const T*>(zeros));
}
// Elements to the end of an array of n rows, ld apart, from one of row r of which `left`
// are left in its row; no more of them are counted than 16 bytes need.
__device__ __forceinline__ int room_of(int64_t n, int64_t r, int64_t ld, int left) {
  const int64_t below = n - 1 - r;
  return (int)(below < 8 ? below : 8) * (int)(ld < 8 ? ld : 8) + left;
}

// 16 bytes from p of which n elements are wanted (n <= 0: none); kWhole: all or none.
// The others come as they may (first_of makes zeros of them, once the load has to have
// arrived anyway: done here it would be waited for at once). room: elements from p to
// the end of the array: where it reaches over 16 bytes what lies behind the row is
// loaded too, so that only the array's last elements take single loads.
template <typename T, bool kWhole>
__device__ __forceinline__ typename Frag<T>::type load_frag(const T* p, int n, int room) {
  const bool single = !kWhole && n > 0 && n < kPer16<T> && room < kPer16<T>;
  typename Frag<T>::type v = load_whole(p, n > 0 && !single);
  if (single) {
#pragma unroll
    for (int i = 0; i < kPer16<T> - 1; ++i) v[i] = *(i < n ? p + i : reinterpret_cast<const T*>(zeros));
  }
  return v;
}

// The first n elements of what load_frag gave, and zeros.
template <typename T, bool kWhole>
__device__ __forceinline__ typename Frag<T>::type first_of(typename Frag<T>::type v, int n) {
  if (kWhole) return v;
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

// Both, for a load that is used at once.
template <typename T, bool kWhole>
__device__ __forceinline__ typename Frag<T>::type load_first(const T* p, int n, int room) {
  return first_of<T, kWhole>(load_frag<T, kWhole>(p, n, room), n);
}

}  // namespace
}  // namespace abcd
