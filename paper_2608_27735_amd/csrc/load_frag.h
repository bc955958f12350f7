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
// The same where only n of them may be there (n <= 0: none).
template <typename T, bool kWhole>
__device__ __forceinline__ typename Frag<T>::type load_frag(const T* p, int n) {
  if (kWhole || n >= kPer16<T> || n <= 0) return load_whole(p, n > 0);
  typename Frag<T>::type v = (T)0.0f;
#pragma unroll
  for (int i = 0; i < kPer16<T> - 1; ++i)
    if (i < n) v[i] = p[i];
  return v;
}

}  // namespace
}  // namespace abcd
