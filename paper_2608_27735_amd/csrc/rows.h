// rows.h -- what the decoder's operators share: the three element types, loads
// and stores of 16 bytes of a row at any element's address, sums over the lanes
// that hold a row, and dropout's generator.
#pragma once

#include <type_traits>

#include "abcd_internal.h"

namespace abcd {

template <typename T, int N>
struct VecOf {
  typedef T type __attribute__((ext_vector_type(N)));
};
template <int N>
using Floats = typename VecOf<float, N>::type;

// Elements of 16 bytes.
template <typename T>
constexpr int kPer16 = 16 / (int)sizeof(T);

// Calls f with a value of the element type that dtype names.
template <typename F>
int32_t with_type(int32_t dtype, F f) {
  if (dtype == ABCD_F32) return f(float{});
  if (dtype == ABCD_F16) return f((_Float16)0);
  return f((__bf16)0);
}

inline size_t type_bytes(int32_t dtype) { return dtype == ABCD_F32 ? 4 : 2; }
inline size_t align256(size_t b) { return (b + 255) & ~size_t(255); }

namespace {
// Where loads of what lies outside an array go: under a condition a load would be
// waited for by itself, at the end of its branch.
__device__ uint32_t zeros[4];
}  // namespace

// N consecutive elements at p as floats, n of them within the row (the others
// are 0 and are not read). One load if all are: gfx950 loads a vector from any
// element's address, so rows of odd widths and strides need no other path.
template <typename T, int N, bool kWhole>
__device__ __forceinline__ Floats<N> load_vec(const T* p, int n) {
  typedef typename VecOf<T, N>::type V __attribute__((aligned(sizeof(T))));
  if (kWhole || n >= N) return __builtin_convertvector(*reinterpret_cast<const V*>(p), Floats<N>);
  Floats<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = (float)*(i < n ? p + i : reinterpret_cast<const T*>(zeros));
  return r;
}

// The same from an array of floats where f32 is set.
template <typename T, int N, bool kWhole>
__device__ __forceinline__ Floats<N> load_param(const void* p, int64_t at, int n, bool f32) {
  return f32 ? load_vec<float, N, kWhole>(static_cast<const float*>(p) + at, n)
             : load_vec<T, N, kWhole>(static_cast<const T*>(p) + at, n);
}

// Rounded once, to nearest with ties to even.
template <typename T, int N, bool kWhole>
__device__ __forceinline__ void store_vec(T* p, Floats<N> v, int n) {
  typedef typename VecOf<T, N>::type V;
  typedef V VU __attribute__((aligned(sizeof(T))));
  const V t = __builtin_convertvector(v, V);
  if (kWhole || n >= N) {
    *reinterpret_cast<VU*>(p) = t;
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < n) p[i] = t[i];
}

// Sum over G consecutive lanes (a power of two, aligned), returned to each.
template <int G>
__device__ __forceinline__ float lanes_sum(float x) {
  auto dpp = [](float v, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, false));
  };
  if (G >= 2) x += dpp(x, std::integral_constant<int, 0xB1>{});   // quad [1,0,3,2]
  if (G >= 4) x += dpp(x, std::integral_constant<int, 0x4E>{});   // quad [2,3,0,1]
  if (G >= 8) x += dpp(x, std::integral_constant<int, 0x141>{});  // half mirror
  if (G >= 16) x += dpp(x, std::integral_constant<int, 0x140>{}); // mirror
  if (G >= 32) x += __shfl_xor(x, 16, 64);
  if (G >= 64) x += __shfl_xor(x, 32, 64);
  return x;
}

// Sum over the G lanes of a row, G <= 64 or the workgroup's kBlock (every thread
// takes part; red: 4 floats of LDS. Of two calls in a row each has its own red:
// a wave that writes one again has met the other's barrier, behind all reads).
template <int G>
__device__ __forceinline__ float row_sum(float x, float* red) {
  if (G <= 64) return lanes_sum<(G <= 64 ? G : 64)>(x);
  x = lanes_sum<64>(x);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// Philox 4x32 with 7 rounds (Salmon et al., "Parallel random numbers: as easy as
// 1, 2, 3", 2011; the fewest rounds that pass their statistical tests), the
// counter (col / 4, row, offset low, offset high): one block serves four
// consecutive elements of a row, whatever the row's width and stride.
struct DropKey {
  uint32_t k0, k1, o0, o1;  // seed and offset
  uint32_t below;           // words below this are dropped: floor(p 2^32)
  float scale;              // 1 / (1 - p)
  int mode;                 // 0: p = 0, all are kept; 1: some; 2: p = 1, none is kept
};

inline DropKey drop_key(double p, uint64_t seed, uint64_t offset) {
  DropKey k{};
  k.k0 = (uint32_t)seed;
  k.k1 = (uint32_t)(seed >> 32);
  k.o0 = (uint32_t)offset;
  k.o1 = (uint32_t)(offset >> 32);
  k.mode = p >= 1.0 ? 2 : p > 0.0 ? 1 : 0;
  k.below = k.mode == 1 ? (uint32_t)(p * 4294967296.0) : 0;
  k.scale = k.mode == 2 ? 0.0f : (float)(1.0 / (1.0 - p));
  return k;
}

// Its four words for the elements (row, 4 quad + 0..3).
__device__ __forceinline__ uint4 drop_words(const DropKey& k, uint32_t row, uint32_t quad) {
  constexpr int kXor3 = 0x96;
  uint32_t c0 = quad, c1 = row, c2 = k.o0, c3 = k.o1, k0 = k.k0, k1 = k.k1;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
    c0 = __builtin_amdgcn_bitop3_b32((uint32_t)(b >> 32), c1, k0, kXor3);
    c1 = (uint32_t)b;
    c2 = __builtin_amdgcn_bitop3_b32((uint32_t)(a >> 32), c3, k1, kXor3);
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// add + dropout of N consecutive elements (a multiple of 4) from column col, a
// multiple of 4. What is dropped becomes 0, infinities and NaN too.
template <int N>
__device__ __forceinline__ Floats<N> drop_vec(Floats<N> v, const DropKey& k, uint32_t row, uint32_t col,
                                              Floats<N> add) {
  if (k.mode == 0) return add + v;
  if (k.mode == 2) return add;
  Floats<N> r;
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    const uint4 w = drop_words(k, row, col / 4 + q);
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[4 * q + i] = fmaf(word[i] >= k.below ? v[4 * q + i] : 0.0f, k.scale, add[4 * q + i]);
  }
  return r;
}

// The same of 8 elements of 16 bits, two a word, without the factor: masks of what is
// kept.
__device__ __forceinline__ uint4 drop_masks(const DropKey& k, uint32_t row, uint32_t col) {
  if (k.mode == 2) return make_uint4(0, 0, 0, 0);
  uint32_t m[4];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const uint4 w = drop_words(k, row, col / 4 + q);
    m[2 * q] = (w.x >= k.below ? 0xFFFFu : 0u) | (w.y >= k.below ? 0xFFFF0000u : 0u);
    m[2 * q + 1] = (w.z >= k.below ? 0xFFFFu : 0u) | (w.w >= k.below ? 0xFFFF0000u : 0u);
  }
  return make_uint4(m[0], m[1], m[2], m[3]);
}

}  // namespace abcd
