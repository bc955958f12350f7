// gated_ffn_few.h -- the gated feed-forward block of a few rows (single tokens and
// small batches), forward.
//
// The weights are read once and bound it. A workgroup takes 16 or 8 columns of the
// result and all rows; its waves divide the contraction, each with many loads of
// 16 bytes in flight straight into the matrix instructions' operands, and LDS joins
// their sums. No operand needs an alignment beyond its elements'. One row of 2,048 x
// 5,632 x 2,048 in bf16: 13 us for the projections (46 MB, 3.5 TB/s) and 8.7 for the way
// down (23 MB, 2.6 TB/s); the tiled products take 75 together.
#pragma once

#include "activation.h"
#include "gated_ffn_args.h"
#include "gemm.h"
#include "load_frag.h"

namespace abcd {
namespace {

// acc[x][s] = sum over the wave's part of the contraction of rows 16 x.. of X and
// rows first.. + 15 of W[s]: lane l gets row l & 15 of X and rows 4 (l >> 4) .. + 3 of W.
template <typename T, int kX, int kSides, int kWaves, bool kWhole>
__device__ __forceinline__ void few_products(f32x4 (&acc)[kX][kSides], const T* x, int64_t ldx, int n,
                                             const T* const (&w)[kSides], int64_t ldw, int first, int rows, int k_end) {
  typedef typename Frag<T>::type F;
  constexpr int kPer = kPer16<T>, kK = 4 * kPer;  // a lane's and a wave's elements of a contraction
  constexpr int kAhead = kX >= 4 ? 4 : 8;
  const int l = threadIdx.x & 63, j = l & 15, q = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < kX; ++i)
#pragma unroll
    for (int s = 0; s < kSides; ++s) acc[i][s] = 0.0f;
  const int steps = (k_end + kK - 1) / kK, per = (steps + kWaves - 1) / kWaves;
  const int end = min(steps, (wave + 1) * per);
  for (int s0 = wave * per; s0 < end; s0 += kAhead) {
    F fw[kSides][kAhead], fx[kX][kAhead];
#pragma unroll
    for (int t = 0; t < kAhead; ++t) {
      const int k = (s0 + t) * kK + q * kPer, left = s0 + t < end ? k_end - k : 0;
#pragma unroll
      for (int s = 0; s < kSides; ++s)
        fw[s][t] = load_frag<T, kWhole>(w[s] + (int64_t)(first + j) * ldw + k, first + j < rows ? left : 0,
                                        room_of(rows, first + j, ldw, left));
#pragma unroll
      for (int i = 0; i < kX; ++i)
        fx[i][t] = load_frag<T, kWhole>(x + (int64_t)(i * 16 + j) * ldx + k, i * 16 + j < n ? left : 0,
                                        room_of(n, i * 16 + j, ldx, left));
    }
#pragma unroll
    for (int t = 0; t < kAhead; ++t) {
      // what is not of the contraction has to be zero on both sides
      const int left = s0 + t < end ? k_end - ((s0 + t) * kK + q * kPer) : 0;
#pragma unroll
      for (int s = 0; s < kSides; ++s) fw[s][t] = first_of<T, kWhole>(fw[s][t], left);
#pragma unroll
      for (int i = 0; i < kX; ++i) {
        fx[i][t] = first_of<T, kWhole>(fx[i][t], left);
#pragma unroll
        for (int s = 0; s < kSides; ++s) acc[i][s] = mma(fw[s][t], fx[i][t], acc[i][s]);
      }
    }
  }
}

// The waves' sums of acc joined in LDS; threads below kX * 64 get theirs: thread t
// row fragment t / 64 as its lane has it.
template <int kX, int kSides, int kWaves>
__device__ __forceinline__ bool few_join(f32x4 (&acc)[kX][kSides], f32x4 (&sum)[kSides]) {
  __shared__ __align__(16) f32x4 red[kWaves][kX][kSides][64];
  const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < kX; ++i)
#pragma unroll
    for (int s = 0; s < kSides; ++s) red[wave][i][s][l] = acc[i][s];
  __syncthreads();
  if (threadIdx.x >= kX * 64) return false;
#pragma unroll
  for (int s = 0; s < kSides; ++s) {
    sum[s] = red[0][wave][s][l];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) sum[s] += red[v][wave][s][l];
  }
  return true;
}

constexpr int kFewInWaves = 8, kFewOutWaves = 16;

template <typename T, int kAct, int kX, bool kWhole>
__global__ __launch_bounds__(kFewInWaves * 64) void ffn_few_in_kernel(FfnIn a) {
  f32x4 acc[kX][2], sum[2];
  const int first = blockIdx.x * 16, n = (int)a.x.len;
  const T* const w[2] = {static_cast<const T*>(a.w.p[0]), static_cast<const T*>(a.w.p[1])};
  few_products<T, kX, 2, kFewInWaves, kWhole>(acc, static_cast<const T*>(a.x.p[0]), a.x.ld, n, w, a.w.ld, first,
                                              (int)a.h, (int)a.d);
  if (!few_join<kX, 2, kFewInWaves>(acc, sum)) return;
  const int l = threadIdx.x & 63, r = (threadIdx.x >> 6) * 16 + (l & 15), c = first + (l >> 4) * 4;
  if (r >= n || c >= a.ldh) return;
  if (a.bg && c < a.h) sum[0] += load_vec<T, 4, false>(static_cast<const T*>(a.bg) + c, (int)a.h - c);
  if (a.bu && c < a.h) sum[1] += load_vec<T, 4, false>(static_cast<const T*>(a.bu) + c, (int)a.h - c);
  f32x4 h, hg, hu;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool in = c + i < a.h;  // else padding, which products read
    const float g = in ? sum[0][i] : 0.0f, u = in ? sum[1][i] : 0.0f;
    float slope;
    hu[i] = activate<kAct, sizeof(T) == 2>(g, slope);
    h[i] = hu[i] * u;
    hg[i] = slope * u;
  }
  const int64_t at = (int64_t)r * a.ldh + c;
  store_vec<T, 4, true>(static_cast<T*>(a.hidden) + at, h, 4);
  if (a.by_gate) {
    store_vec<T, 4, true>(static_cast<T*>(a.by_gate) + at, hg, 4);
    store_vec<T, 4, true>(static_cast<T*>(a.by_up) + at, hu, 4);
  }
}

// 8 columns a workgroup, the other half of the matrix instructions empty, where that
// still is no more than one for a CU: 5,632 x 2,048 in bf16 11.0 us instead of 12.4 (with
// 4 columns 14.5), 2,816 x 1,024 7.4 instead of 8.2.
template <typename T, int kX, bool kWhole>
__global__ __launch_bounds__(kFewOutWaves * 64) void ffn_few_out_kernel(FfnOut a) {
  f32x4 acc[kX][1], sum[1];
  const int columns = (int64_t)gridDim.x * 8 >= a.o ? 8 : 16;
  const int first = blockIdx.x * columns, end = min((int)a.o, first + columns), n = (int)a.hidden.len;
  const T* const w[1] = {static_cast<const T*>(a.w.p[0])};
  few_products<T, kX, 1, kFewOutWaves, kWhole>(acc, static_cast<const T*>(a.hidden.p[0]), a.hidden.ld, n, w, a.w.ld,
                                               first, end, (int)a.h);
  if (!few_join<kX, 1, kFewOutWaves>(acc, sum)) return;
  const int l = threadIdx.x & 63, r = (threadIdx.x >> 6) * 16 + (l & 15), c = first + (l >> 4) * 4;
  const int left = end - c;
  if (r >= n || left <= 0) return;
  if (a.bias) sum[0] += load_vec<T, 4, false>(static_cast<const T*>(a.bias) + c, left);
  f32x4 y = 0.0f;
  if (a.res) y = load_vec<T, 4, false>(static_cast<const T*>(a.res) + r * a.ldr + c, left);
  y = drop_vec<4>(sum[0], a.key, (uint32_t)r, (uint32_t)c, y);
  store_vec<T, 4, false>(static_cast<T*>(a.y) + r * a.ldy + c, y, left);
}

template <typename F>
int32_t with_rows(int64_t n, F f) {
  if (n <= 16) return f(std::integral_constant<int, 1>{});
  if (n <= 32) return f(std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 4>{});
}

template <typename T>
int32_t run_few_in(const FfnIn& a, hipStream_t stream) {
  return with_act(a.act, [&](auto act) -> int32_t {
    return with_rows(a.x.len, [&](auto rows) -> int32_t {
      constexpr int kAct = decltype(act)::value, kX = decltype(rows)::value;
      const int64_t grid = (a.ldh + 15) / 16;
      if (a.d % kPer16<T> == 0)
        ABCD_LAUNCH("ffn_few_in", (ffn_few_in_kernel<T, kAct, kX, true>), grid, kFewInWaves * 64, 0, stream, a);
      else
        ABCD_LAUNCH("ffn_few_in", (ffn_few_in_kernel<T, kAct, kX, false>), grid, kFewInWaves * 64, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    });
  });
}

template <typename T>
int32_t run_few_out(const FfnOut& a, hipStream_t stream) {
  return with_rows(a.hidden.len, [&](auto rows) -> int32_t {
    constexpr int kX = decltype(rows)::value;
    const int64_t grid = (a.o + 7) / 8 <= kCUs ? (a.o + 7) / 8 : (a.o + 15) / 16;
    if (a.h % kPer16<T> == 0)
      ABCD_LAUNCH("ffn_few_out", (ffn_few_out_kernel<T, kX, true>), grid, kFewOutWaves * 64, 0, stream, a);
    else
      ABCD_LAUNCH("ffn_few_out", (ffn_few_out_kernel<T, kX, false>), grid, kFewOutWaves * 64, 0, stream, a);
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

}  // namespace
}  // namespace abcd
