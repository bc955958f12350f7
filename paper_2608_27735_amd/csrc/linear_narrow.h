// linear_narrow.h -- the linear layer of many narrow rows (one per Gaussian), forward and
// backward in one pass over the rows each, for 16-bit element types.
//
// With i and o up to 128 nothing but the rows' arrays counts: forward x and the residual are
// read and y written, backward x and dy read and dx written, and weights, products and
// sums stay in LDS and registers. A wave takes 32 rows by itself, so that no barrier
// stands between loads and stores; the matrix instruction's result (four consecutive
// columns of a row) is the next one's operand without leaving the registers, two results
// side by side being eight indexes of a contraction.
//
// Backward, of 32 rows: z by the weights in LDS, dz = dy act'(z) in registers, dx from dz
// and the weights turned round; then x and dz go through a piece of LDS of the wave's own,
// from which both are read across (ds_read_b64_tr_b16) as operands of dw = dz' x, whose
// sums stay in the wave's registers over all its rows, as do the bias's, of dz before it is
// rounded. The workgroup's four waves add their sums up in LDS, and a second launch adds the
// workgroups' in a fixed order.
//
// 1M x 64 to 64 in bf16: forward with SiLU and a residual 75 us (384 MB, 5.1 TB/s), backward 84
// without an activation (384 MB), 94 with SiLU and 104 with GELU, of an 8-bit checkpoint 74, 88
// and 100 (322 MB): two waves a SIMD, by their registers, wait for loads, products and LDS in turn,
// vector instructions 45 percent busy. 128 to 64: 100 and 180; one wave a SIMD, as two spill.
#pragma once

#include <algorithm>

#include "activation.h"
#include "gemm.h"
#include "linear_args.h"
#include "load_frag.h"
#include "pack8.h"

namespace abcd {
namespace {

constexpr int kNarrowLayerThreads = 256, kNarrowLayerWaves = kNarrowLayerThreads / 64;
constexpr int kLinearKept = 5;  // an "act" whose slope is read

// Which of a result's columns index r of its block b of 16 is: quarter q of a pair of blocks
// holds 8 consecutive columns, and the quarters those of 64 bytes next to each other
// (with all of a quarter's blocks consecutive 1M x 64 to 128 forward takes 173 us).
__device__ __forceinline__ int column_of(int b, int r) { return (b >> 1) * 32 + (r >> 2) * 8 + (b & 1) * 4 + (r & 3); }

// Which of x's columns quarter q of contraction f of 32 begins at: those of rows in memory lie
// 64 bytes of a row next to each other; of an 8-bit checkpoint a quarter has kDF 8 bytes, which
// it so loads at once.
template <int kDF>
__device__ __forceinline__ int column_along(int f, int q, bool packed) {
  return packed ? (q * kDF + f) * 8 : f * 32 + q * 8;
}

// Fragment f of the weights for z: block f / kDF of 16 columns of z, contraction f % kDF of
// 32.
template <typename T, int kDF, bool kWhole>
__device__ __forceinline__ typename Frag<T>::type weights_along(const void* w, int f, int rows, int cols, bool packed) {
  const int l = threadIdx.x & 63, j = l & 15;
  const int row = column_of(f / kDF, j), col = column_along<kDF>(f % kDF, l >> 4, packed);
  const T* const p = static_cast<const T*>(w) + (int64_t)row * cols + col;
  if (kWhole) return load_whole(p, row < rows && col < cols);
  typename Frag<T>::type v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = *(row < rows && col + e < cols ? p + e : reinterpret_cast<const T*>(zeros));
  return v;
}
// Fragment f of the weights turned round, for dx: block f / kOF of 16 columns of dx,
// contraction f % kOF of 32 columns of z.
template <typename T, int kOF>
__device__ __forceinline__ typename Frag<T>::type weights_across(const void* w, int f, int rows, int cols) {
  const int l = threadIdx.x & 63;
  const int col = column_of(f / kOF, l & 15), row = f % kOF * 32 + (l >> 4) * 8;
  typename Frag<T>::type v;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = *(row + e < rows && col < cols ? static_cast<const T*>(w) + (int64_t)(row + e) * cols + col
                                          : reinterpret_cast<const T*>(zeros));
  return v;
}

template <typename T>
__device__ __forceinline__ typename Frag<T>::type round8(f32x4 a, f32x4 b) {
  typename Frag<T>::type r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (T)a[i], r[4 + i] = (T)b[i];
  return r;
}

// kDF: contractions of 32 that hold i; kOB: 16-column blocks of o. kWhole: i and o are
// multiples of 8.
template <typename T, int kAct, int kDF, int kOB, bool kWhole>
__global__ __launch_bounds__(kNarrowLayerThreads, kDF * kOB <= 16 ? 4 : 2) void linear_narrow_kernel(LinearNarrow a) {
  typedef typename Frag<T>::type F;
  constexpr int kFrags = kDF * kOB;
  __shared__ __align__(16) F weights[kFrags * 64];
  __shared__ __align__(16) float bias[kOB * 16];
  const int i = (int)a.i, o = (int)a.o;
  const int l = threadIdx.x & 63, j = l & 15, q = l >> 4, wave = threadIdx.x >> 6;
#pragma unroll 2
  for (int f = wave; f < kFrags; f += kNarrowLayerWaves) weights[f * 64 + l] = weights_along<T, kDF, kWhole>(a.w, f, o, i, false);
  if (threadIdx.x < kOB * 16)
    bias[threadIdx.x] = a.bias && (int)threadIdx.x < o ? (float)static_cast<const T*>(a.bias)[threadIdx.x] : 0.0f;
  __syncthreads();
  const int64_t step = (int64_t)gridDim.x * kNarrowLayerWaves * 32;
  for (int64_t r0 = ((int64_t)blockIdx.x * kNarrowLayerWaves + wave) * 32; r0 < a.n; r0 += step) {
    F x[2][kDF], res[2][kOB / 2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t r = r0 + k * 16 + j;
#pragma unroll
      for (int f = 0; f < kDF; ++f) {
        const int c = f * 32 + q * 8, left = r < a.n ? i - c : 0;
        x[k][f] = load_frag<T, kWhole>(static_cast<const T*>(a.x) + r * a.ldx + c, left, room_of(a.n, r, a.ldx, left));
      }
    }
    if (a.res)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int b = 0; b < kOB / 2; ++b) {
          const int64_t r = r0 + k * 16 + j;
          const int c = b * 32 + q * 8, left = r < a.n ? o - c : 0;
          res[k][b] = load_frag<T, kWhole>(static_cast<const T*>(a.res) + r * a.ldr + c, left, room_of(a.n, r, a.ldr, left));
        }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int f = 0; f < kDF; ++f) x[k][f] = first_of<T, kWhole>(x[k][f], i - (f * 32 + q * 8));
#pragma unroll
    for (int b = 0; b < kOB; b += 2) {
      __builtin_amdgcn_sched_barrier(0);  // one at a time, for the registers' sake
      const int c = b * 16 + q * 8;
      f32x4 z[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        z[0][h] = z[1][h] = *reinterpret_cast<const f32x4*>(&bias[c + h * 4]);
#pragma unroll
        for (int f = 0; f < kDF; ++f) {
          const F w = weights[((b + h) * kDF + f) * 64 + l];
#pragma unroll
          for (int k = 0; k < 2; ++k) z[k][h] = mma(w, x[k][f], z[k][h]);
        }
      }
      const int left = o - c;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t r = r0 + k * 16 + j;
        Floats<8> y, s;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float slope;
          y[e] = activate<kAct, true>(z[k][e / 4][e % 4], slope);
          s[e] = e < left ? slope : 0.0f;
        }
        if (r >= a.n) continue;
        if (left > 0) {
          if (a.res) y += __builtin_convertvector(res[k][b / 2], Floats<8>);
          store_vec<T, 8, kWhole>(static_cast<T*>(a.y) + r * a.ldy + c, y, left);
        }
        if (kAct != ABCD_ACT_NONE && a.slope && c < a.ldslope)
          store_slopes<8>(static_cast<int16_t*>(a.slope) + r * a.ldslope + c, s);
      }
    }
  }
}

// Where element (row, column 4 unit) lies in a wave's LDS, rows of kBytes: neither the lanes
// that write 16 bytes of consecutive rows nor those that read 8 bytes across them meet a
// bank too often.
template <int kBytes>
__device__ __forceinline__ int turned_row(int row, int unit) {
  return row * kBytes + (((unit >> 1) ^ (row & 7)) * 16) + (unit & 1) * 8;
}

template <typename T, int kMode, int kDF, int kOB, bool kWhole>
__global__ __launch_bounds__(kNarrowLayerThreads, kDF * kOB <= 8 ? 2 : 1) void linear_narrow_bwd_kernel(LinearNarrowBwd a) {
  typedef typename Frag<T>::type F;
  typedef __attribute__((address_space(3))) F LdsF;
  constexpr int kIB = 2 * kDF, kOF = kOB / 2, kFrags = kDF * kOB, kXBytes = kDF * 64, kZBytes = kOB * 32;
  constexpr int kWaveBytes = 32 * (kXBytes + kZBytes), kSums = kOB * 16 * kIB * 16;
  constexpr bool kAgain = kMode != ABCD_ACT_NONE && kMode != kLinearKept;  // z is needed
  constexpr bool kEarly = kFrags <= 8 && kWhole;  // where the registers suffice
  constexpr bool kLargest = !std::is_same<T, _Float16>::value;
  constexpr int kPool = kNarrowLayerWaves * kWaveBytes > kSums * 4 ? kNarrowLayerWaves * kWaveBytes : kSums * 4;
  __shared__ __align__(16) F along[kAgain ? kFrags * 64 : 1];
  __shared__ __align__(16) F across[kFrags * 64];
  __shared__ __align__(16) char pool[kPool];
  const int i = (int)a.i, o = (int)a.o;
  const int l = threadIdx.x & 63, j = l & 15, q = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int f = wave; f < kFrags; f += kNarrowLayerWaves) {
    if (kAgain) along[f * 64 + l] = weights_along<T, kDF, kWhole>(a.w, f, o, i, a.q != nullptr);
    across[f * 64 + l] = weights_across<T, kOF>(a.w, f, o, i);
  }
  __syncthreads();
  LdsChar* const xs = (LdsChar*)pool + wave * kWaveBytes;
  LdsChar* const zs = xs + 32 * kXBytes;
  f32x4 dw[kOB][kIB], db[kOB];
#pragma unroll
  for (int b = 0; b < kOB; ++b) {
    db[b] = 0.0f;
#pragma unroll
    for (int k = 0; k < kIB; ++k) dw[b][k] = 0.0f;
  }
  // what is on its way: x (or the 8-bit one: kDF / 2 vectors and then an exponent), dy, the slopes
  F nx[2][kDF], ny[2][kOF];
  VecOf<int16_t, 8>::type ns[2][kOF];
  const int blocks8 = (i + kPackBlock - 1) / kPackBlock;
  auto fetch = [&](int64_t from) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t r = from + k * 16 + j;
      const bool in = r < a.n;
      if (a.q) {
        const bool there = in && q * kDF * 8 < blocks8 * kPackBlock;
        const char* const from = reinterpret_cast<const char*>(a.q) + r * blocks8 * kPackBlock + q * kDF * 8;
#pragma unroll
        for (int f = 0; f < kDF / 2; ++f)
          nx[k][f] = *reinterpret_cast<const F*>(there ? from + f * 16 : reinterpret_cast<const char*>(zeros));
        const uint8_t e = *(there ? a.e + r * blocks8 + q * kDF / 4 : reinterpret_cast<const uint8_t*>(zeros));
        typedef VecOf<uint32_t, 4>::type U4;
        nx[k][kDF / 2] = __builtin_bit_cast(F, (U4){(uint32_t)e, 0u, 0u, 0u});
      } else {
#pragma unroll
        for (int f = 0; f < kDF; ++f) {
          const int c = f * 32 + q * 8, left = in ? i - c : 0;
          nx[k][f] = load_frag<T, kWhole>(static_cast<const T*>(a.x) + r * a.ldx + c, left, room_of(a.n, r, a.ldx, left));
        }
      }
#pragma unroll
      for (int b = 0; b < kOF; ++b) {
        const int c = b * 32 + q * 8, left = in ? o - c : 0;
        ny[k][b] = load_frag<T, kWhole>(static_cast<const T*>(a.dy) + r * a.lddy + c, left, room_of(a.n, r, a.lddy, left));
        if (kMode == kLinearKept) {
          typedef VecOf<int16_t, 8>::type H;
          ns[k][b] = *reinterpret_cast<const H*>(in && c < a.ldslope ? static_cast<const int16_t*>(a.slope) + r * a.ldslope + c
                                                                    : reinterpret_cast<const int16_t*>(zeros));
        }
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * kNarrowLayerWaves * 32;
  int64_t r0 = ((int64_t)blockIdx.x * kNarrowLayerWaves + wave) * 32;
  fetch(r0);
  for (; r0 < a.n; r0 += step) {
    F x[2][kDF], dy[2][kOF];
    Floats<8> slope[2][kOF];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      typedef VecOf<uint32_t, 4>::type U4;
      // (outside the array the exponent is 0: the least one's unit, of numbers that are 0)
      const float unit = packed_unit(max(__builtin_bit_cast(U4, nx[k][kDF / 2])[0], (uint32_t)kPackLeast));
#pragma unroll
      for (int f = 0; f < kDF; ++f) {
        if (a.q) {
          const U4 v = __builtin_bit_cast(U4, nx[k][f / 2]);
          x[k][f] = __builtin_convertvector(unpack_8<kLargest>(v[f % 2 * 2], v[f % 2 * 2 + 1], unit), F);
        } else {
          x[k][f] = first_of<T, kWhole>(nx[k][f], i - (f * 32 + q * 8));
        }
        *(LdsF*)(xs + turned_row<kXBytes>(k * 16 + j, column_along<kDF>(f, q, a.q != nullptr) / 4)) = x[k][f];
      }
#pragma unroll
      for (int b = 0; b < kOF; ++b) {
        dy[k][b] = first_of<T, kWhole>(ny[k][b], o - (b * 32 + q * 8));
        if (kMode == kLinearKept) slope[k][b] = slopes_of<8>(ns[k][b]);
      }
    }
    if (kEarly) fetch(r0 + step);  // past the end: zeros
    F dz[2][kOF];
#pragma unroll
    for (int b = 0; b < kOF; ++b) {
      __builtin_amdgcn_sched_barrier(0);  // one at a time, for the registers' sake
      const int c = b * 32 + q * 8;
      f32x4 z[2][2];
      if (kAgain) {
        const bool some = a.bias && c < o;
        const Floats<8> bias = load_vec<T, 8, kWhole>(some ? static_cast<const T*>(a.bias) + c : reinterpret_cast<const T*>(zeros),
                                                      some ? o - c : 8);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int e = 0; e < 4; ++e) z[0][h][e] = z[1][h][e] = bias[h * 4 + e];
#pragma unroll
          for (int f = 0; f < kDF; ++f) {
            const F w = along[((2 * b + h) * kDF + f) * 64 + l];
#pragma unroll
            for (int k = 0; k < 2; ++k) z[k][h] = mma(w, x[k][f], z[k][h]);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        Floats<8> v = __builtin_convertvector(dy[k][b], Floats<8>);
        if (kMode == kLinearKept) v *= slope[k][b];
        if (kAgain) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float s;
            activate<kAgain ? kMode : ABCD_ACT_NONE, true>(z[k][e / 4][e % 4], s);
            v[e] *= s;
          }
          // rows past the end have dy 0, but a weight's NaN is no row's
          const bool in = r0 + k * 16 + j < a.n;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = in && c + e < o ? v[e] : 0.0f;
        }
        const f32x4 lo = __builtin_shufflevector(v, v, 0, 1, 2, 3), hi = __builtin_shufflevector(v, v, 4, 5, 6, 7);
        db[2 * b] += lo;
        db[2 * b + 1] += hi;
        dz[k][b] = round8<T>(lo, hi);
        *(LdsF*)(zs + turned_row<kZBytes>(k * 16 + j, (b * 4 + q) * 2)) = dz[k][b];
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!kEarly) fetch(r0 + step);  // x's registers are free by now
    if (a.dx)
#pragma unroll
      for (int m = 0; m < kIB; m += 2) {
        __builtin_amdgcn_sched_barrier(0);
        f32x4 ax[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          ax[0][h] = ax[1][h] = 0.0f;
#pragma unroll
          for (int b = 0; b < kOF; ++b) {
            const F w = across[((m + h) * kOF + b) * 64 + l];
#pragma unroll
            for (int k = 0; k < 2; ++k) ax[k][h] = mma(w, dz[k][b], ax[k][h]);
          }
        }
        const int c = m * 16 + q * 8, left = i - c;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int64_t r = r0 + k * 16 + j;
          if (r < a.n && left > 0)
            store_vec<T, 8, kWhole>(static_cast<T*>(a.dx) + r * a.lddx + c,
                                    __builtin_shufflevector(ax[k][0], ax[k][1], 0, 1, 2, 3, 4, 5, 6, 7), left);
        }
      }
    __builtin_amdgcn_sched_barrier(0);
    // the wave's own x and dz across: what it wrote is there (LDS keeps a wave's order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    F xt[kIB];
    const int row = q * 8 + (j >> 2);
#pragma unroll
    for (int m = 0; m < kIB; ++m)
      xt[m] = read_across<T>(xs + turned_row<kXBytes>(row, m * 4 + (j & 3)), xs + turned_row<kXBytes>(row + 4, m * 4 + (j & 3)));
#pragma unroll
    for (int b = 0; b < kOB; ++b) {
      const F zt = read_across<T>(zs + turned_row<kZBytes>(row, b * 4 + (j & 3)), zs + turned_row<kZBytes>(row + 4, b * 4 + (j & 3)));
#pragma unroll
      for (int m = 0; m < kIB; ++m) dw[b][m] = mma(xt[m], zt, dw[b][m]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  if (!a.part) return;
  // The waves' sums one after the other in LDS: [o][i], lane (j, q) of block (b, m) has
  // columns m 16 + 4 q .. + 3 of row b 16 + j.
  float* const sums = reinterpret_cast<float*>(pool);
  constexpr int kPitch = kIB * 16;
  for (int v = 0; v < kNarrowLayerWaves; ++v) {
    __syncthreads();
    if (v != wave) continue;
#pragma unroll
    for (int b = 0; b < kOB; ++b)
#pragma unroll
      for (int m = 0; m < kIB; ++m) {
        f32x4* const at = reinterpret_cast<f32x4*>(&sums[(b * 16 + j) * kPitch + m * 16 + q * 4]);
        *at = v == 0 ? dw[b][m] : *at + dw[b][m];
      }
  }
  __syncthreads();
  float* const part = a.part + (int64_t)blockIdx.x * (a.o * a.i + a.o);
  for (int k = threadIdx.x; k < o * i; k += kNarrowLayerThreads) part[k] = sums[k / i * kPitch + k % i];
  __syncthreads();
  // the bias's: lane (j, q) has those of its rows, of a quarter's columns
#pragma unroll
  for (int b = 0; b < kOB; ++b)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float s = lanes_sum<16>(db[b][e]);
      if (j == 0) sums[wave * kOB * 16 + column_of(b, q * 4 + e)] = s;
    }
  __syncthreads();
  if ((int)threadIdx.x < o) {
    float s = 0.0f;
    for (int v = 0; v < kNarrowLayerWaves; ++v) s += sums[v * kOB * 16 + threadIdx.x];
    part[o * i + threadIdx.x] = s;
  }
}

template <typename T>
int32_t run_linear_narrow(const LinearNarrow& a, int64_t blocks, hipStream_t stream) {
  return with_any_act(a.act, [&](auto act) -> int32_t {
    auto launch = [&](auto df, auto ob) -> int32_t {
      constexpr int kAct = decltype(act)::value, kDF = decltype(df)::value, kOB = decltype(ob)::value;
      if (a.i % 8 == 0 && a.o % 8 == 0)
        ABCD_LAUNCH("linear_narrow", (linear_narrow_kernel<T, kAct, kDF, kOB, true>), blocks, kNarrowLayerThreads, 0, stream, a);
      else
        ABCD_LAUNCH("linear_narrow", (linear_narrow_kernel<T, kAct, kDF, kOB, false>), blocks, kNarrowLayerThreads, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    };
    std::integral_constant<int, 2> i2;
    std::integral_constant<int, 4> i4;
    std::integral_constant<int, 8> i8;
    std::integral_constant<int, 16> i16;
    if (a.o > 128) return launch(i4, i16);
    if (a.i > 128) return a.o > 64 ? launch(i8, i8) : launch(i8, i4);
    if (a.o > 64) return launch(i4, i8);
    return a.i > 64 ? launch(i4, i4) : launch(i2, i4);
  });
}

template <typename T>
int32_t run_linear_narrow_bwd(const LinearNarrowBwd& a, int64_t blocks, hipStream_t stream) {
  auto of = [&](auto mode) -> int32_t {
    auto launch = [&](auto df, auto ob) -> int32_t {
      constexpr int kMode = decltype(mode)::value, kDF = decltype(df)::value, kOB = decltype(ob)::value;
      if (a.i % 8 == 0 && a.o % 8 == 0)
        ABCD_LAUNCH("linear_narrow_bwd", (linear_narrow_bwd_kernel<T, kMode, kDF, kOB, true>), blocks, kNarrowLayerThreads, 0,
                    stream, a);
      else
        ABCD_LAUNCH("linear_narrow_bwd", (linear_narrow_bwd_kernel<T, kMode, kDF, kOB, false>), blocks, kNarrowLayerThreads, 0,
                    stream, a);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    };
    std::integral_constant<int, 2> i2;
    std::integral_constant<int, 4> i4;
    std::integral_constant<int, 8> i8;
    if (a.o > 64) return launch(i2, i8);
    return a.i > 64 ? launch(i4, i4) : launch(i2, i4);
  };
  if (a.slope) return of(std::integral_constant<int, kLinearKept>{});
  return with_any_act(a.act, of);
}

}  // namespace

#define ABCD_LINEAR_NARROW(NAME, TYPE)                                                              \
  int32_t linear_narrow_##NAME(const LinearNarrow& a, int64_t blocks, hipStream_t s) {              \
    return run_linear_narrow<TYPE>(a, blocks, s);                                                   \
  }                                                                                                 \
  int32_t linear_narrow_bwd_##NAME(const LinearNarrowBwd& a, int64_t blocks, hipStream_t s) {       \
    return run_linear_narrow_bwd<TYPE>(a, blocks, s);                                               \
  }

}  // namespace abcd
