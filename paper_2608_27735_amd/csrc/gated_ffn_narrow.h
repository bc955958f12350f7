// gated_ffn_narrow.h -- the gated feed-forward block of many narrow rows (one per
// Gaussian), forward and backward in one launch each, for 16-bit element types.
//
// With d and o of a few dozen the products' results outweigh their inputs: h and
// its derivatives alone would be written and read several times what x and y
// take. Here nothing but x, dy, y and dx passes through memory. The matrix
// instruction's result serves as the next one's operand without leaving the
// registers: a lane of a 16 x 16 result holds four consecutive indexes of one side
// and one of the other, so two results side by side are eight indexes of a
// contraction of 32, in an order that the other operand is laid out to match.
//
// Forward: a wave takes kRowFrags x 16 rows at a time; weights lie in LDS in
// fragment order, loaded once per workgroup, and for every 32 columns of h the
// wave makes g and u, h from them, and adds h's part of y.
//
// Backward: a workgroup takes 64 rows at a time, and each of its 8 waves 16 columns
// of h, so that its part of the weights stays in its registers, and so do its parts of
// dWg, dWu and dWd over all rows that the workgroup takes. An h of more than 128
// columns takes a launch for each 128, which pass dx on in fp32. g, u, dh, dg, du and h are made again in registers; only dg and
// du go through LDS, to the waves that make dx, one round later. x and dz are read
// from LDS along for g, u and dh, and across (ds_read_b64_tr_b16) for the weights'
// gradients. The biases' gradients are products with ones. Workgroups write their
// sums in fp32, and a second launch adds these in a fixed order.
//
// 1M rows of 64 x 128 x 64 in bf16, dropout and biases: forward 100 us (256 MB), backward
// 210 (384 MB). Neither memory nor the matrix instructions (20 and 29 percent busy) bound
// them but issue: the forward's vector instructions (activation, generator, conversions;
// 63 percent busy) at four waves a SIMD, the backward's chain of LDS, products,
// activation and products at the two waves that its registers leave room for (vector
// instructions 46 percent busy, LDS about as much). By the tiled products
// the step takes 2,100 us: g, u, h and their gradients through memory.
#pragma once

#include <algorithm>

#include "activation.h"
#include "gated_ffn_args.h"
#include "gemm.h"
#include "load_frag.h"

namespace abcd {
namespace {

template <typename T>
__device__ __forceinline__ typename Frag<T>::type join(f32x4 a, f32x4 b) {
  typename Frag<T>::type r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (T)a[i], r[4 + i] = (T)b[i];
  return r;
}

// m[row][col], 0 outside rows x cols.
template <typename T>
__device__ __forceinline__ T at_or_0(const void* m, int row, int col, int rows, int cols) {
  const bool in = row < rows && col < cols;
  return *(in ? static_cast<const T*>(m) + (int64_t)row * cols + col : reinterpret_cast<const T*>(zeros));
}

constexpr int kNarrowThreads = 512, kNarrowBwdThreads = 512;

// kWhole: d, h and o are multiples of 8. kDF: contractions of 32 that hold d; kOB:
// 16-column blocks of o; kHC: 32-column chunks of h. Registers for the waves whose
// workgroups' weights fit a CU's LDS: two of the smallest shape, one of the others.
template <typename T, int kAct, int kDF, int kOB, int kHC, bool kWhole>
__global__ __launch_bounds__(kNarrowThreads, (kHC * (4 * kDF + kOB) <= 72 ? 4 : 2)) void ffn_narrow_kernel(FfnNarrow a) {
  typedef typename Frag<T>::type F;
  constexpr int kNarrowWaves = kNarrowThreads / 64, kRowFrags = 2, kRows = kRowFrags * 16;
  constexpr int kChunk = 4 * kDF + kOB;  // fragments of a chunk: gate, up, down
  __shared__ __align__(16) F weights[kHC * kChunk * 64];
  __shared__ __align__(16) float bias[2][kHC * 32];
  __shared__ __align__(16) float bias_down[kOB * 16];
  const int d = (int)a.d, h = (int)a.h, o = (int)a.o;
  constexpr int kTurns = kHC * kChunk * 64 / kNarrowThreads;
  static_assert(kHC * kChunk * 64 % kNarrowThreads == 0, "every thread sets up as many");
#pragma unroll 4
  for (int turn = 0; turn < kTurns; ++turn) {
    const int s = turn * kNarrowThreads + threadIdx.x;
    const int l = s & 63, f = s / 64 % kChunk, c = s / 64 / kChunk;
    F v;
    // gate and up: block f / kDF of (gate 0, gate 1, up 0, up 1), contraction f %
    // kDF; down: lane quarter q of block b holds columns q kOB 4 + 4 b .. + 3 of y,
    // so that a lane's blocks are consecutive columns
    const bool in = f < 4 * kDF;
    const T* const w = static_cast<const T*>(in ? (f < 2 * kDF ? a.w_gate : a.w_up) : a.w_down);
    const int i = l & 15;
    const int row = in ? c * 32 + (f / kDF & 1) * 16 + i : (i >> 2) * (kOB * 4) + (f - 4 * kDF) * 4 + (i & 3);
    const int rows = in ? h : o, cols = in ? d : h;
    if (kWhole) {
      // two halves of 4 elements: next to each other, or a block of h apart
      typedef typename VecOf<T, 4>::type V4;
      typedef V4 V4U __attribute__((aligned(sizeof(T))));
      V4 half[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int col = in ? f % kDF * 32 + (l >> 4) * 8 + e * 4 : c * 32 + e * 16 + (l >> 4) * 4;
        half[e] = *reinterpret_cast<const V4U*>(row < rows && col < cols ? w + (int64_t)row * cols + col
                                                                        : reinterpret_cast<const T*>(zeros));
      }
      v = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = at_or_0<T>(w, row, in ? f % kDF * 32 + (l >> 4) * 8 + e : c * 32 + (e >> 2) * 16 + (l >> 4) * 4 + (e & 3),
                          rows, cols);
    }
    weights[s] = v;
  }
  for (int s = threadIdx.x; s < 2 * kHC * 32; s += kNarrowThreads) {
    const int c = s % (kHC * 32);
    const T* b = static_cast<const T*>(s < kHC * 32 ? a.b_gate : a.b_up);
    bias[s / (kHC * 32)][c] = b && c < h ? (float)b[c] : 0.0f;
  }
  if (threadIdx.x < kOB * 16)
    bias_down[threadIdx.x] =
        a.b_down && threadIdx.x < a.o ? (float)static_cast<const T*>(a.b_down)[threadIdx.x] : 0.0f;
  __syncthreads();
  const int l = threadIdx.x & 63, j = l & 15, q = l >> 4;
  const int64_t step = (int64_t)gridDim.x * kNarrowWaves * kRows;
  int64_t r0 = ((int64_t)blockIdx.x * kNarrowWaves + (threadIdx.x >> 6)) * kRows;
  const int chunks = (h + 31) / 32;
  auto fetch = [&](int64_t from, F (&x)[kRowFrags][kDF]) {
#pragma unroll
    for (int x0 = 0; x0 < kRowFrags; ++x0) {
      const int64_t r = from + x0 * 16 + j;
#pragma unroll
      for (int f = 0; f < kDF; ++f) {
        const int c = f * 32 + q * 8;
        x[x0][f] = load_frag<T, kWhole>(static_cast<const T*>(a.x) + r * a.ldx + c, r < a.n ? d - c : 0,
                                        room_of(a.n, r, a.ldx, d - c));
      }
    }
  };
  for (; r0 < a.n; r0 += step) {
    F x[kRowFrags][kDF];
    fetch(r0, x);
#pragma unroll
    for (int i = 0; i < kRowFrags; ++i)
#pragma unroll
      for (int f = 0; f < kDF; ++f) x[i][f] = first_of<T, kWhole>(x[i][f], d - (f * 32 + q * 8));
    F res[kRowFrags][kOB / 2];  // on its way while the products run
    if (a.res)
#pragma unroll
      for (int i = 0; i < kRowFrags; ++i)
#pragma unroll
        for (int b = 0; b < kOB / 2; ++b) {
          const int64_t r = r0 + i * 16 + j;
          const int c = q * (kOB * 4) + b * 8;
          res[i][b] = load_frag<T, kWhole>(static_cast<const T*>(a.res) + r * a.ldr + c, r < a.n ? o - c : 0,
                                           room_of(a.n, r, a.ldr, o - c));
        }
    f32x4 y[kRowFrags][kOB];
#pragma unroll
    for (int i = 0; i < kRowFrags; ++i)
#pragma unroll
      for (int b = 0; b < kOB; ++b) y[i][b] = *reinterpret_cast<const f32x4*>(&bias_down[q * (kOB * 4) + b * 4]);
    for (int c = 0; c < chunks; ++c) {
      const F* w = weights + c * kChunk * 64 + l;
      f32x4 g[kRowFrags][2], u[kRowFrags][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const f32x4 bg = *reinterpret_cast<const f32x4*>(&bias[0][c * 32 + b * 16 + q * 4]);
        const f32x4 bu = *reinterpret_cast<const f32x4*>(&bias[1][c * 32 + b * 16 + q * 4]);
#pragma unroll
        for (int i = 0; i < kRowFrags; ++i) g[i][b] = bg, u[i][b] = bu;
#pragma unroll
        for (int f = 0; f < kDF; ++f) {
          const F wg = w[(b * kDF + f) * 64], wu = w[((2 + b) * kDF + f) * 64];
#pragma unroll
          for (int i = 0; i < kRowFrags; ++i) {
            g[i][b] = mma(wg, x[i][f], g[i][b]);
            u[i][b] = mma(wu, x[i][f], u[i][b]);
          }
        }
      }
      F hid[kRowFrags];
#pragma unroll
      for (int i = 0; i < kRowFrags; ++i) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float slope;
            g[i][b][e] = activate<kAct, true>(g[i][b][e], slope) * u[i][b][e];
          }
        hid[i] = join<T>(g[i][0], g[i][1]);
      }
#pragma unroll
      for (int b = 0; b < kOB; ++b) {
        const F wd = w[(4 * kDF + b) * 64];
#pragma unroll
        for (int i = 0; i < kRowFrags; ++i) y[i][b] = mma(wd, hid[i], y[i][b]);
      }
    }
#pragma unroll
    for (int i = 0; i < kRowFrags; ++i) {
      const int64_t r = r0 + i * 16 + j;
      if (r >= a.n) continue;
#pragma unroll
      for (int b = 0; b < kOB; b += 2) {
        __builtin_amdgcn_sched_barrier(0);  // one at a time, for the registers' sake
        const int c = q * (kOB * 4) + b * 4, left = o - c;
        if (left <= 0) continue;
        Floats<8> v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = y[i][b + e / 4][e % 4];
        uint32_t at = (uint32_t)c;
        asm volatile("" : "+v"(at));  // keeps the generator's first round out of registers between rows
        Floats<8> add = 0.0f;
        if (a.res) add = __builtin_convertvector(res[i][b / 2], Floats<8>);
        v = drop_vec<8>(v, a.key, (uint32_t)r, at, add);
        store_vec<T, 8, kWhole>(static_cast<T*>(a.y) + r * a.ldy + c, v, left);
      }
    }
  }
}

// Rows of 128 bytes in LDS (64 elements): where the 8 bytes of elements 4 unit .. + 3
// of a row lie, so that neither the lanes that read 16 bytes of consecutive rows nor
// those that read 8 bytes across them meet a bank too often.
__device__ __forceinline__ int row_at(int row, int unit) { return row * 128 + (((unit >> 1) ^ (row & 7)) * 16) + (unit & 1) * 8; }
// The same for dg and du, which are written 8 bytes down 16 rows.
__device__ __forceinline__ int turned_at(int row, int unit) {
  return row * 128 + ((unit ^ (((row & 3) << 2) | ((row >> 2) & 3))) * 8);
}

// d and o up to 64. kGroups: 1: h up to 128, each wave all 64 rows; 2: h up to 64, four
// waves the first 32 rows and four the others, with sums of their own. kMore: the launch
// takes up to 128 columns of an h with more.
template <typename T, int kAct, int kGroups, bool kMore, bool kWhole, bool kDrop>
__global__ __launch_bounds__(kNarrowBwdThreads, 2) void ffn_narrow_bwd_kernel(FfnNarrowBwd a) {
  typedef typename Frag<T>::type F;
  constexpr int kTile = 64 * 128, kH = 128 / kGroups;
  __shared__ __align__(16) char xs[2][kTile];        // [64 rows][64 columns]
  __shared__ __align__(16) char zs[2][kTile];
  __shared__ __align__(16) char turned[2][2 * kH * 128];  // [dg, then du: column of h][64 rows]
  const int d = (int)a.d, h = (int)a.h, o = (int)a.o;
  const int l = threadIdx.x & 63, j = l & 15, q = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The weights pass through LDS in tiles of 64 x 64, from which each wave takes its
  // own: as they lie in memory most of them are needed across their rows.
  const int group = wave / (8 / kGroups), first = wave % (8 / kGroups) * 16, col = first + j;  // its columns of h
  F wg[2], wu[2], wd[2];
  f32x4 bg, bu;
  // what it makes of dx: columns xb * 16 .. + 15 of rows xr * 32 .. + 31
  const int xb = wave & 3, xr = wave >> 2;
  F wx[2][kH / 32];
  // thread t brings row t / 8, columns (t & 7) 8 .. + 7 of a block's x and dz
  const int lr = threadIdx.x >> 3, lc = (threadIdx.x & 7) * 8;
  typedef const __attribute__((address_space(3))) F LdsF;
  {
    LdsChar* const t = (LdsChar*)turned[0];  // gate: [kH][64], then up
    LdsChar* const td = (LdsChar*)turned[1];  // down: [kH / 64][64 of o][64 of h]
#pragma unroll
    for (int k = 0; k < kH / 64; ++k) {
      const int row = k * 64 + lr, col = k * 64 + lc;
      const F g = load_first<T, kWhole>(static_cast<const T*>(a.w_gate) + (int64_t)row * d + lc, row < h ? d - lc : 0,
                                           room_of(h, row, d, d - lc));
      const F u = load_first<T, kWhole>(static_cast<const T*>(a.w_up) + (int64_t)row * d + lc, row < h ? d - lc : 0,
                                           room_of(h, row, d, d - lc));
      const F w = load_first<T, kWhole>(static_cast<const T*>(a.w_down) + (int64_t)lr * a.ldd + col, lr < o ? h - col : 0,
                                           room_of(o, lr, a.ldd, h - col));
      const int at = row_at(lr, lc / 4) + k * kTile;
      *(__attribute__((address_space(3))) F*)(t + at) = g;
      *(__attribute__((address_space(3))) F*)(t + kH * 128 + at) = u;
      *(__attribute__((address_space(3))) F*)(td + at) = w;
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      wg[f] = *(LdsF*)(t + row_at(col, f * 8 + q * 2));
      wu[f] = *(LdsF*)(t + kH * 128 + row_at(col, f * 8 + q * 2));
      const int row = f * 32 + q * 8 + (j >> 2), unit = (first & 63) / 4 + (j & 3);
      wd[f] = read_across<T>(td + first / 64 * kTile + row_at(row, unit), td + first / 64 * kTile + row_at(row + 4, unit));
    }
    bg = a.b_gate ? (float)at_or_0<T>(a.b_gate, 0, col, 1, h) : 0.0f;
    bu = a.b_up ? (float)at_or_0<T>(a.b_up, 0, col, 1, h) : 0.0f;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int k = 0; k < kH / 32; ++k) {
        const int row = k * 32 + q * 8 + (j >> 2), unit = xb * 4 + (j & 3);
        LdsChar* const from = t + s * kH * 128;
        wx[s][k] = read_across<T>(from + row_at(row, unit), from + row_at(row + 4, unit));
      }
    __syncthreads();
  }
  f32x4 dwg[4], dwu[4], dwd[4], sg = 0.0f, su = 0.0f, sz = 0.0f;
#pragma unroll
  for (int k = 0; k < 4; ++k) dwg[k] = dwu[k] = dwd[k] = 0.0f;
  F ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (T)1.0f;

  F nx, nz;
  auto fetch = [&](int64_t block) {
    const int64_t r = block * 64 + lr;
    nx = load_frag<T, kWhole>(static_cast<const T*>(a.x) + r * a.ldx + lc, r < a.n ? d - lc : 0,
                              room_of(a.n, r, a.ldx, d - lc));
    nz = load_frag<T, kWhole>(static_cast<const T*>(a.dy) + r * a.lddy + lc, r < a.n ? o - lc : 0,
                              room_of(a.n, r, a.lddy, o - lc));
  };
  // dz of a block: what the forward kept of dy; the factor comes with the sums, at
  // the end
  auto put = [&](int64_t block, int into) {
    if (kDrop) {
      typedef uint32_t U4 __attribute__((ext_vector_type(4)));
      const uint4 m = drop_masks(a.key, (uint32_t)(block * 64 + lr), lc);
      nz = __builtin_bit_cast(F, __builtin_bit_cast(U4, nz) & U4{m.x, m.y, m.z, m.w});
    }
    nx = first_of<T, kWhole>(nx, d - lc);
    nz = first_of<T, kWhole>(nz, o - lc);
    *reinterpret_cast<F*>(xs[into] + row_at(lr, lc / 4)) = nx;
    *reinterpret_cast<F*>(zs[into] + row_at(lr, lc / 4)) = nz;
  };
  // places in LDS, up to what does not change a swizzle: rows by 16, chunks of h by 32
  int along[2], across[4], read_lo[2], read_hi[2];
#pragma unroll
  for (int f = 0; f < 2; ++f) along[f] = row_at(j, f * 8 + q * 2);
#pragma unroll
  for (int k = 0; k < 4; ++k) across[k] = row_at(q * 4 + (j >> 2), k * 4 + (j & 3));
  const int across_z = row_at(q * 4 + (j >> 2), (wave & 3) * 4 + (j & 3));  // its columns of dbd
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = q * 8 + (j >> 2), unit = (xr * 2 + i) * 4 + (j & 3);
    read_lo[i] = turned_at(row, unit);
    read_hi[i] = turned_at(row + 4, unit);
  }
  f32x4 ax[2], px[2];
  // px: what the columns of h before this launch's made of dx
  auto dx_fetch = [&](int64_t block) {
    if (!kMore) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = block * 64 + xr * 32 + i * 16 + j;
      const int c = xb * 16 + q * 4;
      const bool in = a.dx && a.first > 0 && r >= 0 && r < a.n && c < d;
      px[i] = *reinterpret_cast<const f32x4*>(in ? a.dx_part + r * a.ldp + c : reinterpret_cast<const float*>(zeros));
    }
  };
  // half of dx of a block whose dg and du lie at t
  auto dx_half = [&](const LdsChar* t, int half) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int k = half * kH / 64; k < (half + 1) * kH / 64; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          LdsChar* const at = const_cast<LdsChar*>(t) + (s * kH + k * 32) * 128;
          ax[i] = mma(wx[s][k], read_across<T>(at + read_lo[i], at + read_hi[i]), ax[i]);
        }
  };
  auto dx_store = [&](int64_t block) {
    const int c = xb * 16 + q * 4, left = d - c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = block * 64 + xr * 32 + i * 16 + j;
      if (kMore) ax[i] += px[i];
      if (a.dx && r >= 0 && r < a.n && left > 0) {
        if (kMore && !a.last)
          *reinterpret_cast<f32x4*>(a.dx_part + r * a.ldp + c) = ax[i];
        else
          store_vec<T, 4, kWhole>(static_cast<T*>(a.dx) + r * a.lddx + c, ax[i] * a.scale, left);
      }
    }
  };
  // 32 rows of a block: g, u and dh, from these dg, du and h, which stay in registers
  // for the weights' gradients; dg and du also go to t
  auto half_of = [&](LdsChar* x, LdsChar* z, LdsChar* t, int half) {
    f32x4 vg[2], vu[2], vh[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = (half * 32 + i * 16) * 128;
      f32x4 g = bg, u = bu, dh = 0.0f;
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const F fx = *(LdsF*)(x + row + along[f]);
        const F fz = *(LdsF*)(z + row + along[f]);
        g = mma(fx, wg[f], g);
        u = mma(fx, wu[f], u);
        dh = mma(fz, wd[f], dh);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float slope;
        const float v = activate<kAct, true>(g[e], slope);
        vh[i][e] = v * u[e];
        vg[i][e] = dh[e] * (u[e] * slope);
        vu[i][e] = dh[e] * v;
      }
    }
    const F dg = join<T>(vg[0], vg[1]), du = join<T>(vu[0], vu[1]), hid = join<T>(vh[0], vh[1]);
    typedef typename VecOf<T, 4>::type V4;
    typedef __attribute__((address_space(3))) V4 LdsV4;
    const int unit = half * 8 + q;
    *(LdsV4*)(t + turned_at(col, unit)) = __builtin_shufflevector(dg, dg, 0, 1, 2, 3);
    *(LdsV4*)(t + turned_at(col, unit + 4)) = __builtin_shufflevector(dg, dg, 4, 5, 6, 7);
    *(LdsV4*)(t + turned_at(kH + col, unit)) = __builtin_shufflevector(du, du, 0, 1, 2, 3);
    *(LdsV4*)(t + turned_at(kH + col, unit + 4)) = __builtin_shufflevector(du, du, 4, 5, 6, 7);
    sg = mma(ones, dg, sg);
    su = mma(ones, du, su);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // column 16 k + j, rows half 32 + 4 q .. + 3 and 16 further on
      const int at = half * 32 * 128 + across[k];
      const F fx = read_across<T>(x + at, x + at + 16 * 128);
      const F fz = read_across<T>(z + at, z + at + 16 * 128);
      dwg[k] = mma(fx, dg, dwg[k]);
      dwu[k] = mma(fx, du, dwu[k]);
      dwd[k] = mma(fz, hid, dwd[k]);
    }
    const int at = half * 32 * 128 + across_z;
    sz = mma(read_across<T>(z + at, z + at + 16 * 128), ones, sz);
  };
  // A block: its own two halves, and dx of the one before, whose dg and du are whole.
  // The buffers do not overlap.
  auto turn = [&](LdsChar* __restrict__ x, LdsChar* __restrict__ z, LdsChar* __restrict__ t,
                  const LdsChar* __restrict__ before) {
    ax[0] = ax[1] = 0.0f;
    dx_half(before, 0);
    if (kGroups == 1) half_of(x, z, t, 0);
    dx_half(before, 1);
    half_of(x, z, t, kGroups == 1 ? 1 : group);
  };

  const int64_t blocks = (a.n + 63) / 64;
  int64_t block = blockIdx.x, last = -1;
  int cur = 0;
  fetch(block);
  put(block, 0);
  for (; block < blocks; block += gridDim.x, cur ^= 1) {
    const int64_t next = block + gridDim.x;
    __syncthreads();  // this block's rows are in LDS, and so are the last one's dg and du
    fetch(next);      // past the end: zeros
    dx_fetch(last);
    turn((LdsChar*)xs[cur], (LdsChar*)zs[cur], (LdsChar*)turned[cur], (LdsChar*)turned[cur ^ 1]);
    dx_store(last);  // the first turn's is of no block: its rows are below 0
    last = block;
    put(next, cur ^ 1);
  }
  __syncthreads();
  dx_fetch(last);
  ax[0] = ax[1] = 0.0f;
  dx_half((LdsChar*)turned[cur ^ 1], 0);
  dx_half((LdsChar*)turned[cur ^ 1], 1);
  dx_store(last);

  // sums: [dWg h x d][dWu h x d][dWd o x h][dbg h][dbu h][dbd o], of all of h
  float* const part = a.part + ((int64_t)blockIdx.x * kGroups + group) * a.sums;
  const int64_t up = a.ldd * d, down = 2 * up, biases = down + a.ldd * o, at = a.first + col;
  if (col < h) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int c = k * 16 + q * 4 + e;
        if (c < d) {
          part[at * d + c] = dwg[k][e] * a.scale;
          part[up + at * d + c] = dwu[k][e] * a.scale;
        }
        if (c < o) part[down + c * a.ldd + at] = dwd[k][e] * a.scale;
      }
    if (q == 0) {
      part[biases + at] = sg[0] * a.scale;
      part[biases + a.ldd + at] = su[0] * a.scale;
    }
  }
  if ((kGroups == 2 || wave < 4) && j == 0 && a.first == 0)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = (wave & 3) * 16 + q * 4 + e;
      if (c < o) part[biases + 2 * a.ldd + c] = sz[e] * a.scale;
    }
}

// The smallest of the compiled shapes that holds the block (narrow_shape), with two
// workgroups a CU or, from 72 KB of weights on, one. By the tiled products the larger
// shapes take two to four times as long: 1M rows of 64 x 384 x 64 724 against 200 us,
// 300,000 of 128 x 192 x 128 183 against 78 (20,000 rows: 20 against 22).
template <typename T>
int32_t run_narrow(const FfnNarrow& a, int64_t blocks, hipStream_t stream) {
  return with_act(a.act, [&](auto act) -> int32_t {
    auto launch = [&](auto df, auto ob, auto hc) -> int32_t {
      constexpr int kAct = decltype(act)::value, kDF = decltype(df)::value, kOB = decltype(ob)::value,
                    kHC = decltype(hc)::value;
      if (a.d % 8 == 0 && a.h % 8 == 0 && a.o % 8 == 0)
        ABCD_LAUNCH("ffn_narrow", (ffn_narrow_kernel<T, kAct, kDF, kOB, kHC, true>), blocks, kNarrowThreads, 0, stream, a);
      else
        ABCD_LAUNCH("ffn_narrow", (ffn_narrow_kernel<T, kAct, kDF, kOB, kHC, false>), blocks, kNarrowThreads, 0, stream, a);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    };
    std::integral_constant<int, 2> i2;
    std::integral_constant<int, 4> i4;
    std::integral_constant<int, 6> i6;
    std::integral_constant<int, 8> i8;
    std::integral_constant<int, 12> i12;
    switch (narrow_shape(a.d, a.h, a.o)) {
      case 1: return launch(i2, i4, i4);
      case 2: return launch(i2, i4, i12);
      case 3: return launch(i4, i4, i6);
      default: return launch(i4, i8, i6);
    }
  });
}

template <typename T>
int32_t run_narrow_bwd(const FfnNarrowBwd& a, int64_t blocks, hipStream_t stream) {
  return with_act(a.act, [&](auto act) -> int32_t {
    constexpr int kAct = decltype(act)::value;
    const bool whole = a.d % 8 == 0 && a.h % 8 == 0 && a.o % 8 == 0;
    auto launch = [&](auto groups, auto more, auto drop) {
      constexpr int kGroups = decltype(groups)::value;
      constexpr bool kMore = decltype(more)::value, kDrop = decltype(drop)::value;
      if (whole)
        ABCD_LAUNCH("ffn_narrow_bwd", (ffn_narrow_bwd_kernel<T, kAct, kGroups, kMore, true, kDrop>), blocks,
                    kNarrowBwdThreads, 0, stream, a);
      else
        ABCD_LAUNCH("ffn_narrow_bwd", (ffn_narrow_bwd_kernel<T, kAct, kGroups, kMore, false, kDrop>), blocks,
                    kNarrowBwdThreads, 0, stream, a);
    };
    auto of = [&](auto drop) {
      if (a.ldd > 128)
        launch(std::integral_constant<int, 1>{}, std::true_type{}, drop);
      else if (narrow_groups(a.ldd) == 1)
        launch(std::integral_constant<int, 1>{}, std::false_type{}, drop);
      else
        launch(std::integral_constant<int, 2>{}, std::false_type{}, drop);
    };
    if (a.key.mode != 0)
      of(std::true_type{});
    else
      of(std::false_type{});
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

}  // namespace

#define ABCD_FFN_NARROW(NAME, TYPE)                                                                                  \
  int32_t ffn_narrow_##NAME(const FfnNarrow& a, int64_t blocks, hipStream_t s) { return run_narrow<TYPE>(a, blocks, s); } \
  int32_t ffn_narrow_bwd_##NAME(const FfnNarrowBwd& a, int64_t blocks, hipStream_t s) {                              \
    return run_narrow_bwd<TYPE>(a, blocks, s);                                                                       \
  }

}  // namespace abcd
