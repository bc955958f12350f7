// gemm.h -- tiles of matrix products on the matrix cores, for the gated
// feed-forward block.
//
// A product takes two sides: X, whose index runs along the rows of the result,
// and W, whose index runs along its columns; each is contracted either along its
// rows ("along": element (i, k) at i ld + k) or across them ("across": at
// k ld + i), so no operand is ever transposed in memory. A workgroup computes
// TX x TW elements in steps of kStepBytes of the contraction (64 elements of 16
// bits, 32 of 32): while the matrix cores work on one step's tiles in LDS, the
// next step's are on their way there without passing through registers.
//
// - Loads: raw buffer loads of 16 bytes into LDS. The buffer's bound is set to
//   the last valid element, so rows past either side's end and, across, past the
//   contraction's end come as zeros; along, chunks past the contraction's end
//   are sent out of bounds by their offset.
// - LDS, along: rows of 128 bytes, whose 16-byte chunk c lies at place c ^ (row & 7);
//   the loads fetch the chunk that belongs at their place, and the fragments'
//   16-byte reads meet no bank twice.
// - LDS, across: rows of one contraction index, whose unit u of 16 elements lies
//   at place u ^ across_swizzle(k). In 16 bits ds_read_b64_tr_b16 hands each lane
//   four contraction indexes of its column; in 32 bits the lanes read 4 bytes.
// - Fragments are 16 x 16, with W as the matrix instruction's first operand, so
//   that a lane holds four consecutive columns of one row of the result: stores of
//   four elements, and one block of dropout's generator for them.
// - fp32 uses the same bytes with v_mfma_f32_16x16x4_f32 four times per 16 bytes;
//   the contraction's indexes are taken in another order on both sides alike.
#pragma once

#include "gated_ffn_args.h"

namespace abcd {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;
template <typename T>
constexpr int kStep = kStepBytes / (int)sizeof(T);

// 16 bytes of a lane: 8 elements of 16 bits, or 4 of 32.
template <typename T>
struct Frag {
  typedef typename VecOf<T, kPer16<T>>::type type;
};

__device__ __forceinline__ f32x4 mma(Frag<__bf16>::type w, Frag<__bf16>::type x, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(Frag<_Float16>::type w, Frag<_Float16>::type x, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(Frag<float>::type w, Frag<float>::type x, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], c, 0, 0, 0);
  return c;
}

typedef __attribute__((address_space(3))) void LdsVoid;
typedef __attribute__((address_space(3))) char LdsChar;

__device__ __forceinline__ int across_swizzle16(int k) { return (k & 3) | ((k >> 1) & 4); }
__device__ __forceinline__ int across_swizzle32(int k) { return (k >> 2) & 3; }

// Where this thread's loads of a step come from, as byte offsets from the tile's
// first element.
template <typename T, int TILE, bool kAlong, int NT>
struct TileLoads {
  static constexpr int kLoads = TILE * kStepBytes / 16 / NT;
  uint32_t off[kLoads];
  int chunk;  // along: the 16-byte chunk of its row that this thread loads

  __device__ __forceinline__ void init(int64_t ld) {
    const int tid = threadIdx.x;
    if (kAlong) {
      chunk = (tid & 7) ^ ((tid >> 3) & 7);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        off[i] = (uint32_t)((i * (NT / 8) + (tid >> 3)) * (int)(ld * sizeof(T)) + chunk * 16);
    } else {
      constexpr int kRowChunks = TILE * (int)sizeof(T) / 16, kUnitChunks = (int)sizeof(T);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int q = i * NT + tid, k = q / kRowChunks, at = q % kRowChunks;
        const int sw = sizeof(T) == 2 ? across_swizzle16(k) : across_swizzle32(k);
        off[i] = (uint32_t)(k * (int)(ld * sizeof(T)) + (((at / kUnitChunks) ^ sw) * kUnitChunks + at % kUnitChunks) * 16);
      }
    }
  }
};

// Loads one step's tile into lds. p: the segment's first element of contraction
// index 0 and row 0; i0: the tile's first index; k0, kn: the step's first
// contraction index and the contraction's length. kHalves: the tile's second half
// comes from p2 at the same index.
template <typename T, int TILE, bool kAlong, int NT, bool kHalves>
__device__ __forceinline__ void load_tile(const TileLoads<T, TILE, kAlong, NT>& t, LdsChar* lds, const void* p,
                                          const void* p2, int64_t ld, int64_t len, int64_t i0, int64_t k0,
                                          int64_t kn) {
  constexpr int SZ = sizeof(T), kRows = kHalves ? TILE / 2 : TILE;
  const int64_t first = kAlong ? i0 * ld + k0 : k0 * ld + i0;
  const int64_t left = len - i0;
  const int rows = (int)(left < kRows ? left : kRows);  // at least 1
  uint32_t bytes;
  bool tail = false;
  if (kAlong) {
    const int kb = (int)(((kn - k0) * SZ + 15) & ~15);  // of the last row, from k0 on
    bytes = (uint32_t)((rows - 1) * (int)(ld * SZ) + kb);
    tail = kb < kStepBytes && t.chunk * 16 >= kb;
  } else {
    const int ks = (int)(kn - k0 < kStep<T> ? kn - k0 : kStep<T>);
    bytes = (uint32_t)((ks - 1) * (int)(ld * SZ) + ((rows * SZ + 15) & ~15));
  }
  auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p) + first * SZ), 0, bytes,
                                                0x00020000);
  auto rsrc2 = rsrc;
  if (kHalves)
    rsrc2 = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p2) + first * SZ), 0, bytes,
                                              0x00020000);
  constexpr int kLoads = TileLoads<T, TILE, kAlong, NT>::kLoads;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const bool second = kHalves && i >= kLoads / 2;
    // the second half's rows count from its own first row
    uint32_t off = t.off[second ? i - kLoads / 2 : i];
    if (kAlong && tail) off = 0x80000000u;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(second ? rsrc2 : rsrc, (LdsVoid*)(lds + (i * NT + wave * 64) * 16), 16, off, 0,
                                             0, 0);
  }
}

// Fragment f (16 indexes from unit u0 + f) of half kk of the step.
template <typename T, int TILE, bool kAlong>
__device__ __forceinline__ typename Frag<T>::type read_frag(const LdsChar* lds, int unit, int kk) {
  typedef typename Frag<T>::type F;
  const int l = threadIdx.x & 63;
  if (kAlong) {
    const int row = unit * 16 + (l & 15), c = kk * 4 + (l >> 4);
    return *reinterpret_cast<const __attribute__((address_space(3))) F*>(lds + row * kStepBytes + ((c ^ (l & 7)) * 16));
  }
  constexpr int kRowBytes = TILE * (int)sizeof(T);
  if constexpr (sizeof(T) == 2) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4 LdsS4;
    const int k = kk * 32 + (l >> 4) * 8 + ((l & 15) >> 2);
    LdsChar* at = const_cast<LdsChar*>(lds) + k * kRowBytes + ((unit ^ across_swizzle16(k)) * 32) + (l & 3) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)(at + 4 * kRowBytes));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(F, v);
  } else {
    F v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = kk * 16 + (l >> 4) * 4 + e;
      v[e] = *reinterpret_cast<const __attribute__((address_space(3))) float*>(
          lds + k * kRowBytes + ((unit ^ across_swizzle32(k)) * 64) + (l & 15) * 4);
    }
    return v;
  }
}

// The place in order of workgroup b of `tiles`. Workgroups go round the 8 XCDs, each
// with an L2 of its own: an XCD takes consecutive places.
__device__ __forceinline__ int xcd_order(int b, int tiles) {
  const int q = tiles / 8, r = tiles % 8, xcd = b % 8;
  return xcd * q + (xcd < r ? xcd : r) + b / 8;
}
// The tile at a place: down 8 tiles of X before the next tile of W, so that what runs
// together on an XCD shares both.
__device__ __forceinline__ void tile_at(int place, int tiles_x, int tiles_w, int& tx, int& tw) {
  const int group = place / (8 * tiles_w), g0 = group * 8;
  const int gx = tiles_x - g0 < 8 ? tiles_x - g0 : 8, in = place - g0 * tiles_w;
  tx = g0 + in % gx;
  tw = in / gx;
}
__device__ __forceinline__ void tile_of(int b, int tiles_x, int tiles_w, int& tx, int& tw) {
  tile_at(xcd_order(b, tiles_x * tiles_w), tiles_x, tiles_w, tx, tw);
}

// The accumulators of a wave: fragments x by w of its part of the tile.
// Waves: kWX along X, the others along W.
template <typename T, int TX, int TW, int kWX, int kWW, bool kXAlong, bool kWAlong, bool kHalves>
struct Product {
  static constexpr int NT = kWX * kWW * 64;
  static constexpr int FX = TX / kWX / 16, FW = TW / kWW / 16;
  static constexpr int kLdsBytes = (TX + TW) * kStepBytes;
  f32x4 acc[FX][FW];

  // The unit of 16 that fragment w of this wave takes of the tile; with halves the
  // first FW / 2 lie in the first one and the others at the same place of the second.
  __device__ __forceinline__ static int unit_w(int w) {
    const int ww = (threadIdx.x >> 6) % kWW;
    if (kHalves) return (w >= FW / 2 ? TW / 32 : 0) + ww * (FW / 2) + w % (FW / 2);
    return ww * FW + w;
  }
  __device__ __forceinline__ static int unit_x(int x) { return (threadIdx.x >> 6) / kWW * FX + x; }

  __device__ __forceinline__ void step(const LdsChar* lds) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      typename Frag<T>::type fx[FX], fw[FW];
#pragma unroll
      for (int w = 0; w < FW; ++w) fw[w] = read_frag<T, TW, kWAlong>(lds + TX * kStepBytes, unit_w(w), kk);
#pragma unroll
      for (int x = 0; x < FX; ++x) fx[x] = read_frag<T, TX, kXAlong>(lds, unit_x(x), kk);
#pragma unroll
      for (int x = 0; x < FX; ++x)
#pragma unroll
        for (int w = 0; w < FW; ++w) acc[x][w] = mma(fw[w], fx[x], acc[x][w]);
    }
  }

  // The results by rows: f(x, row, col, v) with 8 consecutive columns col.. of row `row`
  // of the tile, eight or more lanes next to each other in a row; with halves f(x, row,
  // col, v, v2), the same columns of both. kGroups calls for each x. The accumulators
  // pass through LDS 16 rows at a time, each wave by itself: stored as the lanes hold
  // them, 4 columns of each of 16 rows, they would take twice the instructions and touch
  // lines a quarter at a time (an epilogue that reads two arrays and writes two took 64
  // us of a tile's 118).
  static constexpr int kLanes = kHalves ? FW : 2 * FW;  // lanes of a row
  static constexpr int kGroups = 16 * kLanes / 64;
  __device__ __forceinline__ static int row_of(int x, int group) {
    return unit_x(x) * 16 + group * (64 / kLanes) + (threadIdx.x & 63) / kLanes;
  }
  __device__ __forceinline__ static int col_of() {
    return (threadIdx.x >> 6) % kWW * (kLanes * 8) + (threadIdx.x & 63) % kLanes * 8;
  }
  template <typename Fn>
  __device__ __forceinline__ void by_rows(LdsChar* lds, const Fn& f) {
    constexpr int kPitch = FW * 64 + 16;
    static_assert(kWX * kWW * 16 * kPitch <= 2 * kLdsBytes, "the waves' rows fit in the tiles' LDS");
    typedef __attribute__((address_space(3))) f32x4 LdsF4;
    const int l = threadIdx.x & 63;
    LdsChar* const buf = lds + (threadIdx.x >> 6) * 16 * kPitch;
    __syncthreads();  // nothing reads the tiles any more
#pragma unroll
    for (int x = 0; x < FX; ++x) {
#pragma unroll
      for (int w = 0; w < FW; ++w) *(LdsF4*)(buf + (l & 15) * kPitch + w * 64 + (l >> 4) * 16) = acc[x][w];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        LdsChar* const at = buf + (g * (64 / kLanes) + l / kLanes) * kPitch + l % kLanes * 32;
        Floats<8> v[2];
#pragma unroll
        for (int k = 0; k < (kHalves ? 2 : 1); ++k) {
          const f32x4 lo = *(LdsF4*)(at + k * FW * 32), hi = *(LdsF4*)(at + k * FW * 32 + 16);
          v[k] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        if constexpr (kHalves)
          f(x, g, v[0], v[1]);
        else
          f(x, g, v[0]);
      }
    }
  }

  // acc = sum over the segments' contractions [kbeg, kend) of X and W at the tile's
  // first indexes ix, iw. lds0, lds1: kLdsBytes each.
  template <int kSegments>
  __device__ __forceinline__ void run(const Side& X, const Side& W, int64_t ix, int64_t iw, int64_t kbeg, int64_t kend,
                                      LdsChar* lds0, LdsChar* lds1) {
#pragma unroll
    for (int x = 0; x < FX; ++x)
#pragma unroll
      for (int w = 0; w < FW; ++w) acc[x][w] = 0.0f;
    TileLoads<T, TX, kXAlong, NT> lx;
    TileLoads<T, TW, kWAlong, NT> lw;
    lx.init(X.ld);
    lw.init(W.ld);
    const int per = (int)((kend - kbeg + kStep<T> - 1) / kStep<T>), steps = per * kSegments;
    auto fetch = [&](int s, LdsChar* lds) {
      const int seg = kSegments > 1 && s >= per ? 1 : 0;
      const int64_t k0 = kbeg + (int64_t)(s - seg * per) * kStep<T>;
      load_tile<T, TX, kXAlong, NT, false>(lx, lds, X.p[seg], nullptr, X.ld, X.len, ix, k0, kend);
      load_tile<T, TW, kWAlong, NT, kHalves>(lw, lds + TX * kStepBytes, W.p[kHalves ? 0 : seg], W.p[1], W.ld, W.len, iw,
                                            k0, kend);
    };
    if (steps > 0) fetch(0, lds0);
    for (int s = 0; s < steps; ++s) {
      __syncthreads();  // step s has arrived, and nothing reads the other buffer any more
      turn(fetch, s + 1, s + 1 < steps, lds1, lds0);
      LdsChar* const t = lds0;
      lds0 = lds1;
      lds1 = t;
    }
  }

  // One step: the next one's loads, then the products of this one. The buffers do
  // not overlap: only by knowing that does the compiler let the reads of one go
  // ahead while the loads into the other are in flight.
  template <typename Fetch>
  __device__ __forceinline__ void turn(const Fetch& fetch, int next, bool more, LdsChar* __restrict__ into,
                                       const LdsChar* __restrict__ from) {
    if (more) fetch(next, into);
    step(from);
  }
};

}  // namespace abcd
