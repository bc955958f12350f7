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
//   at place u ^ across_swizzle(k); ds_read_b64_tr_b16 hands each lane four
//   contraction indexes of its column.
// - Fragments are 16 x 16, with W as the matrix instruction's first operand, so
//   that a lane holds four consecutive columns of one row of the result: stores of
//   four elements, and one block of dropout's generator for them.
// - fp32: every number is the sum of three of 8 bits each, the second and third of
//   what rounding left (exact down to 2^-110, where the third part's bits end), and a
//   product the six products of parts that are not below its last bit, on the same matrix
//   instructions with fp32 sums: 96 cycles of a SIMD for what v_mfma_f32_16x16x4_f32
//   takes 256 for. The parts left out are at most 2^-24 of a product, to either side; the
//   instruction's own sum is within an ulp and leans down by 0.1 of one. The parts are
//   made on the way from memory to LDS, through registers. An infinity among the operands
//   gives NaN. (137 x 1,696 x 3,208 x 63, forward and backward: 147 us, with the fp32
//   instruction, and no split contractions, 615.)
//
// What the matrix instructions' rate bounds runs at 1.1 to 1.3 PFLOP/s in bf16, a large
// library product at 1.35: two 256 x 256 tiles of 64 contraction indexes fill the LDS of
// a CU, which so holds one workgroup of 8 waves, and nothing overlaps its first loads and
// its last stores.
#pragma once

#include "gated_ffn_args.h"

namespace abcd {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;
template <typename T>
constexpr int kStep = kStepBytes / (int)sizeof(T);
template <typename T>
__host__ __device__ inline int steps_of(int64_t kn) {
  return (int)((kn + kStep<T> - 1) / kStep<T>);
}

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

__device__ __forceinline__ int across_swizzle(int k) { return (k & 3) | ((k >> 1) & 4); }

// Where this thread's loads of a step come from, as byte offsets from the tile's
// first element (16-bit types).
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
      constexpr int kRowChunks = TILE * (int)sizeof(T) / 16;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int q = i * NT + tid, k = q / kRowChunks, at = q % kRowChunks;
        off[i] = (uint32_t)(k * (int)(ld * sizeof(T)) + (((at >> 1) ^ across_swizzle(k)) * 2 + (at & 1)) * 16);
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

// 16 indexes of one contraction row's units each, four contraction indexes from each
// of two places: a fragment across.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type read_across(LdsChar* lo, LdsChar* hi) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) s16x4 LdsS4;
  const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)lo);
  const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)hi);
  return __builtin_bit_cast(typename Frag<T>::type, (s16x8)__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Fragment `unit` (16 indexes) of half kk of the step.
template <typename T, int TILE, bool kAlong>
__device__ __forceinline__ typename Frag<T>::type read_frag(const LdsChar* lds, int unit, int kk) {
  typedef typename Frag<T>::type F;
  const int l = threadIdx.x & 63;
  if (kAlong) {
    const int row = unit * 16 + (l & 15), c = kk * 4 + (l >> 4);
    return *reinterpret_cast<const __attribute__((address_space(3))) F*>(lds + row * kStepBytes + ((c ^ (l & 7)) * 16));
  }
  constexpr int kRowBytes = TILE * (int)sizeof(T);
  const int k = kk * 32 + (l >> 4) * 8 + ((l & 15) >> 2);
  LdsChar* at = const_cast<LdsChar*>(lds) + k * kRowBytes + ((unit ^ across_swizzle(k)) * 32) + (l & 3) * 8;
  return read_across<T>(at, at + 4 * kRowBytes);
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
template <int TX, int TW, int kWX, int kWW, bool kHalves>
struct Accumulators {
  static constexpr int NT = kWX * kWW * 64;
  static constexpr int FX = TX / kWX / 16, FW = TW / kWW / 16;
  f32x4 acc[FX][FW];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int x = 0; x < FX; ++x)
#pragma unroll
      for (int w = 0; w < FW; ++w) acc[x][w] = 0.0f;
  }

  // The unit of 16 that fragment w of this wave takes of the tile; with halves the
  // first FW / 2 lie in the first one and the others at the same place of the second.
  __device__ __forceinline__ static int unit_w(int w) {
    const int ww = (threadIdx.x >> 6) % kWW;
    if (kHalves) return (w >= FW / 2 ? TW / 32 : 0) + ww * (FW / 2) + w % (FW / 2);
    return ww * FW + w;
  }
  __device__ __forceinline__ static int unit_x(int x) { return (threadIdx.x >> 6) / kWW * FX + x; }

  // The results by rows: f(x, group, v) with 8 consecutive columns, col_of().., of row
  // row_of(x, group) of the tile, eight or more lanes next to each other in a row; with
  // halves f(x, group, v, v2), the same columns of both. The accumulators
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
  static constexpr int kPitch = FW * 64 + 16, kRowsBytes = kWX * kWW * 16 * kPitch;  // of LDS
  template <typename Fn>
  __device__ __forceinline__ void by_rows(LdsChar* lds, const Fn& f) {
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

};

// 16-bit types.
template <typename T, int TX, int TW, int kWX, int kWW, bool kXAlong, bool kWAlong, bool kHalves>
struct Product : Accumulators<TX, TW, kWX, kWW, kHalves> {
  typedef Accumulators<TX, TW, kWX, kWW, kHalves> Base;
  using Base::acc, Base::FW, Base::FX, Base::NT, Base::unit_w, Base::unit_x;
  static constexpr int kStageBytes = (TX + TW) * kStepBytes, kLdsBytes = 2 * kStageBytes;
  static_assert(Base::kRowsBytes <= kLdsBytes, "the waves' rows fit in the tiles' LDS");

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

  // acc = the sum over steps [begin, end) of X and W at the tile's first indexes ix, iw:
  // kSegments contractions of length kn one after the other, each in steps_of(kn) steps.
  // lds: kLdsBytes.
  template <int kSegments>
  __device__ __forceinline__ void run(const Side& X, const Side& W, int64_t ix, int64_t iw, int64_t kn, int begin,
                                      int end, LdsChar* lds) {
    this->clear();
    LdsChar *lds0 = lds, *lds1 = lds + kStageBytes;
    TileLoads<T, TX, kXAlong, NT> lx;
    TileLoads<T, TW, kWAlong, NT> lw;
    lx.init(X.ld);
    lw.init(W.ld);
    const int per = steps_of<T>(kn);
    auto fetch = [&](int s, LdsChar* lds) {
      const int seg = kSegments > 1 && s >= per ? 1 : 0;
      const int64_t k0 = (int64_t)(s - seg * per) * kStep<T>;
      load_tile<T, TX, kXAlong, NT, false>(lx, lds, X.p[seg], nullptr, X.ld, X.len, ix, k0, kn);
      load_tile<T, TW, kWAlong, NT, kHalves>(lw, lds + TX * kStepBytes, W.p[kHalves ? 0 : seg], W.p[1], W.ld, W.len, iw,
                                            k0, kn);
    };
    if (begin < end) fetch(begin, lds0);
    for (int s = begin; s < end; ++s) {
      __syncthreads();  // step s has arrived, and nothing reads the other buffer any more
      turn(fetch, s + 1, s + 1 < end, lds1, lds0);
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

// ------------------------------------------------------------------ fp32

// Three bf16 whose sum is v, of two numbers a word: each what is left, rounded to
// nearest, so that what is left is signed and at most half of the part's last bit. (The
// first not past the largest bf16: a v up to 2^-9 above it would round to infinity.)
struct Parts {
  uint32_t p[3];
};
__device__ __forceinline__ Parts parts_of(float a, float b) {
  typedef VecOf<__bf16, 2>::type B2;
  constexpr float kMost = 0x1.FEp127f;
  Parts r;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    Floats<2> v = {a, b};
    if (i == 0) v = {__builtin_amdgcn_fmed3f(a, -kMost, kMost), __builtin_amdgcn_fmed3f(b, -kMost, kMost)};
    r.p[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, B2));
    if (i < 2) {
      a -= __uint_as_float(r.p[i] << 16);
      b -= __uint_as_float(r.p[i] & 0xFFFF0000u);
    }
  }
  return r;
}

// One side's loads of a step of 32, 16 bytes (4 numbers) each, and where their parts go
// in LDS: planes of TILE x 64 bytes. Along: rows of 32 elements whose 16-byte chunk c
// lies at place c ^ ((row >> 1) & 3); across: as in 16 bits.
template <int TILE, bool kAlong, int NT, bool kHalves>
struct PartLoads {
  static constexpr int kLoads = TILE * 32 / 4 / NT, kPlane = TILE * 64;
  uint32_t off[kLoads];
  int at[kLoads];
  f32x4 v[kLoads];

  __device__ __forceinline__ void init(int64_t ld) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int q = i * NT + threadIdx.x;
      if (kAlong) {
        const int row = q >> 3, c = q & 7, from = kHalves && i >= kLoads / 2 ? row - TILE / 2 : row;
        off[i] = (uint32_t)(from * (int)(ld * 4) + c * 16);
        at[i] = row * 64 + (((c >> 1) ^ ((row >> 1) & 3)) * 16) + (c & 1) * 8;
      } else {
        const int k = q / (TILE / 4), c = q % (TILE / 4);
        off[i] = (uint32_t)(k * (int)(ld * 4) + c * 16);
        at[i] = k * (TILE * 2) + (((c >> 2) ^ across_swizzle(k)) * 32) + (c & 3) * 8;
      }
    }
  }

  // (arguments as load_tile's)
  __device__ __forceinline__ void fetch(const void* p, const void* p2, int64_t ld, int64_t len, int64_t i0, int64_t k0,
                                        int64_t kn) {
    constexpr int kRows = kHalves ? TILE / 2 : TILE;
    const int64_t first = kAlong ? i0 * ld + k0 : k0 * ld + i0, left = len - i0;
    const int rows = (int)(left < kRows ? left : kRows);
    const int ks = (int)(kn - k0 < 32 ? kn - k0 : 32);
    const uint32_t bytes = kAlong ? (uint32_t)((rows - 1) * (int)(ld * 4) + ((ks * 4 + 15) & ~15))
                                  : (uint32_t)((ks - 1) * (int)(ld * 4) + ((rows * 4 + 15) & ~15));
    const bool tail = kAlong && (int)(threadIdx.x & 7) * 4 >= ks;  // past the contraction's end
    auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(static_cast<const float*>(p) + first), 0, bytes,
                                                  0x00020000);
    auto rsrc2 = rsrc;
    if (kHalves)
      rsrc2 = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(static_cast<const float*>(p2) + first), 0, bytes,
                                                0x00020000);
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      v[i] = __builtin_bit_cast(f32x4, (u32x4)__builtin_amdgcn_raw_buffer_load_b128(
                                           kHalves && i >= kLoads / 2 ? rsrc2 : rsrc, tail ? 0x80000000u : off[i], 0, 0));
  }

  __device__ __forceinline__ void put(LdsChar* lds) const {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) u32x2 LdsU2;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const Parts a = parts_of(v[i][0], v[i][1]), b = parts_of(v[i][2], v[i][3]);
#pragma unroll
      for (int k = 0; k < 3; ++k) *(LdsU2*)(lds + k * kPlane + at[i]) = u32x2{a.p[k], b.p[k]};
    }
  }
};

template <int TILE, bool kAlong>
__device__ __forceinline__ Frag<__bf16>::type read_part(const LdsChar* lds, int unit) {
  typedef Frag<__bf16>::type F;
  const int l = threadIdx.x & 63;
  if (kAlong) {
    const int row = unit * 16 + (l & 15);
    return *reinterpret_cast<const __attribute__((address_space(3))) F*>(lds + row * 64 +
                                                                          (((l >> 4) ^ ((row >> 1) & 3)) * 16));
  }
  const int k = (l >> 4) * 8 + ((l & 15) >> 2);
  LdsChar* at = const_cast<LdsChar*>(lds) + k * (TILE * 2) + ((unit ^ across_swizzle(k)) * 32) + (l & 3) * 8;
  return read_across<__bf16>(at, at + 4 * (TILE * 2));
}

template <int TX, int TW, int kWX, int kWW, bool kXAlong, bool kWAlong, bool kHalves>
struct Product<float, TX, TW, kWX, kWW, kXAlong, kWAlong, kHalves> : Accumulators<TX, TW, kWX, kWW, kHalves> {
  typedef Accumulators<TX, TW, kWX, kWW, kHalves> Base;
  using Base::acc, Base::FW, Base::FX, Base::NT, Base::unit_w, Base::unit_x;
  typedef Frag<__bf16>::type F;
  static constexpr int kXBytes = 3 * TX * 64;
  static constexpr int kLdsBytes = kXBytes + 3 * TW * 64;
  static_assert(Base::kRowsBytes <= kLdsBytes, "the waves' rows fit in the tiles' LDS");

  __device__ __forceinline__ void step(const LdsChar* lds) {
    F w[3][FW];
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int i = 0; i < FW; ++i) w[k][i] = read_part<TW, kWAlong>(lds + kXBytes + k * TW * 64, unit_w(i));
#pragma unroll
    for (int x = 0; x < FX; ++x) {
      F f[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) f[k] = read_part<TX, kXAlong>(lds + k * TX * 64, unit_x(x));
      // the smallest products first
#pragma unroll
      for (int sum = 2; sum >= 0; --sum)
#pragma unroll
        for (int k = sum; k >= 0; --k)
#pragma unroll
          for (int i = 0; i < FW; ++i) acc[x][i] = mma(w[k][i], f[sum - k], acc[x][i]);
    }
  }

  template <int kSegments>
  __device__ __forceinline__ void run(const Side& X, const Side& W, int64_t ix, int64_t iw, int64_t kn, int begin,
                                      int end, LdsChar* lds) {
    this->clear();
    PartLoads<TX, kXAlong, NT, false> lx;
    PartLoads<TW, kWAlong, NT, kHalves> lw;
    lx.init(X.ld);
    lw.init(W.ld);
    const int per = steps_of<float>(kn);
    auto fetch = [&](int s) {
      const int seg = kSegments > 1 && s >= per ? 1 : 0;
      const int64_t k0 = (int64_t)(s - seg * per) * 32;
      lx.fetch(X.p[seg], nullptr, X.ld, X.len, ix, k0, kn);
      lw.fetch(W.p[kHalves ? 0 : seg], W.p[1], W.ld, W.len, iw, k0, kn);
    };
    if (begin < end) fetch(begin);
    for (int s = begin; s < end; ++s) {
      __syncthreads();  // nothing reads the last step's parts any more
      lx.put(lds);
      lw.put(lds + kXBytes);
      if (s + 1 < end) fetch(s + 1);
      __syncthreads();
      step(lds);
    }
  }
};

}  // namespace abcd
