// product.h -- products of any shape from the tiles of gemm.h: which tiles, split
// contractions, and what becomes of the sums.
#pragma once

#include <algorithm>

#include "load_frag.h"

namespace abcd {
namespace {

// Tiles: 256 x 256 by 8 waves, each 128 x 64 of it, where there are enough of
// them; else 128 x 128 by 4 waves of 64 x 64. For two halves of columns the waves lie
// the other way, so that each has 64 columns of both and writes whole lines.
struct Big {
  static constexpr int TX = 256, TW = 256, WX = 2, WW = 4;
};
struct BigHalves {
  static constexpr int TX = 256, TW = 256, WX = 4, WW = 2;
};
struct Small {
  static constexpr int TX = 128, TW = 128, WX = 2, WW = 2;
};

// Of what is left of a row, up to the 8 elements that a lane takes.
__device__ __forceinline__ int left_of(int64_t n) { return n < 8 ? (int)n : 8; }

template <typename T, typename Cfg, bool kXAlong, bool kWAlong, bool kHalves>
using ProductOf = Product<T, Cfg::TX, Cfg::TW, Cfg::WX, Cfg::WW, kXAlong, kWAlong, kHalves>;

#define ABCD_TILE_LDS(P)                            \
  __shared__ __align__(16) char tiles_[P::kLdsBytes]; \
  LdsChar* const lds = (LdsChar*)tiles_

template <typename T>
using V8 = typename VecOf<T, 8>::type;

// 8 elements from p as they are, n of them there (others 0).
template <typename T>
__device__ __forceinline__ V8<T> load8(const void* p, int64_t at, int n) {
  typedef V8<T> V8U __attribute__((aligned(sizeof(T))));
  const T* const q = static_cast<const T*>(p) + at;
  if (n >= 8) return *reinterpret_cast<const V8U*>(q);
  V8<T> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = *(i < n ? q + i : reinterpret_cast<const T*>(zeros));
  return v;
}

// What becomes of each product's sums, 8 consecutive columns of a row at a time:
// column(c) is what a lane keeps of its columns c.., ahead(column, row) what it loads of
// a row before the sums are there, and put(column, row, ahead, sums) writes. Columns from
// end() on do not exist.
template <typename T, typename Cfg, typename End, bool kSplit>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_product_kernel(End e) {
  typedef ProductOf<T, Cfg, End::kXAlong, End::kWAlong, End::kHalves> P;
  ABCD_TILE_LDS(P);
  const Tiling& t = e.a.t;
  int tx, tw;
  tile_of(blockIdx.x, t.tiles_x, t.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * (End::kHalves ? Cfg::TW / 2 : Cfg::TW);
  int begin = 0, end = End::kSegments * steps_of<T>(e.length());
  if (kSplit) {
    begin = blockIdx.y * t.steps;
    end = min(end, begin + t.steps);
  }
  P p;
  p.template run<End::kSegments>(e.x(), e.w(), ix, iw, e.length(), begin, end, lds);
  const int64_t c = iw + P::col_of(), rows = e.rows();
  if constexpr (kSplit) {
    const int64_t pitch = (e.cols() + 7) & ~int64_t(7);
    auto at = [&](int half, int64_t r) {
      return t.part + (((int64_t)blockIdx.y * (End::kHalves ? 2 : 1) + half) * rows + r) * pitch + c;
    };
    if constexpr (End::kHalves)
      p.by_rows(lds, [&](int x, int g, Floats<8> v, Floats<8> v2) {
        const int64_t r = ix + P::row_of(x, g);
        if (r >= rows || c >= pitch) return;
        store_vec<float, 8, true>(at(0, r), v, 8);
        store_vec<float, 8, true>(at(1, r), v2, 8);
      });
    else
      p.by_rows(lds, [&](int x, int g, Floats<8> v) {
        const int64_t r = ix + P::row_of(x, g);
        if (r < rows && c < pitch) store_vec<float, 8, true>(at(0, r), v, 8);
      });
  } else {
    const bool inside = c < e.end();
    const typename End::Column col = e.column(c);
    typename End::Ahead ahead[2][P::kGroups];
    auto fetch = [&](int x) {  // 16 rows ahead
#pragma unroll
      for (int g = 0; g < P::kGroups; ++g) {
        const int64_t r = ix + P::row_of(x, g);
        ahead[x & 1][g] = e.ahead(col, r < rows ? r : ix);
      }
    };
    fetch(0);
    auto put = [&](int x, int g, auto... v) {
      if (g == 0 && x + 1 < P::FX) fetch(x + 1);
      const int64_t r = ix + P::row_of(x, g);
      if (r < rows && inside) e.put(col, r, ahead[x & 1][g], v...);
    };
    p.by_rows(lds, put);
  }
}

// The parts of a split contraction added up in order, and what becomes of the sums: a
// thread for 8 columns of a row.
template <typename End>
__global__ __launch_bounds__(kBlock) void ffn_join_kernel(End e) {
  const int64_t pitch = (e.cols() + 7) & ~int64_t(7), rows = e.rows(), vecs = pitch / 8;
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i >= rows * vecs) return;
  const int64_t r = i / vecs, c = i % vecs * 8;
  const typename End::Column col = e.column(c);
  const typename End::Ahead ahead = e.ahead(col, r);
  Floats<8> v[End::kHalves ? 2 : 1];
#pragma unroll
  for (int k = 0; k < (End::kHalves ? 2 : 1); ++k) {
    const float* p = e.a.t.part + (k * rows + r) * pitch + c;
    v[k] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < e.a.t.splits; ++s)
      v[k] += load_vec<float, 8, true>(p + (int64_t)s * (End::kHalves ? 2 : 1) * rows * pitch, 8);
  }
  if constexpr (End::kHalves)
    e.put(col, r, ahead, v[0], v[1]);
  else
    e.put(col, r, ahead, v[0]);
}

inline int64_t tiles(int64_t len, int tile) { return (len + tile - 1) / tile; }

// The large tile (in 16-bit types: fp32's parts are made on the way to LDS, which has
// room for the small one) where it gives most of the CUs one. A CU holds two of the
// small workgroups but one large, whose end nothing overlaps: after a short contraction,
// or where half of a large tile would lie outside, the small ones win (bf16, 300,000
// rows, K = 128: h Wd' 57 against 95 us, dh 72 against 87; 65,536 rows, K = 1024: 66
// against 55). Not in the first product, whose small tiles have 64 columns of a side
// (the same rows, K = 64 to 192: 5 to 15 percent slower). A split contraction where
// the small ones leave half of the workgroups idle.
// A linear layer's product, which has nothing else to go by, takes the tiles whose rounds over
// the GPU cost less: a round of the small ones is half of the large ones' work at 1.1 times the
// time (bf16, 6,000 x 3,000 to 3,000: 164 against 184 us; 8,192 x 2,048 to 2,048 77 against 71).
template <typename End, typename = void>
struct ByRounds : std::false_type {};
template <typename End>
struct ByRounds<End, std::enable_if_t<End::kByRounds>> : std::true_type {};
inline bool small_rounds(int64_t large, int64_t small) {
  auto rounds = [](int64_t tiles, int64_t slots) { return (tiles + slots - 1) / slots; };
  return 0.55 * (double)rounds(small, kSmallSlots) < (double)rounds(large, kBigSlots);
}

template <typename T, typename End>
int32_t run_product(const char* label, End e, hipStream_t stream) {
  constexpr int kHalf = End::kHalves ? 2 : 1;
  Tiling& t = e.a.t;
  auto deal = [&](auto cfg) -> int64_t {
    typedef decltype(cfg) Cfg;
    t.tiles_x = (int)tiles(e.rows(), Cfg::TX);
    t.tiles_w = (int)tiles(e.cols(), Cfg::TW / kHalf);
    return (int64_t)t.tiles_x * t.tiles_w;
  };
  t.splits = 1;
  const int steps = End::kSegments * steps_of<T>(e.length());
  if constexpr (sizeof(T) == 2) {
    typedef typename End::Large L;
    const int64_t grid = deal(L{});
    const bool others = ByRounds<End>::value && small_rounds(grid, product_tiles(e.rows(), e.cols(), kHalf));
    if (grid >= 192 && !others && (End::kHalves || (steps > 8 && e.cols() > Small::TW))) {
      REQUIRE(grid < (int64_t(1) << 31), "too many tiles");
      ABCD_LAUNCH(label, (ffn_product_kernel<T, L, End, false>), grid, L::WX* L::WW * 64, 0, stream, e);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    }
  }
  const int64_t grid = deal(Small{});
  REQUIRE(grid < (int64_t(1) << 31), "too many tiles");
  t.splits = product_splits(sizeof(T), e.rows(), e.cols(), kHalf, steps);
  if (t.splits == 1) {
    ABCD_LAUNCH(label, (ffn_product_kernel<T, Small, End, false>), grid, Small::WX* Small::WW * 64, 0, stream, e);
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  }
  t.steps = (steps + t.splits - 1) / t.splits;
  ABCD_LAUNCH(label, (ffn_product_kernel<T, Small, End, true>), dim3(grid, t.splits), Small::WX* Small::WW * 64, 0,
              stream, e);
  ABCD_HIP(hipGetLastError());
  const int64_t vecs = e.rows() * ((e.cols() + 7) / 8);
  ABCD_LAUNCH("ffn_join", (ffn_join_kernel<End>), (vecs + kBlock - 1) / kBlock, kBlock, 0, stream, e);
  ABCD_HIP(hipGetLastError());
  return ABCD_OK;
}

}  // namespace
}  // namespace abcd
