// gated_ffn.h -- the gated feed-forward block's kernels, for one element type
// (gated_ffn_f32.hip, gated_ffn_f16.hip and gated_ffn_bf16.hip each compile them
// for theirs).
//
//   g = x Wg' + bg, u = x Wu' + bu, h = a(g) u, y = residual + dropout(h Wd' + bd)
// and, with dz = dropout's gradient of dy,
//   dh = dz Wd, dg = dh u a'(g), du = dh a(g), dx = dg Wg + du Wu,
//   dWg = dg' x, dWu = du' x, dWd = dz' h, and the biases' gradients the column sums.
// Five products: both projections in one (a tile holds the same columns of g and
// of u, so h is made from the accumulators), the down projection, dh (whose
// accumulators become dg and du by h's derivatives, which the forward kept), dx as
// one product of twice the contraction, and the weights' gradients, split along
// the rows where the result has too few tiles to fill the GPU. Products accumulate
// in fp32. Between the launches h, dg and du are rounded to the element type, as
// the matrix cores read them, and so are dh/dg = u a'(g) and dh/du = a(g): kept in
// place of g and u they cost as much memory, dg and du take one rounding from each
// instead of two or three, and the backward evaluates no activation. dz is dy with
// zeros, exact; its factor 1 / (1 - p) is applied to the products' fp32 sums.
//
// 8,192 rows of 2,048 x 5,632 x 2,048 in bf16, forward and backward: 1,524 us, 1.12
// PFLOP/s. First product 341 us (1,108 TFLOP/s, with three arrays of 92 MB written), down
// 163 (1,159), dh 215 (879: two such arrays read and two written), dx 298 (1,268), the
// three weights' gradients 477 and 12 for the sums of split tiles (1,159).
#pragma once

#include <algorithm>

#include "activation.h"
#include "gated_ffn_args.h"
#include "gated_ffn_few.h"
#include "gemm.h"
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
template <typename T, int kAct>
struct InEnd {
  static constexpr bool kXAlong = true, kWAlong = true, kHalves = true;
  static constexpr int kSegments = 1;
  typedef BigHalves Large;
  FfnIn a;
  __device__ const Side& x() const { return a.x; }
  __device__ const Side& w() const { return a.w; }
  __host__ __device__ int64_t rows() const { return a.x.len; }
  __host__ __device__ int64_t cols() const { return a.h; }
  __host__ __device__ int64_t end() const { return a.ldh; }
  __host__ __device__ int64_t length() const { return a.d; }
  struct Column {
    int64_t c;
    Floats<8> bg, bu;
  };
  struct Ahead {};
  __device__ __forceinline__ Column column(int64_t c) const {
    Column k{c, 0.0f, 0.0f};
    if (a.bg && c < a.h) k.bg = load_vec<T, 8, false>(static_cast<const T*>(a.bg) + c, left_of(a.h - c));
    if (a.bu && c < a.h) k.bu = load_vec<T, 8, false>(static_cast<const T*>(a.bu) + c, left_of(a.h - c));
    return k;
  }
  __device__ __forceinline__ Ahead ahead(const Column&, int64_t) const { return Ahead{}; }
  __device__ __forceinline__ void put(const Column& k, int64_t r, const Ahead&, Floats<8> g, Floats<8> u) const {
    g += k.bg;
    u += k.bu;
    Floats<8> h, hg, hu;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (k.c + i >= a.h) g[i] = u[i] = 0.0f;  // the padding, which products read
      float slope;
      hu[i] = activate<kAct, sizeof(T) == 2>(g[i], slope);
      h[i] = hu[i] * u[i];
      hg[i] = slope * u[i];
    }
    const int64_t at = r * a.ldh + k.c;
    store_vec<T, 8, true>(static_cast<T*>(a.hidden) + at, h, 8);
    if (a.by_gate) {
      store_vec<T, 8, true>(static_cast<T*>(a.by_gate) + at, hg, 8);
      store_vec<T, 8, true>(static_cast<T*>(a.by_up) + at, hu, 8);
    }
  }
};

template <typename T>
struct OutEnd {
  static constexpr bool kXAlong = true, kWAlong = true, kHalves = false;
  static constexpr int kSegments = 1;
  typedef Big Large;
  FfnOut a;
  __device__ const Side& x() const { return a.hidden; }
  __device__ const Side& w() const { return a.w; }
  __host__ __device__ int64_t rows() const { return a.hidden.len; }
  __host__ __device__ int64_t cols() const { return a.o; }
  __host__ __device__ int64_t end() const { return a.o; }
  __host__ __device__ int64_t length() const { return a.h; }
  struct Column {
    int64_t c;
    int left;
    Floats<8> b;
  };
  struct Ahead {
    V8<T> res;
  };
  __device__ __forceinline__ Column column(int64_t c) const {
    Column k{c, left_of(a.o - c), 0.0f};
    if (a.bias && k.left > 0) k.b = load_vec<T, 8, false>(static_cast<const T*>(a.bias) + c, k.left);
    return k;
  }
  __device__ __forceinline__ Ahead ahead(const Column& k, int64_t r) const {
    return Ahead{load8<T>(a.res, r * a.ldr + k.c, a.res ? k.left : 0)};
  }
  __device__ __forceinline__ void put(const Column& k, int64_t r, const Ahead& f, Floats<8> v) const {
    v = drop_vec<8>(v + k.b, a.key, (uint32_t)r, (uint32_t)k.c, __builtin_convertvector(f.res, Floats<8>));
    store_vec<T, 8, false>(static_cast<T*>(a.y) + r * a.ldy + k.c, v, k.left);
  }
};

template <typename T>
struct DHiddenEnd {
  static constexpr bool kXAlong = true, kWAlong = false, kHalves = false;
  static constexpr int kSegments = 1;
  typedef Big Large;
  FfnDHidden a;
  __device__ const Side& x() const { return a.dz; }
  __device__ const Side& w() const { return a.w; }
  __host__ __device__ int64_t rows() const { return a.dz.len; }
  __host__ __device__ int64_t cols() const { return a.h; }
  __host__ __device__ int64_t end() const { return a.ldh; }
  __host__ __device__ int64_t length() const { return a.o; }
  struct Column {
    int64_t c;
  };
  struct Ahead {
    V8<T> hg, hu;
  };
  __device__ __forceinline__ Column column(int64_t c) const { return Column{c}; }
  __device__ __forceinline__ Ahead ahead(const Column& k, int64_t r) const {
    const int64_t at = r * a.ldh + (k.c < a.ldh ? k.c : 0);
    return Ahead{*reinterpret_cast<const V8<T>*>(static_cast<const T*>(a.by_gate) + at),
                 *reinterpret_cast<const V8<T>*>(static_cast<const T*>(a.by_up) + at)};
  }
  __device__ __forceinline__ void put(const Column& k, int64_t r, const Ahead& f, Floats<8> dh) const {
    dh *= a.scale;
    Floats<8> dg = dh * __builtin_convertvector(f.hg, Floats<8>), du = dh * __builtin_convertvector(f.hu, Floats<8>);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k.c + i >= a.h) dg[i] = du[i] = 0.0f;  // the padding, which products read
    const int64_t at = r * a.ldh + k.c;
    store_vec<T, 8, true>(static_cast<T*>(a.dgate) + at, dg, 8);
    store_vec<T, 8, true>(static_cast<T*>(a.dup) + at, du, 8);
  }
};

template <typename T>
struct DXEnd {
  static constexpr bool kXAlong = true, kWAlong = false, kHalves = false;
  static constexpr int kSegments = 2;
  typedef Big Large;
  FfnDX a;
  __device__ const Side& x() const { return a.dgu; }
  __device__ const Side& w() const { return a.w; }
  __host__ __device__ int64_t rows() const { return a.dgu.len; }
  __host__ __device__ int64_t cols() const { return a.d; }
  __host__ __device__ int64_t end() const { return a.d; }
  __host__ __device__ int64_t length() const { return a.h; }
  struct Column {
    int64_t c;
  };
  struct Ahead {};
  __device__ __forceinline__ Column column(int64_t c) const { return Column{c}; }
  __device__ __forceinline__ Ahead ahead(const Column&, int64_t) const { return Ahead{}; }
  __device__ __forceinline__ void put(const Column& k, int64_t r, const Ahead&, Floats<8> v) const {
    store_vec<T, 8, false>(static_cast<T*>(a.dx) + r * a.lddx + k.c, v, left_of(a.d - k.c));
  }
};

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

// Which product a tile of the weights' gradients belongs to, and its place there.
__device__ __forceinline__ const FfnDWeight::One& dweight_at(const FfnDWeight& a, int tile, int& tx, int& tw) {
  int k = 0;
  while (k + 1 < a.count && tile >= a.one[k + 1].first) ++k;
  tile_at(tile - a.one[k].first, a.one[k].tiles_x, a.one[k].tiles_w, tx, tw);
  return a.one[k];
}

template <typename T, typename Cfg>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_dweight_kernel(FfnDWeight a) {
  typedef ProductOf<T, Cfg, false, false, false> P;
  ABCD_TILE_LDS(P);
  const int b = blockIdx.x, rest = b - a.whole;
  const int tile = rest < 0 ? xcd_order(b, a.whole) : a.whole + rest / a.splits;
  int tx, tw;
  const FfnDWeight::One& m = dweight_at(a, tile, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * Cfg::TW;
  int begin = 0, end = steps_of<T>(a.n);
  if (rest >= 0) {
    begin = rest % a.splits * a.steps;
    end = min(end, begin + a.steps);
  }
  P p;
  p.template run<1>(Side{{m.x, nullptr}, m.ldx, m.rows}, Side{{m.w, nullptr}, m.ldw, m.cols}, ix, iw, a.n, begin, end,
                    lds);
  const int cw = P::col_of();
  const int left = left_of(m.cols - (iw + cw));
  p.by_rows(lds, [&](int x, int group, Floats<8> v) {
    const int rx = P::row_of(x, group);
    if (rest >= 0)
      store_vec<float, 8, true>(a.part + ((int64_t)rest * Cfg::TX + rx) * Cfg::TW + cw, v, 8);
    else if (ix + rx < m.rows && left > 0)
      store_vec<T, 8, false>(static_cast<T*>(m.out) + (ix + rx) * m.cols + iw + cw, v * m.scale, left);
  });
}

// Tile blockIdx.x of those that were split: the sum of its parts, rows blockIdx.y 4 ..
// + 3 of it by TW / 4 threads each.
template <typename T, int TX, int TW>
__global__ __launch_bounds__(TW) void ffn_dweight_sum_kernel(FfnDWeight a) {
  int tx, tw;
  const FfnDWeight::One& m = dweight_at(a, a.whole + blockIdx.x, tx, tw);
  const int rx = blockIdx.y * 4 + threadIdx.x / (TW / 4), cw = threadIdx.x % (TW / 4) * 4;
  const int64_t r = (int64_t)tx * TX + rx, c = (int64_t)tw * TW + cw, left = m.cols - c;
  if (r >= m.rows || left <= 0) return;
  const float* part = a.part + ((int64_t)blockIdx.x * a.splits * TX + rx) * TW + cw;
  f32x4 s = 0.0f;
#pragma unroll 4
  for (int k = 0; k < a.splits; ++k) s += *reinterpret_cast<const f32x4*>(part + (int64_t)k * TX * TW);
  store_vec<T, 4, false>(static_cast<T*>(m.out) + r * m.cols + c, s * m.scale, (int)(left > 4 ? 4 : left));
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
    if (grid >= 192 && (End::kHalves || (steps > 8 && e.cols() > Small::TW))) {
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

template <typename T>
int32_t run_in(const FfnIn& a, hipStream_t stream) {
  return with_act(a.act, [&](auto act) -> int32_t {
    return run_product<T>("ffn_in", InEnd<T, decltype(act)::value>{a}, stream);
  });
}
template <typename T>
int32_t run_out(const FfnOut& a, hipStream_t stream) {
  return run_product<T>("ffn_out", OutEnd<T>{a}, stream);
}
template <typename T>
int32_t run_dhidden(const FfnDHidden& a, hipStream_t stream) {
  return run_product<T>("ffn_dhidden", DHiddenEnd<T>{a}, stream);
}
template <typename T>
int32_t run_dx(const FfnDX& a, hipStream_t stream) {
  return run_product<T>("ffn_dx", DXEnd<T>{a}, stream);
}

template <typename T, typename Cfg>
int32_t run_dweight_tiles(FfnDWeight a, int slots, hipStream_t stream) {
  int64_t total = 0;
  for (int i = 0; i < a.count; ++i) {
    a.one[i].tiles_x = (int)tiles(a.one[i].rows, Cfg::TX);
    a.one[i].tiles_w = (int)tiles(a.one[i].cols, Cfg::TW);
    a.one[i].first = (int)total;
    total += (int64_t)a.one[i].tiles_x * a.one[i].tiles_w;
  }
  a.tiles = (int)total;
  // As many tiles whole as make full rounds of the GPU; the rows of the others are
  // split so that they make one more.
  const int left = a.tiles % slots;
  a.splits = left == 0 ? 1 : (int)std::min<int64_t>(slots / left, dweight_splits(steps_of<T>(a.n)));
  a.whole = a.splits > 1 ? a.tiles - left : a.tiles;
  a.steps = (steps_of<T>(a.n) + a.splits - 1) / a.splits;
  const int rest = a.tiles - a.whole;
  ABCD_LAUNCH("ffn_dweight", (ffn_dweight_kernel<T, Cfg>), a.whole + rest * a.splits, Cfg::WX* Cfg::WW * 64, 0, stream,
              a);
  ABCD_HIP(hipGetLastError());
  if (rest > 0) {
    ABCD_LAUNCH("ffn_dweight_sum", (ffn_dweight_sum_kernel<T, Cfg::TX, Cfg::TW>), dim3(rest, Cfg::TX / 4), Cfg::TW, 0,
                stream, a);
    ABCD_HIP(hipGetLastError());
  }
  return ABCD_OK;
}

template <typename T>
int32_t run_dweight(const FfnDWeight& a, hipStream_t stream) {
  int64_t big = 0;
  for (int i = 0; i < a.count; ++i) big += tiles(a.one[i].rows, Big::TX) * tiles(a.one[i].cols, Big::TW);
  if constexpr (sizeof(T) == 2)
    if (big >= 192) return run_dweight_tiles<T, Big>(a, kBigSlots, stream);
  return run_dweight_tiles<T, Small>(a, kSmallSlots, stream);
}

}  // namespace

#define ABCD_FFN_KERNELS(NAME, TYPE)                                                                   \
  int32_t ffn_in_##NAME(const FfnIn& a, hipStream_t s) { return run_in<TYPE>(a, s); }                  \
  int32_t ffn_few_in_##NAME(const FfnIn& a, hipStream_t s) { return run_few_in<TYPE>(a, s); }          \
  int32_t ffn_few_out_##NAME(const FfnOut& a, hipStream_t s) { return run_few_out<TYPE>(a, s); }       \
  int32_t ffn_out_##NAME(const FfnOut& a, hipStream_t s) { return run_out<TYPE>(a, s); }               \
  int32_t ffn_dhidden_##NAME(const FfnDHidden& a, hipStream_t s) { return run_dhidden<TYPE>(a, s); }   \
  int32_t ffn_dx_##NAME(const FfnDX& a, hipStream_t s) { return run_dx<TYPE>(a, s); }                  \
  int32_t ffn_dweight_##NAME(const FfnDWeight& a, hipStream_t s) { return run_dweight<TYPE>(a, s); }

}  // namespace abcd
