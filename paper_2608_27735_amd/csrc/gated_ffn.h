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
#pragma once

#include <algorithm>

#include "activation.h"
#include "gated_ffn_args.h"
#include "gated_ffn_few.h"
#include "gemm.h"

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

template <typename T, typename Cfg, int kAct>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_in_kernel(FfnIn a) {
  typedef ProductOf<T, Cfg, true, true, true> P;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * (Cfg::TW / 2);
  P p;
  p.template run<1>(a.x, a.w, ix, iw, 0, a.d, lds);
  const int64_t c = iw + P::col_of();
  const bool inside = c < a.ldh;
  Floats<8> bg = 0.0f, bu = 0.0f;
  if (a.bg && c < a.h) bg = load_vec<T, 8, false>(static_cast<const T*>(a.bg) + c, left_of(a.h - c));
  if (a.bu && c < a.h) bu = load_vec<T, 8, false>(static_cast<const T*>(a.bu) + c, left_of(a.h - c));
  p.by_rows(lds, [&](int x, int group, Floats<8> g, Floats<8> u) {
    const int64_t r = ix + P::row_of(x, group);
    if (r >= a.x.len || !inside) return;
    g += bg;
    u += bu;
    Floats<8> h, hg, hu;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (c + i >= a.h) g[i] = u[i] = 0.0f;  // the padding, which products read
      float slope;
      hu[i] = activate<kAct>(g[i], slope);
      h[i] = hu[i] * u[i];
      hg[i] = slope * u[i];
    }
    const int64_t at = r * a.ldh + c;
    store_vec<T, 8, true>(static_cast<T*>(a.hidden) + at, h, 8);
    if (a.by_gate) {
      store_vec<T, 8, true>(static_cast<T*>(a.by_gate) + at, hg, 8);
      store_vec<T, 8, true>(static_cast<T*>(a.by_up) + at, hu, 8);
    }
  });
}

template <typename T, typename Cfg>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_out_kernel(FfnOut a) {
  typedef ProductOf<T, Cfg, true, true, false> P;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * Cfg::TW;
  P p;
  p.template run<1>(a.hidden, a.w, ix, iw, 0, a.h, lds);
  const int64_t c = iw + P::col_of();
  const int left = left_of(a.o - c);
  Floats<8> b = 0.0f;
  if (a.bias && left > 0) b = load_vec<T, 8, false>(static_cast<const T*>(a.bias) + c, left);
  p.by_rows(lds, [&](int x, int group, Floats<8> v) {
    const int64_t r = ix + P::row_of(x, group);
    if (r >= a.hidden.len || left <= 0) return;
    Floats<8> y = 0.0f;
    if (a.res) y = load_vec<T, 8, false>(static_cast<const T*>(a.res) + r * a.ldr + c, left);
    y = drop_vec<8>(v + b, a.key, (uint32_t)r, (uint32_t)c, y);
    store_vec<T, 8, false>(static_cast<T*>(a.y) + r * a.ldy + c, y, left);
  });
}

template <typename T, typename Cfg>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_dhidden_kernel(FfnDHidden a) {
  typedef ProductOf<T, Cfg, true, false, false> P;
  typedef typename VecOf<T, 8>::type V8;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * Cfg::TW;
  P p;
  p.template run<1>(a.dz, a.w, ix, iw, 0, a.o, lds);
  const int64_t c = iw + P::col_of();
  const bool inside = c < a.ldh;
  // h's derivatives, 16 rows ahead
  V8 hg[2][P::kGroups], hu[2][P::kGroups];
  auto fetch = [&](int x) {
#pragma unroll
    for (int g = 0; g < P::kGroups; ++g) {
      const int64_t r = ix + P::row_of(x, g), at = (r < a.dz.len ? r : ix) * a.ldh + (inside ? c : 0);
      hg[x & 1][g] = *reinterpret_cast<const V8*>(static_cast<const T*>(a.by_gate) + at);
      hu[x & 1][g] = *reinterpret_cast<const V8*>(static_cast<const T*>(a.by_up) + at);
    }
  };
  fetch(0);
  p.by_rows(lds, [&](int x, int g, Floats<8> dh) {
    if (g == 0 && x + 1 < P::FX) fetch(x + 1);
    const int64_t r = ix + P::row_of(x, g);
    if (r >= a.dz.len || !inside) return;
    dh *= a.scale;
    Floats<8> dg = dh * __builtin_convertvector(hg[x & 1][g], Floats<8>);
    Floats<8> du = dh * __builtin_convertvector(hu[x & 1][g], Floats<8>);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i >= a.h) dg[i] = du[i] = 0.0f;  // the padding, which products read
    const int64_t at = r * a.ldh + c;
    store_vec<T, 8, true>(static_cast<T*>(a.dgate) + at, dg, 8);
    store_vec<T, 8, true>(static_cast<T*>(a.dup) + at, du, 8);
  });
}

template <typename T, typename Cfg>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_dx_kernel(FfnDX a) {
  typedef ProductOf<T, Cfg, true, false, false> P;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * Cfg::TW;
  P p;
  p.template run<2>(a.dgu, a.w, ix, iw, 0, a.h, lds);
  const int64_t c = iw + P::col_of();
  const int left = left_of(a.d - c);
  p.by_rows(lds, [&](int x, int group, Floats<8> v) {
    const int64_t r = ix + P::row_of(x, group);
    if (r < a.dgu.len && left > 0) store_vec<T, 8, false>(static_cast<T*>(a.dx) + r * a.lddx + c, v, left);
  });
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
  int64_t k0 = 0, k1 = a.n;
  if (rest >= 0) {
    k0 = rest % a.splits * a.per;
    k1 = k0 + a.per < a.n ? k0 + a.per : a.n;
  }
  P p;
  p.template run<1>(Side{{m.x, nullptr}, m.ldx, m.rows}, Side{{m.w, nullptr}, m.ldw, m.cols}, ix, iw, k0, k1, lds);
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

// The big tile where it gives most of the CUs one. (fp32, whose parts are
// made on the way to LDS, has the small one only.)
template <typename T>
bool use_big(int64_t nx, int64_t nw, int tw) {
  return sizeof(T) == 2 && tiles(nx, Big::TX) * tiles(nw, tw) >= 192;
}

#define ABCD_FFN_LAUNCH(label, kernel, Big_, a, nx, nw, half, stream, ...)                                \
  do {                                                                                                    \
    const bool big_ = use_big<T>(nx, nw, Big::TW / (half));                                               \
    a.tiles_x = (int)tiles(nx, big_ ? Big::TX : Small::TX);                                               \
    a.tiles_w = (int)tiles(nw, (big_ ? Big::TW : Small::TW) / (half));                                    \
    const int64_t grid_ = (int64_t)a.tiles_x * a.tiles_w;                                                 \
    REQUIRE(grid_ < (int64_t(1) << 31), "too many tiles");                                                \
    if constexpr (sizeof(T) == 2)                                                                         \
      if (big_)                                                                                           \
        ABCD_LAUNCH(label, (kernel<T, Big_ __VA_ARGS__>), grid_, Big::WX* Big::WW * 64, 0, stream, a);      \
    if (!big_)                                                                                            \
      ABCD_LAUNCH(label, (kernel<T, Small __VA_ARGS__>), grid_, Small::WX* Small::WW * 64, 0, stream, a); \
    ABCD_HIP(hipGetLastError());                                                                          \
  } while (0)

template <typename T>
int32_t run_in(FfnIn a, hipStream_t stream) {
  return with_act(a.act, [&](auto act) -> int32_t {
    ABCD_FFN_LAUNCH("ffn_in", ffn_in_kernel, BigHalves, a, a.x.len, a.h, 2, stream, , decltype(act)::value);
    return ABCD_OK;
  });
}
template <typename T>
int32_t run_out(FfnOut a, hipStream_t stream) {
  ABCD_FFN_LAUNCH("ffn_out", ffn_out_kernel, Big, a, a.hidden.len, a.o, 1, stream);
  return ABCD_OK;
}
template <typename T>
int32_t run_dhidden(FfnDHidden a, hipStream_t stream) {
  ABCD_FFN_LAUNCH("ffn_dhidden", ffn_dhidden_kernel, Big, a, a.dz.len, a.h, 1, stream);
  return ABCD_OK;
}
template <typename T>
int32_t run_dx(FfnDX a, hipStream_t stream) {
  ABCD_FFN_LAUNCH("ffn_dx", ffn_dx_kernel, Big, a, a.dgu.len, a.d, 1, stream);
  return ABCD_OK;
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
  // split so that they make one more, but for at least 512 rows a part.
  const int left = a.tiles % slots;
  a.splits = left == 0 ? 1 : (int)std::min<int64_t>(slots / left, std::max<int64_t>(1, a.n / 512));
  a.whole = a.splits > 1 ? a.tiles - left : a.tiles;
  a.per = ((a.n + a.splits - 1) / a.splits + kStep<T> - 1) / kStep<T> * kStep<T>;
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
