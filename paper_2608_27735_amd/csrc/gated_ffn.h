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
// them; else 128 x 128 by 4 waves of 64 x 64.
struct Big {
  static constexpr int TX = 256, TW = 256, WX = 2, WW = 4;
};
struct Small {
  static constexpr int TX = 128, TW = 128, WX = 2, WW = 2;
};

template <typename T, typename Cfg, bool kXAlong, bool kWAlong, bool kHalves>
using ProductOf = Product<T, Cfg::TX, Cfg::TW, Cfg::WX, Cfg::WW, kXAlong, kWAlong, kHalves>;

#define ABCD_TILE_LDS(P)                    \
  __shared__ __align__(16) char tile0[P::kLdsBytes]; \
  __shared__ __align__(16) char tile1[P::kLdsBytes]; \
  LdsChar* const lds0 = (LdsChar*)tile0;    \
  LdsChar* const lds1 = (LdsChar*)tile1

template <typename T>
__device__ __forceinline__ f32x4 load4(const void* p, int64_t at, int64_t n) {
  return load_vec<T, 4, false>(static_cast<const T*>(p) + at, n > 4 ? 4 : (int)n);
}

template <typename T, typename Cfg, int kAct>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_in_kernel(FfnIn a) {
  typedef ProductOf<T, Cfg, true, true, true> P;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * (Cfg::TW / 2);
  P p;
  p.template run<1>(a.x, a.w, ix, iw, 0, a.d, lds0, lds1);
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int w = 0; w < P::FW / 2; ++w) {
    const int64_t c = iw + P::unit_w(w) * 16 + (l >> 4) * 4;
    if (c >= a.ldh) continue;
    f32x4 bg = 0.0f, bu = 0.0f;
    if (a.bg && c < a.h) bg = load4<T>(a.bg, c, a.h - c);
    if (a.bu && c < a.h) bu = load4<T>(a.bu, c, a.h - c);
#pragma unroll
    for (int x = 0; x < P::FX; ++x) {
      __builtin_amdgcn_sched_barrier(0);  // one fragment's addresses and values at a time
      const int64_t r = ix + P::unit_x(x) * 16 + (l & 15);
      if (r >= a.x.len) continue;
      f32x4 g = p.acc[x][w] + bg, u = p.acc[x][w + P::FW / 2] + bu, h, hg, hu;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (c + i >= a.h) g[i] = u[i] = 0.0f;  // the padding, which products read
        float slope;
        hu[i] = activate<kAct>(g[i], slope);
        h[i] = hu[i] * u[i];
        hg[i] = slope * u[i];
      }
      const int64_t at = r * a.ldh + c;
      store_vec<T, 4, true>(static_cast<T*>(a.hidden) + at, h, 4);
      if (a.by_gate) {
        store_vec<T, 4, true>(static_cast<T*>(a.by_gate) + at, hg, 4);
        store_vec<T, 4, true>(static_cast<T*>(a.by_up) + at, hu, 4);
      }
    }
  }
}

template <typename T, typename Cfg>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_out_kernel(FfnOut a) {
  typedef ProductOf<T, Cfg, true, true, false> P;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * Cfg::TW;
  P p;
  p.template run<1>(a.hidden, a.w, ix, iw, 0, a.h, lds0, lds1);
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int w = 0; w < P::FW; ++w) {
    const int64_t c = iw + P::unit_w(w) * 16 + (l >> 4) * 4, left = a.o - c;
    if (left <= 0) continue;
    f32x4 b = 0.0f;
    if (a.bias) b = load4<T>(a.bias, c, left);
#pragma unroll
    for (int x = 0; x < P::FX; ++x) {
      __builtin_amdgcn_sched_barrier(0);  // one fragment's addresses and values at a time
      const int64_t r = ix + P::unit_x(x) * 16 + (l & 15);
      if (r >= a.hidden.len) continue;
      f32x4 y = 0.0f;
      if (a.res) y = load4<T>(a.res, r * a.ldr + c, left);
      y = drop_vec<4>(p.acc[x][w] + b, a.key, (uint32_t)r, (uint32_t)c, y);
      store_vec<T, 4, false>(static_cast<T*>(a.y) + r * a.ldy + c, y, (int)(left > 4 ? 4 : left));
    }
  }
}

template <typename T, typename Cfg>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_dhidden_kernel(FfnDHidden a) {
  typedef ProductOf<T, Cfg, true, false, false> P;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * Cfg::TW;
  P p;
  p.template run<1>(a.dz, a.w, ix, iw, 0, a.o, lds0, lds1);
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int w = 0; w < P::FW; ++w) {
    const int64_t c = iw + P::unit_w(w) * 16 + (l >> 4) * 4;
    if (c >= a.ldh) continue;
#pragma unroll
    for (int x = 0; x < P::FX; ++x) {
      __builtin_amdgcn_sched_barrier(0);  // one fragment's addresses and values at a time
      const int64_t r = ix + P::unit_x(x) * 16 + (l & 15);
      if (r >= a.dz.len) continue;
      const int64_t at = r * a.ldh + c;
      const f32x4 hg = load_vec<T, 4, true>(static_cast<const T*>(a.by_gate) + at, 4);
      const f32x4 hu = load_vec<T, 4, true>(static_cast<const T*>(a.by_up) + at, 4);
      f32x4 dg, du;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float dh = p.acc[x][w][i] * a.scale;
        const bool in = c + i < a.h;
        dg[i] = in ? dh * hg[i] : 0.0f;
        du[i] = in ? dh * hu[i] : 0.0f;
      }
      store_vec<T, 4, true>(static_cast<T*>(a.dgate) + at, dg, 4);
      store_vec<T, 4, true>(static_cast<T*>(a.dup) + at, du, 4);
    }
  }
}

template <typename T, typename Cfg>
__global__ __launch_bounds__(Cfg::WX* Cfg::WW * 64, 2) void ffn_dx_kernel(FfnDX a) {
  typedef ProductOf<T, Cfg, true, false, false> P;
  ABCD_TILE_LDS(P);
  int tx, tw;
  tile_of(blockIdx.x, a.tiles_x, a.tiles_w, tx, tw);
  const int64_t ix = (int64_t)tx * Cfg::TX, iw = (int64_t)tw * Cfg::TW;
  P p;
  p.template run<2>(a.dgu, a.w, ix, iw, 0, a.h, lds0, lds1);
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int w = 0; w < P::FW; ++w) {
    const int64_t c = iw + P::unit_w(w) * 16 + (l >> 4) * 4, left = a.d - c;
    if (left <= 0) continue;
#pragma unroll
    for (int x = 0; x < P::FX; ++x) {
      __builtin_amdgcn_sched_barrier(0);  // one fragment's addresses and values at a time
      const int64_t r = ix + P::unit_x(x) * 16 + (l & 15);
      if (r < a.dgu.len)
        store_vec<T, 4, false>(static_cast<T*>(a.dx) + r * a.lddx + c, p.acc[x][w], (int)(left > 4 ? 4 : left));
    }
  }
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
  p.template run<1>(Side{{m.x, nullptr}, m.ldx, m.rows}, Side{{m.w, nullptr}, m.ldw, m.cols}, ix, iw, k0, k1, lds0,
                    lds1);
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int w = 0; w < P::FW; ++w) {
    const int cw = P::unit_w(w) * 16 + (l >> 4) * 4;
    const int64_t c = iw + cw, left = m.cols - c;
#pragma unroll
    for (int x = 0; x < P::FX; ++x) {
      __builtin_amdgcn_sched_barrier(0);  // one fragment's addresses and values at a time
      const int rx = P::unit_x(x) * 16 + (l & 15);
      if (rest >= 0)
        *reinterpret_cast<f32x4*>(a.part + ((int64_t)rest * Cfg::TX + rx) * Cfg::TW + cw) = p.acc[x][w];
      else if (ix + rx < m.rows && left > 0)
        store_vec<T, 4, false>(static_cast<T*>(m.out) + (ix + rx) * m.cols + c, p.acc[x][w] * m.scale,
                               (int)(left > 4 ? 4 : left));
    }
  }
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

// The big tile where it gives most of the CUs one.
inline bool use_big(int64_t nx, int64_t nw, int tw) { return tiles(nx, Big::TX) * tiles(nw, tw) >= 192; }

#define ABCD_FFN_LAUNCH(label, kernel, a, nx, nw, half, stream, ...)                                      \
  do {                                                                                                    \
    const bool big_ = use_big(nx, nw, Big::TW / (half));                                                  \
    a.tiles_x = (int)tiles(nx, big_ ? Big::TX : Small::TX);                                               \
    a.tiles_w = (int)tiles(nw, (big_ ? Big::TW : Small::TW) / (half));                                    \
    const int64_t grid_ = (int64_t)a.tiles_x * a.tiles_w;                                                 \
    REQUIRE(grid_ < (int64_t(1) << 31), "too many tiles");                                                \
    if (big_)                                                                                             \
      ABCD_LAUNCH(label, (kernel<T, Big __VA_ARGS__>), grid_, Big::WX* Big::WW * 64, 0, stream, a);       \
    else                                                                                                  \
      ABCD_LAUNCH(label, (kernel<T, Small __VA_ARGS__>), grid_, Small::WX* Small::WW * 64, 0, stream, a); \
    ABCD_HIP(hipGetLastError());                                                                          \
  } while (0)

template <typename T>
int32_t run_in(FfnIn a, hipStream_t stream) {
  return with_act(a.act, [&](auto act) -> int32_t {
    ABCD_FFN_LAUNCH("ffn_in", ffn_in_kernel, a, a.x.len, a.h, 2, stream, , decltype(act)::value);
    return ABCD_OK;
  });
}
template <typename T>
int32_t run_out(FfnOut a, hipStream_t stream) {
  ABCD_FFN_LAUNCH("ffn_out", ffn_out_kernel, a, a.hidden.len, a.o, 1, stream);
  return ABCD_OK;
}
template <typename T>
int32_t run_dhidden(FfnDHidden a, hipStream_t stream) {
  ABCD_FFN_LAUNCH("ffn_dhidden", ffn_dhidden_kernel, a, a.dz.len, a.h, 1, stream);
  return ABCD_OK;
}
template <typename T>
int32_t run_dx(FfnDX a, hipStream_t stream) {
  ABCD_FFN_LAUNCH("ffn_dx", ffn_dx_kernel, a, a.dgu.len, a.d, 1, stream);
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
  return big >= 192 ? run_dweight_tiles<T, Big>(a, kBigSlots, stream) : run_dweight_tiles<T, Small>(a, kSmallSlots, stream);
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
