// dweight.h -- the weights' gradients: products contracted over the rows, which are split
// where the results have too few tiles to fill the GPU.
#pragma once

#include "product.h"

namespace abcd {
namespace {

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
    if (ix + rx >= m.rows || left <= 0) return;
    if (rest >= 0)
      store_vec<float, 8, true>(a.part + ((int64_t)rest * Cfg::TX + rx) * Cfg::TW + cw, v, 8);
    else
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

// The same of a tile of many parts: 64 vectors of four columns a workgroup, the parts dealt
// to its 16 waves (59 x 96 of 512 parts in fp32: 43 us by the kernel above).
template <typename T, int TX, int TW>
__global__ __launch_bounds__(16 * kWave) void dweight_tall_kernel(FfnDWeight a) {
  __shared__ __align__(16) f32x4 red[16][kWave];
  int tx, tw;
  const FfnDWeight::One& m = dweight_at(a, a.whole + blockIdx.x, tx, tw);
  const int w = threadIdx.x / kWave, l = threadIdx.x % kWave, at = ((int)blockIdx.y * kWave + l) * 4;
  const int rx = at / TW, cw = at % TW;
  const int64_t r = (int64_t)tx * TX + rx, c = (int64_t)tw * TW + cw, left = m.cols - c;
  const bool in = r < m.rows && left > 0;
  if (!__syncthreads_or(in)) return;
  f32x4 s = 0.0f;
  if (in) {
    const float* const part = a.part + (int64_t)blockIdx.x * a.splits * TX * TW + at;
    int k = w;
    for (; k + 7 * 16 < a.splits; k += 8 * 16) {
      f32x4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const f32x4*>(part + (int64_t)(k + u * 16) * TX * TW);
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; k < a.splits; k += 16) s += *reinterpret_cast<const f32x4*>(part + (int64_t)k * TX * TW);
  }
  red[w][l] = s;
  __syncthreads();
  if (w != 0 || !in) return;
  for (int v = 1; v < 16; ++v) s += red[v][l];
  store_vec<T, 4, false>(static_cast<T*>(m.out) + r * m.cols + c, s * m.scale, (int)(left > 4 ? 4 : left));
}

// kTall: parts may be added up by the kernel for many of them.
template <typename T, typename Cfg, bool kTall>
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
  if (kTall && rest > 0 && a.splits >= 32) {
    ABCD_LAUNCH("ffn_dweight_sum", (dweight_tall_kernel<T, Cfg::TX, Cfg::TW>), dim3(rest, Cfg::TX * Cfg::TW / (4 * kWave)),
                16 * kWave, 0, stream, a);
    ABCD_HIP(hipGetLastError());
  } else if (rest > 0) {
    ABCD_LAUNCH("ffn_dweight_sum", (ffn_dweight_sum_kernel<T, Cfg::TX, Cfg::TW>), dim3(rest, Cfg::TX / 4), Cfg::TW, 0,
                stream, a);
    ABCD_HIP(hipGetLastError());
  }
  return ABCD_OK;
}

template <typename T, bool kTall = false>
int32_t run_dweight(const FfnDWeight& a, hipStream_t stream) {
  int64_t big = 0;
  for (int i = 0; i < a.count; ++i) big += tiles(a.one[i].rows, Big::TX) * tiles(a.one[i].cols, Big::TW);
  if constexpr (sizeof(T) == 2)
    if (big >= 192) return run_dweight_tiles<T, Big, kTall>(a, kBigSlots, stream);
  return run_dweight_tiles<T, Small, kTall>(a, kSmallSlots, stream);
}

}  // namespace
}  // namespace abcd
