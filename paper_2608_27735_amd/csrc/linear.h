// linear.h -- the linear layer's kernels, for one element type (linear_f32.hip,
// linear_f16.hip and linear_bf16.hip each compile them for theirs).
//
//   z = x w' + b, y = res + act(z); dz = dy act'(z), dx = dz w, dw = dz' x, db = sum dz
// Products accumulate in fp32, and bias, activation and residual are applied to the
// accumulators. The backward has act'(z) from the forward (SlopeOf) or makes z again, and
// rounds dz to the element type, as the matrix cores read it, for both products: in two parts it
// would double their matrix instructions. That rounding is as large as the results' own: dx and
// dw have an L2 error of 0.0024 in bf16 and 0.0003 in fp16, where rounding them alone leaves
// 0.0017 and 0.0002. db sums dz before it, but where a product of tiles makes the slopes again.
//
// 8,192 x 2,048 to 2,048 in bf16 with GELU, bias and residual, slopes kept, forward and backward: 242
// to 252 us, by the card. Forward 84 to 89 (770 to 820 TFLOP/s: one round of 256 tiles, whose ends, 15
// to 20 us with activation and three arrays, overlap nothing; small tiles take 6 percent longer), dz
// and the bias's sums 21 (memory), dx 62 to 66 (1,050 to 1,110), dw 65 to 70 and 8 for the sums of its
// two parts (880 to 940 with them).
#pragma once

#include "activation.h"
#include "gated_ffn_few.h"
#include "linear_args.h"
#include "dweight.h"

namespace abcd {
namespace {

template <typename T, int kAct>
struct LinearOutEnd {
  static constexpr bool kXAlong = true, kWAlong = true, kHalves = false;
  static constexpr int kSegments = 1;
  static constexpr bool kByRounds = true;
  typedef Big Large;
  LinearOut a;
  __device__ const Side& x() const { return a.x; }
  __device__ const Side& w() const { return a.w; }
  __host__ __device__ int64_t rows() const { return a.x.len; }
  __host__ __device__ int64_t cols() const { return a.o; }
  __host__ __device__ int64_t end() const { return a.slope ? a.ldslope : a.o; }
  __host__ __device__ int64_t length() const { return a.i; }
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
    v += k.b;
    Floats<8> y, s;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float slope;
      y[e] = activate<kAct, sizeof(T) == 2>(v[e], slope);
      s[e] = e < k.left ? slope : 0.0f;
    }
    if (a.res) y += __builtin_convertvector(f.res, Floats<8>);
    store_vec<T, 8, false>(static_cast<T*>(a.y) + r * a.ldy + k.c, y, k.left);
    if (kAct != ABCD_ACT_NONE && a.slope) store_slopes<8>(static_cast<SlopeOf<T>*>(a.slope) + r * a.ldslope + k.c, s);
  }
};

template <typename T, int kAct>
struct LinearDzEnd {
  static constexpr bool kXAlong = true, kWAlong = true, kHalves = false;
  static constexpr int kSegments = 1;
  static constexpr bool kByRounds = true;
  typedef Big Large;
  LinearDz a;
  __device__ const Side& x() const { return a.x; }
  __device__ const Side& w() const { return a.w; }
  __host__ __device__ int64_t rows() const { return a.x.len; }
  __host__ __device__ int64_t cols() const { return a.o; }
  __host__ __device__ int64_t end() const { return a.lddz; }
  __host__ __device__ int64_t length() const { return a.i; }
  typedef typename LinearOutEnd<T, kAct>::Column Column;
  struct Ahead {
    V8<T> dy;
  };
  __device__ __forceinline__ Column column(int64_t c) const {
    Column k{c, left_of(a.o - c), 0.0f};
    if (a.bias && k.left > 0) k.b = load_vec<T, 8, false>(static_cast<const T*>(a.bias) + c, k.left);
    return k;
  }
  __device__ __forceinline__ Ahead ahead(const Column& k, int64_t r) const {
    return Ahead{load8<T>(a.dy, r * a.lddy + k.c, k.left)};
  }
  __device__ __forceinline__ void put(const Column& k, int64_t r, const Ahead& f, Floats<8> v) const {
    v += k.b;
    const Floats<8> dy = __builtin_convertvector(f.dy, Floats<8>);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float slope;
      activate<kAct, sizeof(T) == 2>(v[e], slope);
      v[e] = e < k.left ? dy[e] * slope : 0.0f;
    }
    store_vec<T, 8, true>(static_cast<T*>(a.dz) + r * a.lddz + k.c, v, 8);
  }
};

template <typename T>
struct LinearDxEnd {
  static constexpr bool kXAlong = true, kWAlong = false, kHalves = false;
  static constexpr int kSegments = 1;
  static constexpr bool kByRounds = true;
  typedef Big Large;
  LinearDx a;
  __device__ const Side& x() const { return a.dz; }
  __device__ const Side& w() const { return a.w; }
  __host__ __device__ int64_t rows() const { return a.dz.len; }
  __host__ __device__ int64_t cols() const { return a.i; }
  __host__ __device__ int64_t end() const { return a.i; }
  __host__ __device__ int64_t length() const { return a.o; }
  struct Column {
    int64_t c;
  };
  struct Ahead {};
  __device__ __forceinline__ Column column(int64_t c) const { return Column{c}; }
  __device__ __forceinline__ Ahead ahead(const Column&, int64_t) const { return Ahead{}; }
  __device__ __forceinline__ void put(const Column& k, int64_t r, const Ahead&, Floats<8> v) const {
    store_vec<T, 8, false>(static_cast<T*>(a.dx) + r * a.lddx + k.c, v, left_of(a.i - k.c));
  }
};

// Few rows: the weights are read once and bound it (gated_ffn_few.h). 8 waves a workgroup where
// rows of the weights are short, else 16 (one row in bf16, weights from memory: 2,048 to 5,632
// 7.6 against 10.0 us, 512 to 1,376 4.3 against 5.3, but 5,632 to 2,048 10.2 against 10.1 and
// 33 rows of 2,048 to 2,048 12.7 against 10.4). kDz: the backward's product made again, and
// the bias's sums (bf16 with SiLU, the whole backward replayed from a graph, against the tiles': one
// row of 512 to 1,376 16.5 against 23.9 us, of 5,632 to 2,048 31.5 against 38.2, 16 rows of 2,048 to
// 2,048 21.4 against 28.0, 32 27.3 against 28.9).
template <typename T, int kAct, int kX, int kWaves, bool kWhole, bool kDz>
__global__ __launch_bounds__(kWaves * 64) void linear_few_kernel(LinearOut a, int columns) {
  f32x4 acc[kX][1], sum[1];
  const int first = blockIdx.x * columns, end = min((int)a.o, first + columns), n = (int)a.x.len;
  const T* const w[1] = {static_cast<const T*>(a.w.p[0])};
  few_products<T, kX, 1, kWaves, kWhole>(acc, static_cast<const T*>(a.x.p[0]), a.x.ld, n, w, a.w.ld, first, end,
                                               (int)a.i);
  if (!few_join<kX, 1, kWaves>(acc, sum)) return;
  const int l = threadIdx.x & 63, r = (threadIdx.x >> 6) * 16 + (l & 15), c = first + (l >> 4) * 4;
  const int left = end - c;
  if (left <= 0 || (!kDz && r >= n)) return;
  if (a.bias) sum[0] += load_vec<T, 4, false>(static_cast<const T*>(a.bias) + c, left);
  f32x4 y, s;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float slope;
    y[e] = activate<kAct, sizeof(T) == 2>(sum[0][e], slope);
    s[e] = e < left ? slope : 0.0f;
  }
  if (kDz) {
    f32x4 dz = 0.0f;
    if (r < n) {
      T* const to = static_cast<T*>(a.y) + r * a.ldy;
      dz = s * load_vec<T, 4, false>(static_cast<const T*>(a.dy) + r * a.lddy + c, left);
      store_vec<T, 4, true>(to + c, dz, 4);
      if (a.o - c <= 4 && c + 4 < a.ldy) store_vec<T, 4, true>(to + c + 4, Floats<4>(0.0f), 4);
    }
    // the bias's sums, of dz before it is rounded: of these 16 rows
    if (a.db || a.part) {
#pragma unroll
      for (int e = 0; e < 4; ++e) dz[e] = lanes_sum<16>(dz[e]);
      if ((l & 15) != 0) return;
      if (a.db)
        store_vec<T, 4, false>(static_cast<T*>(a.db) + c, dz, left);
      else
        store_vec<float, 4, false>(a.part + (threadIdx.x >> 6) * a.o + c, dz, left);
    }
    return;
  }
  if (a.res) y += load_vec<T, 4, false>(static_cast<const T*>(a.res) + r * a.ldr + c, left);
  store_vec<T, 4, false>(static_cast<T*>(a.y) + r * a.ldy + c, y, left);
  if (kAct != ABCD_ACT_NONE && a.slope) {
    SlopeOf<T>* const to = static_cast<SlopeOf<T>*>(a.slope) + r * a.ldslope;
    store_slopes<4>(to + c, s);
    // the columns past o that this lane's four do not reach
    if (a.o - c <= 4 && c + 4 < a.ldslope) store_slopes<4>(to + c + 4, Floats<4>(0.0f));
  }
}

// dz = dy slope, and the sums of its rows: a thread for 8 columns, `lanes` of them next to
// each other, of rows blockIdx.y, + gridDim.y rows.. Without slopes only the sums. (8,192 x 2,048 in
// bf16 20.6 us; with the choice inside the loop, which keeps the loads apart, 25.3.)
template <typename T, bool kSlope>
__global__ __launch_bounds__(kBlock) void linear_slope_kernel(LinearSlope a) {
  __shared__ float red[kBlock * 8];
  const int t = threadIdx.x & (a.lanes - 1), rows = kBlock / a.lanes;
  const int64_t c = ((int64_t)blockIdx.x * a.lanes + t) * 8;
  Floats<8> sum = 0.0f;
  if (c < a.lddz)
#pragma unroll 4
    for (int64_t r = (int64_t)blockIdx.y * rows + threadIdx.x / a.lanes; r < a.n; r += (int64_t)gridDim.y * rows) {
      const Floats<8> dy = __builtin_convertvector(load8<T>(a.dy, r * a.lddy + c, left_of(a.o - c)), Floats<8>);
      Floats<8> v = dy;
      if (kSlope) {
        v *= load_slopes<8>(static_cast<const SlopeOf<T>*>(a.slope) + r * a.ldslope + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < a.o ? v[e] : 0.0f;
        store_vec<T, 8, true>(static_cast<T*>(a.dz) + r * a.lddz + c, v, 8);
      }
      sum += v;
    }
  if (!a.part && !a.db) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) red[threadIdx.x * 8 + e] = sum[e];
  __syncthreads();
  for (int k = threadIdx.x; k < a.lanes * 8; k += kBlock) {
    const int64_t at = (int64_t)blockIdx.x * a.lanes * 8 + k;
    if (at >= a.o) break;
    float v = 0.0f;
    for (int r = 0; r < rows; ++r) v += red[r * a.lanes * 8 + k];
    if (a.db)
      static_cast<T*>(a.db)[at] = (T)v;
    else
      a.part[(int64_t)blockIdx.y * a.o + at] = v;
  }
}

template <typename T>
int32_t run_linear_out(const LinearOut& a, hipStream_t stream) {
  return with_any_act(a.act, [&](auto act) -> int32_t {
    return run_product<T>("linear_out", LinearOutEnd<T, decltype(act)::value>{a}, stream);
  });
}
template <typename T>
int32_t run_linear_dz(const LinearDz& a, hipStream_t stream) {
  return with_any_act(a.act, [&](auto act) -> int32_t {
    return run_product<T>("linear_dz", LinearDzEnd<T, decltype(act)::value>{a}, stream);
  });
}
template <typename T>
int32_t run_linear_dx(const LinearDx& a, hipStream_t stream) {
  return run_product<T>("linear_dx", LinearDxEnd<T>{a}, stream);
}

// Columns a workgroup: those that leave a CU the fewest in turn, one more counted for what each
// workgroup costs (one row in bf16, weights from memory, 8, 12 and 16: 2,048 to 5,632 8.6, 7.6 and
// 8.6 us; 4,096 to 4,096 11.4, 12.2 and 9.8; 2,048 to 2,048 5.1, 5.3 and 5.5; 4 of them 11.9, 16.2
// and 6.1).
inline int few_columns(int64_t o) {
  int best = 0;
  int64_t least = 0;
  for (int columns : {16, 12, 8}) {
    const int64_t takes = ((o + columns - 1) / columns + kCUs - 1) / kCUs * (columns + 1);
    if (best == 0 || takes < least) best = columns, least = takes;
  }
  return best;
}

template <typename T>
int32_t run_linear_few(const LinearOut& a, hipStream_t stream) {
  return with_any_act(a.act, [&](auto act) -> int32_t {
    return with_rows(a.x.len, [&](auto rows) -> int32_t {
      constexpr int kAct = decltype(act)::value, kX = decltype(rows)::value;
      const int columns = few_columns(a.o);
      const int64_t grid = (a.o + columns - 1) / columns;
      auto launch = [&](auto waves, auto dz) {
        constexpr int kWaves = decltype(waves)::value;
        constexpr bool kDz = decltype(dz)::value;
        if (a.i % kPer16<T> == 0)
          ABCD_LAUNCH("linear_few", (linear_few_kernel<T, kAct, kX, kWaves, true, kDz>), grid, kWaves * 64, 0, stream, a, columns);
        else
          ABCD_LAUNCH("linear_few", (linear_few_kernel<T, kAct, kX, kWaves, false, kDz>), grid, kWaves * 64, 0, stream, a, columns);
      };
      auto by_waves = [&](auto dz) {
        if (kX == 1 && a.i * (int64_t)sizeof(T) <= 4096)
          launch(std::integral_constant<int, kX == 1 ? 8 : 16>{}, dz);
        else
          launch(std::integral_constant<int, 16>{}, dz);
      };
      if (kAct != ABCD_ACT_NONE && a.dy)
        by_waves(std::integral_constant<bool, kAct != ABCD_ACT_NONE>{});
      else
        by_waves(std::false_type{});
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    });
  });
}

template <typename T>
int32_t run_linear_slope(const LinearSlope& a, int64_t parts, hipStream_t stream) {
  const dim3 grid((a.lddz / 8 + a.lanes - 1) / a.lanes, parts);
  if (a.slope)
    ABCD_LAUNCH("linear_slope", (linear_slope_kernel<T, true>), grid, kBlock, 0, stream, a);
  else
    ABCD_LAUNCH("linear_slope", (linear_slope_kernel<T, false>), grid, kBlock, 0, stream, a);
  ABCD_HIP(hipGetLastError());
  return ABCD_OK;
}

}  // namespace

#define ABCD_LINEAR_KERNELS(NAME, TYPE)                                                                    \
  int32_t linear_dw_##NAME(const FfnDWeight& a, hipStream_t s) { return run_dweight<TYPE, true>(a, s); }   \
  int32_t linear_out_##NAME(const LinearOut& a, hipStream_t s) { return run_linear_out<TYPE>(a, s); }      \
  int32_t linear_few_##NAME(const LinearOut& a, hipStream_t s) { return run_linear_few<TYPE>(a, s); }      \
  int32_t linear_dz_##NAME(const LinearDz& a, hipStream_t s) { return run_linear_dz<TYPE>(a, s); }         \
  int32_t linear_dx_##NAME(const LinearDx& a, hipStream_t s) { return run_linear_dx<TYPE>(a, s); }         \
  int32_t linear_slope_##NAME(const LinearSlope& a, int64_t parts, hipStream_t s) {                          \
    return run_linear_slope<TYPE>(a, parts, s);                                                            \
  }

}  // namespace abcd
