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
#include "dweight.h"
#include "product.h"

namespace abcd {
namespace {

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
