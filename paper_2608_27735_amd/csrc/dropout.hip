// dropout.hip -- dropout from a counter-based generator, and its gradient.
//
// y = residual + keep x / (1 - p), keep from Philox 4x32-7 at (row, column)
// (rows.h): the mask is a function of seed, offset and place, so the gradient is
// the same call on dy and no mask is stored. Bytes bound it: x and residual read
// once, y written once. A thread takes 16 bytes of a row (two blocks of the
// generator in 16-bit types, one in 32), columns along the lanes. 1M x 64 in bf16
// with a residual: 68 us, 5.7 TB/s; the generator's seven rounds, two 32-bit products
// each with a high half, take about half as long in the vector units and are hidden.
#include <algorithm>

#include "load_frag.h"

namespace abcd {
namespace {

struct DropArgs {
  const void* x;
  const void* res;
  void* y;
  int64_t ldx, ldr, ldy, n;
  int d, lanes;  // lanes: threads along a row, a power of two that divides kBlock
  DropKey key;
};

template <typename T, bool kWhole>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropArgs a) {
  constexpr int N = kPer16<T>;
  const int t = threadIdx.x & (a.lanes - 1), rows = kBlock / a.lanes;
  for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / a.lanes; row < a.n;
       row += (int64_t)gridDim.x * rows) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* res = a.res ? static_cast<const T*>(a.res) + row * a.ldr : nullptr;
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    for (int c = t * N; c < a.d; c += a.lanes * N) {
      const int left = a.d - c;
      // (what lies behind the row is not stored)
      const typename Frag<T>::type v = load_frag<T, kWhole>(x + c, left, room_of(a.n, row, a.ldx, left));
      Floats<N> r = 0.0f;
      if (res) r = __builtin_convertvector((load_frag<T, kWhole>(res + c, left, room_of(a.n, row, a.ldr, left))), Floats<N>);
      store_vec<T, N, kWhole>(y + c, drop_vec<N>(__builtin_convertvector(v, Floats<N>), a.key, (uint32_t)row, (uint32_t)c, r), a.d - c);
    }
  }
}

}  // namespace

int32_t launch_dropout(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx, const void* residual,
                       int64_t ldr, void* y, int64_t ldy, double p, uint64_t seed, uint64_t offset,
                       hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  DropArgs a{x, residual, y, ldx, ldr, ldy, n, (int)d, 0, drop_key(p, seed, offset)};
  return with_type(dtype, [&](auto z) -> int32_t {
    typedef decltype(z) T;
    const int nvec = (int)((d + kPer16<T> - 1) / kPer16<T>);
    // the most threads along a row that leave the fewest idle in its last round;
    // eight at least where the row has them, so that a wave's accesses cover lines
    int best = 1 << 30;
    for (int l = nvec >= 8 ? 8 : 1; l <= kBlock; l *= 2) {
      const int used = (nvec + l - 1) / l * l;
      if (used <= best) best = used, a.lanes = l;
    }
    const int64_t rows = kBlock / a.lanes;
    const int64_t blocks = std::min<int64_t>((n + rows - 1) / rows, 1 << 20);
    if (d % kPer16<T> == 0)
      ABCD_LAUNCH("dropout", (dropout_kernel<T, true>), blocks, kBlock, 0, stream, a);
    else
      ABCD_LAUNCH("dropout", (dropout_kernel<T, false>), blocks, kBlock, 0, stream, a);
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

}  // namespace abcd
