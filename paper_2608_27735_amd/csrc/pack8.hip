// pack8.hip -- checkpoints of activations in 8 bits: rows written as blocks of 32
// numbers of 8 bits with one exponent each, and read back.
//
// With 2^e the largest power of two that does not exceed the block's largest finite
// magnitude (e at least -120): q = rint(x 2^(6 - e)) between -127 and 127, which
// stands for q 2^(e - 6); what is not finite is q = -128, read back as NaN. The scale is a
// power of two, so that nothing but rint rounds, and q 2^(e - 6) is a number of all
// three element types: a product that takes a checkpoint loses nothing more. The error is
// half a step of 2^(e - 6), at most 1 / 128 of the block's largest magnitude (a whole
// step for what lies above 127.5 steps); 8 bits of floating point would be off by up to
// 1 / 16 of each number.
//
// Bytes bound both ways. A thread takes 16 bytes of a row, and 4 or 8 next to each other
// a block, whose largest magnitude they find by exchanging bits of their registers. 1M x 64 in
// bf16: written 40 us (194 MB, 4.8 TB/s; with the numbers rounded, cut off and put together one
// by one the vector units were 78 percent busy and it took 48), read back 34 (5.7 TB/s).
#include <algorithm>

#include "pack8.h"

namespace abcd {
namespace {

struct PackArgs {
  const void* x;
  void* y;
  int8_t* q;
  uint8_t* e;
  int64_t ld, n;
  int d, blocks, lanes;  // lanes: threads along a row, a power of two
};

// Largest over G consecutive lanes, returned to each.
template <int G>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  auto dpp = [](uint32_t v, auto ctrl) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, false);
  };
  x = max(x, dpp(x, std::integral_constant<int, 0xB1>{}));
  x = max(x, dpp(x, std::integral_constant<int, 0x4E>{}));
  if (G >= 8) x = max(x, dpp(x, std::integral_constant<int, 0x141>{}));
  return x;
}

template <typename T, bool kWhole>
__global__ __launch_bounds__(kBlock) void pack8_kernel(PackArgs a) {
  constexpr int N = kPer16<T>, kLanes = kPackBlock / N;
  const int t = threadIdx.x & (a.lanes - 1), rows = kBlock / a.lanes;
  const int64_t pitch = (int64_t)a.blocks * kPackBlock;
  for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / a.lanes; row < a.n; row += (int64_t)gridDim.x * rows) {
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
    for (int c = t * N; c < pitch; c += a.lanes * N) {
      const int left = a.d - c;
      const typename Frag<T>::type raw = load_first<T, kWhole>(x + c, left, room_of(a.n, row, a.ld, left));
      const Floats<N> v = __builtin_convertvector(raw, Floats<N>);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
      const bool finite = top < 0x7F800000u;
      // infinities and NaN, which no block's exponent takes part of, for all lanes of a wave
      if (__builtin_expect(__any(!finite), 0)) {
        top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t m = __float_as_uint(v[i]) & 0x7FFFFFFFu;
          top = max(top, m < 0x7F800000u ? m : 0u);
        }
      }
      const uint32_t e = max(lanes_max<kLanes>(top) >> 23, (uint32_t)kPackLeast);
      // rint(v 2^(6 - e)) as the low bits of a sum with 1.5 x 2^23; cut off at 127 steps before
      const float up = __uint_as_float((127 + 127 + 6 - e) << 23), most = 127.0f * packed_unit(e);
      uint32_t q[N];
#pragma unroll
      for (int i = 0; i < N; ++i) q[i] = __float_as_uint(fmaf(__builtin_amdgcn_fmed3f(v[i], -most, most), up, 12582912.0f));
      if (__builtin_expect(__any(!finite), 0)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if ((__float_as_uint(v[i]) & 0x7F800000u) == 0x7F800000u) q[i] = 0x80;
      }
      typedef typename VecOf<uint32_t, N / 4>::type Words;
      Words w;
#pragma unroll
      for (int i = 0; i < N / 4; ++i)
        w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0C0C0400u),
                                     __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0C0C0400u), 0x05040100u);
      *reinterpret_cast<Words*>(a.q + row * pitch + c) = w;
      if (t % kLanes == 0) a.e[row * a.blocks + c / kPackBlock] = (uint8_t)e;
    }
  }
}

template <typename T, bool kWhole>
__global__ __launch_bounds__(kBlock) void unpack8_kernel(PackArgs a) {
  constexpr int N = kPer16<T>;
  const int t = threadIdx.x & (a.lanes - 1), rows = kBlock / a.lanes;
  const int64_t pitch = (int64_t)a.blocks * kPackBlock;
  for (int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / a.lanes; row < a.n; row += (int64_t)gridDim.x * rows) {
    T* y = static_cast<T*>(a.y) + row * a.ld;
    for (int c = t * N; c < a.d; c += a.lanes * N) {
      typedef typename VecOf<uint32_t, N / 4>::type Words;
      const Words w = *reinterpret_cast<const Words*>(a.q + row * pitch + c);
      const float unit = packed_unit(a.e[row * a.blocks + c / kPackBlock]);
      Floats<N> v;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = unpacked(w[i / 4], i % 4, unit);
      store_vec<T, N, kWhole>(y + c, v, a.d - c);
    }
  }
}

// Threads along a row of nvec vectors: as many as leave the fewest idle in its last round;
// eight at least where the row has them, so that a wave's accesses cover lines.
int row_lanes(int nvec) {
  int least = 1;
  while (least < 8 && least < nvec) least *= 2;
  int best = 1 << 30, lanes = least;
  for (int l = least; l <= kBlock; l *= 2) {
    const int used = (nvec + l - 1) / l * l;
    if (used <= best) best = used, lanes = l;
  }
  return lanes;
}

}  // namespace

int32_t launch_pack8(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx, int8_t* q, uint8_t* e,
                     hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  PackArgs a{x, nullptr, q, e, ldx, n, (int)d, (int)pack_blocks(d), 0};
  return with_type(dtype, [&](auto z) -> int32_t {
    typedef decltype(z) T;
    a.lanes = std::max(row_lanes(a.blocks * kPackBlock / kPer16<T>), 8);  // those of a block at least
    const int64_t rows = kBlock / a.lanes, blocks = std::min<int64_t>((n + rows - 1) / rows, 1 << 20);
    if (d % kPer16<T> == 0)
      ABCD_LAUNCH("pack8", (pack8_kernel<T, true>), blocks, kBlock, 0, stream, a);
    else
      ABCD_LAUNCH("pack8", (pack8_kernel<T, false>), blocks, kBlock, 0, stream, a);
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

int32_t launch_unpack8(int32_t dtype, int64_t n, int64_t d, const int8_t* q, const uint8_t* e, void* y, int64_t ldy,
                       hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  PackArgs a{nullptr, y, const_cast<int8_t*>(q), const_cast<uint8_t*>(e), ldy, n, (int)d, (int)pack_blocks(d), 0};
  return with_type(dtype, [&](auto z) -> int32_t {
    typedef decltype(z) T;
    a.lanes = row_lanes((int)((d + kPer16<T> - 1) / kPer16<T>));
    const int64_t rows = kBlock / a.lanes, blocks = std::min<int64_t>((n + rows - 1) / rows, 1 << 20);
    if (d % kPer16<T> == 0)
      ABCD_LAUNCH("unpack8", (unpack8_kernel<T, true>), blocks, kBlock, 0, stream, a);
    else
      ABCD_LAUNCH("unpack8", (unpack8_kernel<T, false>), blocks, kBlock, 0, stream, a);
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

}  // namespace abcd
