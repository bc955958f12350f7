// sides.h -- how a call's arrays become the sides of products: copies of what 16-byte
// loads cannot take, column sums, and a workspace's pieces.
#pragma once

#include <algorithm>

#include "load_frag.h"

namespace abcd {
namespace {

// Copies of up to five arrays in one launch, each rows of `cols` elements into rows of
// ldd, the rest of each zeroed, with dropout where the key says so: what a product
// reads has to start on 16 bytes, its rows a multiple of that apart, with zeros up to it.
struct Packs {
  struct One {
    const void* src;
    void* dst;
    int64_t ld, ldd, n;
    int cols, lanes, first, blocks;
    DropKey key;
  } one[5];
  int count = 0, blocks = 0;
};

template <typename T>
__global__ __launch_bounds__(kBlock) void pack_rows_kernel(Packs packs) {
  constexpr int N = kPer16<T>;
  int k = 0;
  while (k + 1 < packs.count && (int)blockIdx.x >= packs.one[k + 1].first) ++k;
  const Packs::One& a = packs.one[k];
  const int t = threadIdx.x & (a.lanes - 1), rows = kBlock / a.lanes;
  for (int64_t row = (int64_t)((int)blockIdx.x - a.first) * rows + threadIdx.x / a.lanes; row < a.n;
       row += (int64_t)a.blocks * rows) {
    const T* s = static_cast<const T*>(a.src) + row * a.ld;
    T* d = static_cast<T*>(a.dst) + row * a.ldd;
    for (int c = t * N; c < a.ldd; c += a.lanes * N) {
      const int left = a.cols - c;
      const Floats<N> v =
          __builtin_convertvector((load_first<T, false>(s + c, left, room_of(a.n, row, a.ld, left))), Floats<N>);
      store_vec<T, N, true>(d + c, drop_vec<N>(v, a.key, (uint32_t)row, (uint32_t)c, 0.0f), N);
    }
  }
}

// Column sums of up to three matrices of n rows (blockIdx.z): part[blockIdx.y][first + c]
// = scale times the sum over rows blockIdx.y, + gridDim.y rows.. of m[row][c]. `lanes`
// threads along a row, the workgroup's other threads on other rows.
struct ColumnSums {
  struct One {
    const void* m;
    int64_t ld, first;
    int cols, lanes;
    float scale;
  } one[3];
  float* part;
  int64_t n, cols;  // of all together
};
template <typename T>
__global__ __launch_bounds__(kBlock) void column_sums_kernel(ColumnSums a) {
  constexpr int N = kPer16<T>;
  __shared__ float red[kBlock * N];
  const ColumnSums::One m = a.one[blockIdx.z];
  const int t = threadIdx.x & (m.lanes - 1), rows = kBlock / m.lanes;
  const int c = ((int)blockIdx.x * m.lanes + t) * N;
  if ((int)blockIdx.x * m.lanes * N >= m.cols) return;
  Floats<N> s = 0.0f;
  if (c < m.cols) {
#pragma unroll 4
    for (int64_t row = (int64_t)blockIdx.y * rows + threadIdx.x / m.lanes; row < a.n; row += (int64_t)gridDim.y * rows)
      s += __builtin_convertvector((load_first<T, false>(static_cast<const T*>(m.m) + row * m.ld + c, m.cols - c,
                                                         room_of(a.n, row, m.ld, m.cols - c))),
                                   Floats<N>);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) red[threadIdx.x * N + i] = s[i];
  __syncthreads();
  for (int i = threadIdx.x; i < m.lanes * N; i += kBlock) {
    const int64_t at = (int64_t)blockIdx.x * m.lanes * N + i;
    if (at >= m.cols) break;
    float v = 0.0f;
    for (int r = 0; r < rows; ++r) v += red[r * m.lanes * N + i];
    a.part[(int64_t)blockIdx.y * a.cols + m.first + at] = v * m.scale;
  }
}

inline int lanes_for(int nvec) {
  int l = 1;
  while (l < kBlock && l < nvec) l *= 2;
  return l;
}

inline int64_t sum_parts_of(int64_t n) { return std::max<int64_t>(1, std::min<int64_t>((n + 63) / 64, 256)); }

// The column sums of up to three matrices of n rows, in two launches. part: sum_parts_of(n)
// parts of all columns.
struct SumCall {
  int32_t dtype;
  int64_t n;
  float* part;
  ColumnSums cs{};
  SumOuts outs{};
  int64_t widest = 0;

  SumCall(int32_t dtype, int64_t n, float* part) : dtype(dtype), n(n), part(part) {}
  void add(void* out, const void* m, int64_t ld, int64_t cols, float factor) {
    if (!out) return;
    const int per16 = 16 / (int)type_bytes(dtype);
    const int lanes = std::min(lanes_for((int)((cols + per16 - 1) / per16)), 64);
    cs.one[outs.count] = ColumnSums::One{m, ld, cs.cols, (int)cols, lanes, factor};
    outs.add(out, cols);
    cs.cols += cols;
    widest = std::max<int64_t>(widest, (cols + lanes * per16 - 1) / (lanes * per16));
  }
  int32_t launch(hipStream_t stream) {
    if (outs.count == 0) return ABCD_OK;
    const int64_t parts = sum_parts_of(n);
    cs.part = part;
    cs.n = n;
    TRY_STATUS(with_type(dtype, [&](auto z) -> int32_t {
      ABCD_LAUNCH("column_sums", (column_sums_kernel<decltype(z)>), dim3(widest, parts, outs.count), kBlock, 0, stream,
                  cs);
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    }));
    return launch_sum_parts(part, parts, outs, dtype, stream);
  }
};

inline void add_pack(Packs& p, int32_t dtype, int64_t n, int64_t cols, const void* src, int64_t ld, void* dst, int64_t ldd,
              const DropKey& key) {
  const int lanes = lanes_for((int)(ldd * (int64_t)type_bytes(dtype) / 16));
  const int64_t rows = kBlock / lanes;
  const int blocks = (int)std::min<int64_t>((n + rows - 1) / rows, 1 << 20);
  p.one[p.count++] = Packs::One{src, dst, ld, ldd, n, (int)cols, lanes, p.blocks, blocks, key};
  p.blocks += blocks;
}

inline int32_t launch(const Packs& p, int32_t dtype, hipStream_t stream) {
  if (p.blocks == 0) return ABCD_OK;
  return with_type(dtype, [&](auto z) -> int32_t {
    ABCD_LAUNCH("pack_rows", (pack_rows_kernel<decltype(z)>), p.blocks, kBlock, 0, stream, p);
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

inline int64_t up8(int64_t v) { return (v + 7) & ~int64_t(7); }

// Whether products can read rows of `cols` elements at p, ld apart, as they are.
inline bool direct(int32_t dtype, const void* p, int64_t cols, int64_t ld) {
  const size_t sz = type_bytes(dtype);
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * sz) % 16 == 0 && (cols * sz) % 16 == 0 &&
         ld <= (int64_t(1) << 20);
}

// Hands out a workspace in 256-byte pieces; with no base it only adds up.
struct Pieces {
  char* base;
  size_t used = 0;
  void* take(size_t bytes) {
    char* p = base ? base + used : nullptr;
    used += align256(bytes);
    return p;
  }
};

// n rows of `cols` elements as products read them: themselves or a copy.
inline Side side_of(Packs& p, int32_t dtype, const void* m, int64_t n, int64_t cols, int64_t ld, void* copy) {
  if (direct(dtype, m, cols, ld)) return Side{{m, nullptr}, ld, n};
  add_pack(p, dtype, n, cols, m, ld, copy, up8(cols), DropKey{});
  return Side{{copy, nullptr}, up8(cols), n};
}

}  // namespace
}  // namespace abcd
