// reduce.hip -- sums of partial results in a fixed order.
#include <algorithm>

#include "rows.h"

namespace abcd {
namespace {

constexpr int kPartWaves = 16;

// Column c of the parts belongs to the output whose range holds it; out[i] = sum
// over p of part[p][c]: 64 columns per workgroup, the parts dealt to its 16 waves with
// eight loads in flight each, whose sums LDS joins. 256 parts of 24,896 columns (25 MB):
// 6 us; a launch of little work 4.5.
template <typename T>
__global__ __launch_bounds__(kPartWaves* kWave) void sum_parts_kernel(const float* part, int64_t parts,
                                                                     SumOuts outs) {
  __shared__ float red[kPartWaves][kWave];
  const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
  const int64_t c = (int64_t)blockIdx.x * kWave + l, cols = outs.begin[outs.count];
  float s = 0.0f;
  if (c < cols) {
    int64_t p = w;
    for (; p + 7 * kPartWaves < parts; p += 8 * kPartWaves) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = part[(p + i * kPartWaves) * cols + c];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    for (; p < parts; p += kPartWaves) s += part[p * cols + c];
  }
  red[w][l] = s;
  __syncthreads();
  if (w != 0 || c >= cols) return;
  for (int i = 1; i < kPartWaves; ++i) s += red[i][l];
  int k = 0;
  while (c >= outs.begin[k + 1]) ++k;
  if (outs.out[k]) static_cast<T*>(outs.out[k])[c - outs.begin[k]] = (T)s;
}

}  // namespace

int32_t launch_sum_parts(const float* part, int64_t parts, const SumOuts& outs, int32_t dtype, hipStream_t stream) {
  return with_type(dtype, [&](auto zero) -> int32_t {
    typedef decltype(zero) T;
    const int64_t cols = outs.begin[outs.count];
    ABCD_LAUNCH("sum_parts", (sum_parts_kernel<T>), (cols + kWave - 1) / kWave, kPartWaves * kWave, 0, stream, part,
                parts, outs);
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

}  // namespace abcd
