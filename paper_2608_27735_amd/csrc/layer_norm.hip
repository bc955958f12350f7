// layer_norm.hip -- layer norm of rows, and its gradients.
//
// mu = mean(x), rstd = 1 / sqrt(mean((x - mu)^2) + eps), z = (x - mu) rstd,
// y = z weight + bias. Backward, with v = dy weight:
//   dx = add + rstd (v - mean(v) - z mean(v z)),
//   dweight = sum over rows of dy z, dbias = sum over rows of dy.
// Bytes bound both: every array is read or written once. A row stays in the
// registers of G lanes (a part of a wave, a wave, or a workgroup), R vectors of
// 16 bytes each, so that the variance is taken about the mean without a second
// read; statistics and sums are fp32. The backward keeps a lane's columns of both
// column sums in registers over all rows that its workgroup takes, and a second
// launch adds the workgroups' sums in a fixed order: no atomics, the same result
// on every run. Rows too long for the registers are read again from the caches
// (the wide kernels). Forward, 1M x 64 in bf16: 52 us, 5.1 TB/s. Backward, 1M x 64 in
// fp32: 187 us, 5.5 TB/s; 16,384 x 4,096 in bf16: 102 us, 5.3 TB/s, 5 of them the sums.
#include <algorithm>

#include "load_frag.h"

namespace abcd {
namespace {

// sum / d, rounded once or nearly so (a constant row has to give its own value:
// what its mean is off by, rstd multiplies by up to 1 / sqrt(eps)). An infinite sum
// leaves nothing to correct.
__device__ __forceinline__ float mean_of(float sum, float d, float inv_d) {
  const float m = sum * inv_d;
  return __builtin_isinf(m) ? m : fmaf(fmaf(-m, d, sum), inv_d, m);
}

// 1 / sqrt(v), also where v is subnormal, of which the instruction makes an infinity.
__device__ __forceinline__ float rsqrt_of(float v) {
  const bool small = v < 0x1p-126f;
  return __builtin_amdgcn_rsqf(small ? v * 0x1p24f : v) * (small ? 0x1p12f : 1.0f);
}

struct NormArgs {
  const void* x;
  const void* w;
  const void* b;
  void* y;
  float* mean;
  float* rstd;
  int64_t ldx, ldy, n;
  int d;
  int wf32;
  float eps, inv_d;
};

template <typename T, int G, int R, bool kWhole>
__global__ __launch_bounds__(kBlock) void layer_norm_kernel(NormArgs a) {
  constexpr int N = kPer16<T>, kRows = kBlock / G;
  __shared__ float red[2][4];
  const int t = threadIdx.x % G;
  Floats<N> w[R], b[R];  // this lane's columns of weight and bias
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int c = (j * G + t) * N;
    w[j] = 1.0f;
    b[j] = 0.0f;
    if (a.w && c < a.d) w[j] = load_param<T, N, kWhole>(a.w, c, a.d - c, a.wf32);
    if (a.b && c < a.d) b[j] = load_param<T, N, kWhole>(a.b, c, a.d - c, a.wf32);
  }
  const int64_t step = (int64_t)gridDim.x * kRows;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G; row < a.n; row += step) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    typename Frag<T>::type raw[R];
    Floats<N> v[R];
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      raw[j] = load_frag<T, kWhole>(x + c, a.d - c, room_of(a.n, row, a.ldx, a.d - c));
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      v[j] = __builtin_convertvector((first_of<T, kWhole>(raw[j], a.d - (j * G + t) * N)), Floats<N>);
#pragma unroll
      for (int i = 0; i < N; ++i) s += v[j][i];
    }
    const float mean = mean_of(row_sum<G>(s, red[0]), (float)a.d, a.inv_d);
    s = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float e = c + i < a.d ? v[j][i] - mean : 0.0f;
        v[j][i] = e;
        s += e * e;
      }
    }
    const float rstd = rsqrt_of(row_sum<G>(s, red[1]) * a.inv_d + a.eps);
    T* y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      if (c >= a.d) continue;
      store_vec<T, N, kWhole>(y + c, v[j] * rstd * w[j] + b[j], a.d - c);
    }
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

// Rows longer than kBlock threads hold: a workgroup per row, three passes over it.
template <typename T, bool kWhole>
__global__ __launch_bounds__(kBlock) void layer_norm_wide_kernel(NormArgs a) {
  constexpr int N = kPer16<T>;
  __shared__ float red[2][4];
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    float s = 0.0f;
    for (int c = threadIdx.x * N; c < a.d; c += kBlock * N) {
      const Floats<N> v = load_vec<T, N, kWhole>(x + c, a.d - c);
#pragma unroll
      for (int i = 0; i < N; ++i) s += v[i];
    }
    const float mean = mean_of(row_sum<kBlock>(s, red[0]), (float)a.d, a.inv_d);
    s = 0.0f;
    for (int c = threadIdx.x * N; c < a.d; c += kBlock * N) {
      const Floats<N> v = load_vec<T, N, kWhole>(x + c, a.d - c);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float e = c + i < a.d ? v[i] - mean : 0.0f;
        s += e * e;
      }
    }
    const float rstd = rsqrt_of(row_sum<kBlock>(s, red[1]) * a.inv_d + a.eps);
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    for (int c = threadIdx.x * N; c < a.d; c += kBlock * N) {
      Floats<N> v = (load_vec<T, N, kWhole>(x + c, a.d - c) - mean) * rstd;
      if (a.w) v *= load_param<T, N, kWhole>(a.w, c, a.d - c, a.wf32);
      if (a.b) v += load_param<T, N, kWhole>(a.b, c, a.d - c, a.wf32);
      store_vec<T, N, kWhole>(y + c, v, a.d - c);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
  }
}

struct NormBwdArgs {
  const void* dy;
  const void* x;
  const float* mean;
  const float* rstd;
  const void* w;
  const void* add;
  void* dx;
  float* part;  // [gridDim.x][2][d]: the workgroups' sums of dy z and of dy
  void *dw, *db;  // what they add up to; NULL: not wanted
  int64_t lddy, ldx, ldadd, lddx, n;
  int d;
  int wf32;
  float inv_d;
};

// A workgroup's (of `parts`) sums of N columns: a part, or, where there is but one, the
// result.
template <typename T, int N, bool kWhole>
__device__ __forceinline__ void put_sums(const NormBwdArgs& a, int which, int parts, int at, int c, Floats<N> v) {
  if (parts > 1) {
    store_vec<float, N, kWhole>(a.part + ((int64_t)at * 2 + which) * a.d + c, v, a.d - c);
    return;
  }
  void* const out = which ? a.db : a.dw;
  if (!out) return;
  if (a.wf32)
    store_vec<float, N, kWhole>(static_cast<float*>(out) + c, v, a.d - c);
  else
    store_vec<T, N, kWhole>(static_cast<T*>(out) + c, v, a.d - c);
}

template <typename T, int G, int R, bool kWhole>
__global__ __launch_bounds__(kBlock) void layer_norm_bwd_kernel(NormBwdArgs a) {
  constexpr int N = kPer16<T>, kRows = kBlock / G;
  constexpr int kWaves = kBlock / kWave;
  __shared__ float red[2][4];
  __shared__ float cols[G <= 64 ? kWaves : 1][G <= 64 ? G * R * N : 1];
  typedef typename Frag<T>::type Raw;
  const int t = threadIdx.x % G;
  Floats<N> w[R], dw[R], db[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int c = (j * G + t) * N;
    w[j] = 1.0f;
    if (a.w && c < a.d) w[j] = load_param<T, N, kWhole>(a.w, c, a.d - c, a.wf32);
    dw[j] = db[j] = 0.0f;
  }
  const int64_t step = (int64_t)gridDim.x * kRows;
  // A row's values as they are in memory. The next row's are on their way while one is
  // worked on, where rows are long: 16,384 x 4,096 in bf16 take 113 us instead of 141,
  // 65,536 x 1,024 117 instead of 150. Short rows have waves enough without, and
  // registers for more of them: 1M x 64 in fp32 183 us instead of 192.
  constexpr bool kAhead = G * R > 64;
  Raw nx[R], ndy[R], nadd[R];
  float nmean, nrstd;
  auto fetch = [&](int64_t row) {
    const bool in = row < a.n;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N, left = in ? a.d - c : 0;
      nx[j] = load_frag<T, kWhole>(static_cast<const T*>(a.x) + row * a.ldx + c, left, room_of(a.n, row, a.ldx, left));
      ndy[j] = load_frag<T, kWhole>(static_cast<const T*>(a.dy) + row * a.lddy + c, left, room_of(a.n, row, a.lddy, left));
      nadd[j] = load_frag<T, kWhole>(static_cast<const T*>(a.add) + row * a.ldadd + c, a.add ? left : 0,
                                     room_of(a.n, row, a.ldadd, left));
    }
    nmean = in ? a.mean[row] : 0.0f;
    nrstd = in ? a.rstd[row] : 0.0f;
  };
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  if (kAhead) fetch(row);
  for (; row < a.n; row += step) {
    if (!kAhead) fetch(row);
    const float mean = nmean, rstd = nrstd;
    Floats<N> z[R], v[R];
    Raw add[R];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int left = a.d - (j * G + t) * N;
      z[j] = __builtin_convertvector((first_of<T, kWhole>(nx[j], left)), Floats<N>);
      v[j] = __builtin_convertvector((first_of<T, kWhole>(ndy[j], left)), Floats<N>);
      add[j] = nadd[j];
    }
    if (kAhead) fetch(row + step);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
#pragma unroll
      for (int i = 0; i < N; ++i) z[j][i] = c + i < a.d ? (z[j][i] - mean) * rstd : 0.0f;
      dw[j] += v[j] * z[j];
      db[j] += v[j];
      v[j] *= w[j];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s1 += v[j][i];
        s2 += v[j][i] * z[j][i];
      }
    }
    if (a.dx) {
      const float c1 = row_sum<G>(s1, red[0]) * a.inv_d, c2 = row_sum<G>(s2, red[1]) * a.inv_d;
      T* dx = static_cast<T*>(a.dx) + row * a.lddx;
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int c = (j * G + t) * N;
        if (c >= a.d) continue;
        Floats<N> r = rstd * (v[j] - c1 - z[j] * c2);
        if (a.add) r += __builtin_convertvector(add[j], Floats<N>);
        store_vec<T, N, kWhole>(dx + c, r, a.d - c);
      }
    }
  }
  if (!a.dw && !a.db) return;
  if (G > 64) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      if (c >= a.d) continue;
      put_sums<T, N, kWhole>(a, 0, gridDim.x, blockIdx.x, c, dw[j]);
      put_sums<T, N, kWhole>(a, 1, gridDim.x, blockIdx.x, c, db[j]);
    }
    return;
  }
  // the wave's groups added across the lanes, then the waves' sums through LDS
#pragma unroll
  for (int which = 0; which < 2; ++which) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      Floats<N> v = which ? db[j] : dw[j];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float e = v[i];
        for (int off = G; off < 64; off *= 2) e += __shfl_xor(e, off, 64);
        if ((threadIdx.x & 63) < G) cols[threadIdx.x >> 6][(j * G + t) * N + i] = e;
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += kBlock) {
      float e = 0.0f;
      for (int w = 0; w < kWaves; ++w) e += cols[w][c];
      put_sums<T, 1, true>(a, which, gridDim.x, blockIdx.x, c, Floats<1>(e));
    }
    __syncthreads();
  }
}

// Long rows: dx by a workgroup per row that reads it twice,
template <typename T, bool kWhole>
__global__ __launch_bounds__(kBlock) void layer_norm_bwd_wide_kernel(NormBwdArgs a) {
  constexpr int N = kPer16<T>;
  __shared__ float red[2][4];
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x * N; c < a.d; c += kBlock * N) {
      const Floats<N> z = (load_vec<T, N, kWhole>(x + c, a.d - c) - mean) * rstd;
      Floats<N> v = load_vec<T, N, kWhole>(dy + c, a.d - c);
      if (a.w) v *= load_param<T, N, kWhole>(a.w, c, a.d - c, a.wf32);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s1 += v[i];
        s2 += c + i < a.d ? v[i] * z[i] : 0.0f;
      }
    }
    const float c1 = row_sum<kBlock>(s1, red[0]) * a.inv_d, c2 = row_sum<kBlock>(s2, red[1]) * a.inv_d;
    for (int c = threadIdx.x * N; c < a.d; c += kBlock * N) {
      const Floats<N> z = (load_vec<T, N, kWhole>(x + c, a.d - c) - mean) * rstd;
      Floats<N> v = load_vec<T, N, kWhole>(dy + c, a.d - c);
      if (a.w) v *= load_param<T, N, kWhole>(a.w, c, a.d - c, a.wf32);
      Floats<N> r = rstd * (v - c1 - z * c2);
      if (a.add)
        r += load_vec<T, N, kWhole>(static_cast<const T*>(a.add) + row * a.ldadd + c, a.d - c);
      store_vec<T, N, kWhole>(static_cast<T*>(a.dx) + row * a.lddx + c, r, a.d - c);
    }
  }
}

// and the column sums by threads that own a vector of columns each: workgroup
// (x, y) takes columns [x kBlock N, ..) of the rows y, y + gridDim.y, ...
template <typename T, bool kWhole>
__global__ __launch_bounds__(kBlock) void layer_norm_cols_kernel(NormBwdArgs a) {
  constexpr int N = kPer16<T>;
  const int64_t c = ((int64_t)blockIdx.x * kBlock + threadIdx.x) * N;
  if (c >= a.d) return;
  const int left = a.d - (int)c;
  Floats<N> dw = 0.0f, db = 0.0f;
  for (int64_t row = blockIdx.y; row < a.n; row += gridDim.y) {
    const Floats<N> z =
        (load_vec<T, N, kWhole>(static_cast<const T*>(a.x) + row * a.ldx + c, left) - a.mean[row]) * a.rstd[row];
    const Floats<N> v = load_vec<T, N, kWhole>(static_cast<const T*>(a.dy) + row * a.lddy + c, left);
    dw += v * z;
    db += v;
  }
  put_sums<T, N, kWhole>(a, 0, gridDim.y, blockIdx.y, (int)c, dw);
  put_sums<T, N, kWhole>(a, 1, gridDim.y, blockIdx.y, (int)c, db);
}

// Rows of G lanes by R vectors that a kernel is compiled for; f(G, R) with the
// smallest that holds nvec, and false if none does.
template <int G, int R>
struct RowShape {
  static constexpr int g = G, r = R;
};
template <typename F>
bool with_shape(int nvec, bool few, F f) {
  if (nvec <= 8) return f(RowShape<8, 1>{}), true;
  if (nvec <= 16) return f(RowShape<16, 1>{}), true;
  if (nvec <= 32) return f(RowShape<32, 1>{}), true;
  if (nvec <= 64) return f(RowShape<64, 1>{}), true;
  if (nvec <= 128 && !few) return f(RowShape<64, 2>{}), true;
  if (nvec <= 256) return f(RowShape<kBlock, 1>{}), true;
  if (nvec <= 512) return f(RowShape<kBlock, 2>{}), true;
  if (nvec <= 1024) return f(RowShape<kBlock, 4>{}), true;
  return false;
}

// Workgroups of the backward, each with its own column sums: these are 8 bytes a
// column written and read, so there are no more of them than what a workgroup reads
// of its rows outweighs by far, but one for every CU. What one workgroup does in two
// turns it does alone, and saves the second launch (16 x 224 in float16: 18.4 us with the
// call's host time, with two workgroups and their sum 21.4).
int64_t bwd_blocks(int64_t n, int nvec, int64_t item) {
  const int64_t rows = nvec <= 8 ? 32 : nvec <= 16 ? 16 : nvec <= 32 ? 8 : nvec <= 128 ? 4 : 1;
  const int64_t most = std::max<int64_t>(256, std::min<int64_t>(n * item / 24, nvec <= 128 ? 1024 : 512));
  return n <= 2 * rows ? 1 : std::min<int64_t>((n + rows - 1) / rows, most);
}

}  // namespace

size_t layer_norm_bwd_workspace_bytes(int32_t dtype, int64_t n, int64_t d) {
  const int per = 16 / (int)type_bytes(dtype);
  return align256((size_t)bwd_blocks(n, (int)((d + per - 1) / per), type_bytes(dtype)) * 2 * d * sizeof(float));
}

int32_t launch_layer_norm(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx, int32_t wdtype,
                          const void* weight, const void* bias, float eps, void* y, int64_t ldy, float* mean,
                          float* rstd, hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  const NormArgs a{x,   weight, bias, y, mean, rstd, ldx, ldy, n, (int)d, wdtype == ABCD_F32 && dtype != ABCD_F32,
                   eps, 1.0f / (float)d};
  return with_type(dtype, [&](auto zero) -> int32_t {
    typedef decltype(zero) T;
    const int nvec = (int)((d + kPer16<T> - 1) / kPer16<T>);
    const bool whole = d % kPer16<T> == 0;
    const bool held = with_shape(nvec, n <= 1024, [&](auto shape) {
      constexpr int G = decltype(shape)::g, R = decltype(shape)::r;
      const int64_t rows = kBlock / G;
      const int64_t blocks = std::min<int64_t>((n + rows - 1) / rows, G > 64 ? 4096 : 2048);
      if (whole)
        ABCD_LAUNCH("layer_norm", (layer_norm_kernel<T, G, R, true>), blocks, kBlock, 0, stream, a);
      else
        ABCD_LAUNCH("layer_norm", (layer_norm_kernel<T, G, R, false>), blocks, kBlock, 0, stream, a);
    });
    if (!held) {
      const int64_t blocks = std::min<int64_t>(n, 2048);
      if (whole)
        ABCD_LAUNCH("layer_norm", (layer_norm_wide_kernel<T, true>), blocks, kBlock, 0, stream, a);
      else
        ABCD_LAUNCH("layer_norm", (layer_norm_wide_kernel<T, false>), blocks, kBlock, 0, stream, a);
    }
    ABCD_HIP(hipGetLastError());
    return ABCD_OK;
  });
}

int32_t launch_layer_norm_bwd(int32_t dtype, int64_t n, int64_t d, const void* dy, int64_t lddy, const void* x,
                              int64_t ldx, const float* mean, const float* rstd, int32_t wdtype,
                              const void* weight, const void* add, int64_t ldadd, void* dx, int64_t lddx,
                              void* dweight, void* dbias, void* workspace, hipStream_t stream) {
  const bool wf32 = wdtype == ABCD_F32;
  float* part = static_cast<float*>(workspace);
  const NormBwdArgs a{dy,  x,     mean, rstd, weight, add,  dx, part, dweight, dbias, lddy,
                      ldx, ldadd, lddx, n, (int)d, wf32 && dtype != ABCD_F32, 1.0f / (float)d};
  int64_t blocks = 0;
  if (n > 0)
    TRY_STATUS(with_type(dtype, [&](auto zero) -> int32_t {
      typedef decltype(zero) T;
      const int nvec = (int)((d + kPer16<T> - 1) / kPer16<T>);
      const bool whole = d % kPer16<T> == 0;
      blocks = bwd_blocks(n, nvec, sizeof(T));
      const bool held = with_shape(nvec, false, [&](auto shape) {
        constexpr int G = decltype(shape)::g, R = decltype(shape)::r;
        if (whole)
          ABCD_LAUNCH("layer_norm_bwd", (layer_norm_bwd_kernel<T, G, R, true>), blocks, kBlock, 0, stream, a);
        else
          ABCD_LAUNCH("layer_norm_bwd", (layer_norm_bwd_kernel<T, G, R, false>), blocks, kBlock, 0, stream, a);
      });
      if (!held) {
        // the column sums first: dx may be dy
        if (dweight || dbias) {
          const dim3 grid((nvec + kBlock - 1) / kBlock, blocks);
          if (whole)
            ABCD_LAUNCH("layer_norm_cols", (layer_norm_cols_kernel<T, true>), grid, kBlock, 0, stream, a);
          else
            ABCD_LAUNCH("layer_norm_cols", (layer_norm_cols_kernel<T, false>), grid, kBlock, 0, stream, a);
        }
        if (dx) {
          const int64_t rows = std::min<int64_t>(n, 2048);
          if (whole)
            ABCD_LAUNCH("layer_norm_bwd", (layer_norm_bwd_wide_kernel<T, true>), rows, kBlock, 0, stream, a);
          else
            ABCD_LAUNCH("layer_norm_bwd", (layer_norm_bwd_wide_kernel<T, false>), rows, kBlock, 0, stream, a);
        }
      }
      ABCD_HIP(hipGetLastError());
      return ABCD_OK;
    }));
  if ((dweight || dbias) && blocks != 1) {
    const int32_t to = wf32 ? ABCD_F32 : dtype;
    SumOuts outs{};
    outs.add(dweight, d);
    outs.add(dbias, d);
    TRY_STATUS(launch_sum_parts(part, blocks, outs, to, stream));
  }
  return ABCD_OK;
}

}  // namespace abcd
