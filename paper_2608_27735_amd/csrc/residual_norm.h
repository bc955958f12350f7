// residual_norm.h -- the joint between two blocks, forward and backward, for one
// element type (residual_norm_f32.hip, _f16.hip and _bf16.hip each compile it for theirs).
//
//   t = post(f), y = x + scale gate t, z = pre(y)
// with post and pre each a layer norm, an RMS norm or nothing. Backward, with v^ the
// normalised rows of v and J(v; u) = rstd (u - mean(u) - v^ mean(u v^)), without mean(u) of
// an RMS norm, the gradient through a norm:
//   g = dy + J(y; dz wpre) is y's and x's gradient; dgate = g scale t (its sum over the row
//   where the gate is one number a row); df = J(f; g gate scale wpost);
//   dwpre = sum dz y^, dbpre = sum dz over the rows, and with S1 = sum g gate f^ and
//   S0 = sum g gate: dwpost = scale S1, dbpost = scale S0, dscale = wpost S1 + bpost S0.
// Bytes bound both: forward f and x are read and y and z written once, backward dz, dy, y
// and f read and dx and df written once; layer norms and products one after the other
// would move twice as much. A row stays in the registers of G lanes (a part of a wave, a
// wave, or a workgroup), R vectors of 16 bytes each; statistics and sums are fp32, and z
// is the norm of y before y is rounded. The four column sums stay in registers over all
// rows that a workgroup takes, and a second launch adds the workgroups' in a fixed order.
// Rows too long for a workgroup's registers are read again (the wide kernels).
#pragma once

#include <algorithm>

#include "load_frag.h"
#include "residual_norm_args.h"

namespace abcd {
namespace {

template <int G>
constexpr int kJointThreads = G > kBlock ? G : kBlock;

// Sums of K values over the G lanes of a row, returned to each. `turn` alternates
// between the two halves of red, so that a wave that writes one again has met the
// other's barrier, behind all reads.
template <int G, int K>
__device__ __forceinline__ void joint_sums(float (&v)[K], float (*red)[K][G / 64 + 1], int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = lanes_sum<(G <= 64 ? G : 64)>(v[k]);
  if (G <= 64) return;
  float(&r)[K][G / 64 + 1] = red[turn & 1];
  ++turn;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) r[k][threadIdx.x >> 6] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) s += r[k][w];
    v[k] = s;
  }
}

// sum / d, rounded once or nearly so (a constant row has to give its own value: what its
// mean is off by, rstd multiplies by up to 1 / sqrt(eps)). An infinite sum leaves
// nothing to correct.
__device__ __forceinline__ float joint_mean(float sum, float d, float inv_d) {
  const float m = sum * inv_d;
  return __builtin_isinf(m) ? m : fmaf(fmaf(-m, d, sum), inv_d, m);
}

// 1 / sqrt(v), also where v is subnormal, of which the instruction makes an infinity.
__device__ __forceinline__ float joint_rsqrt(float v) {
  const bool small = v < 0x1p-126f;
  return __builtin_amdgcn_rsqf(small ? v * 0x1p24f : v) * (small ? 0x1p12f : 1.0f);
}

// A parameter's columns of a lane; `none` without one. Past the row's end 0.
template <typename T, int N, bool kWhole>
__device__ __forceinline__ Floats<N> joint_param(const JointArgs& a, const void* p, int c, float none) {
  if (!p) return none;
  return c < a.d ? load_param<T, N, kWhole>(p, c, a.d - c, a.wf32) : Floats<N>(0.0f);
}

template <typename T, int N, bool kWhole>
__device__ __forceinline__ Floats<N> joint_load(const void* p, int64_t row, int64_t ld, int c, const JointArgs& a) {
  const int left = row < a.n ? a.d - c : 0;
  return __builtin_convertvector(
      (load_first<T, kWhole>(static_cast<const T*>(p) + row * ld + c, left, room_of(a.n, row, ld, left))), Floats<N>);
}

// Mean (0 of an RMS norm) and 1 / sd of the row whose columns the lanes hold.
template <int G, int R, int N>
__device__ __forceinline__ void joint_stats(const JointArgs& a, const Floats<N> (&v)[R], int t, int kind,
                                            float (*red)[1][G / 64 + 1], int& turn, float& mean, float& rstd) {
  float s[1];
  mean = 0.0f;
  if (kind == ABCD_NORM_LAYER) {
    s[0] = 0.0f;
#pragma unroll
    for (int j = 0; j < R; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) s[0] += (j * G + t) * N + i < a.d ? v[j][i] : 0.0f;
    joint_sums<G, 1>(s, red, turn);
    mean = joint_mean(s[0], (float)a.d, a.inv_d);
  }
  s[0] = 0.0f;
#pragma unroll
  for (int j = 0; j < R; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = (j * G + t) * N + i < a.d ? v[j][i] - mean : 0.0f;
      s[0] += e * e;
    }
  joint_sums<G, 1>(s, red, turn);
  rstd = joint_rsqrt(s[0] * a.inv_d + a.eps);
}

template <typename T, int G, int R, bool kWhole>
__global__ __launch_bounds__(kJointThreads<G>) void residual_norm_kernel(JointArgs a) {
  constexpr int N = kPer16<T>, kRows = kJointThreads<G> / G;
  __shared__ float red[2][1][G / 64 + 1];
  int turn = 0;
  const int t = threadIdx.x % G;
  Floats<N> wp[R], bp[R], wn[R], bn[R], sc[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int c = (j * G + t) * N;
    wp[j] = joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f);
    bp[j] = joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f);
    wn[j] = joint_param<T, N, kWhole>(a, a.pre_w, c, 1.0f);
    bn[j] = joint_param<T, N, kWhole>(a, a.pre_b, c, 0.0f);
    sc[j] = joint_param<T, N, kWhole>(a, a.scale, c, 1.0f);
  }
  const int64_t step = (int64_t)gridDim.x * kRows;
  // Every lane of a row takes part in its sums: rows past the end are worked on as zeros.
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += step) {
    const int64_t row = first + threadIdx.x / G;
    const bool in = row < a.n;
    Floats<N> v[R], x[R], g[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      v[j] = joint_load<T, N, kWhole>(a.f, row, a.ldf, c, a);
      x[j] = joint_load<T, N, kWhole>(a.x, row, a.ldx, c, a);
      g[j] = 1.0f;
      if (a.gate_mode == 2) g[j] = joint_load<T, N, kWhole>(a.gate, row, a.ldg, c, a);
    }
    if (a.gate_mode == 1) {
      const float one = in ? (float)static_cast<const T*>(a.gate)[row * a.ldg] : 0.0f;
#pragma unroll
      for (int j = 0; j < R; ++j) g[j] = one;
    }
    float mean, rstd;
    if (a.post != ABCD_NORM_NONE) {
      joint_stats<G, R, N>(a, v, t, a.post, red, turn, mean, rstd);
#pragma unroll
      for (int j = 0; j < R; ++j) v[j] = (v[j] - mean) * rstd * wp[j] + bp[j];
      if (t == 0 && in) {
        if (a.post_mean) a.post_mean[row] = mean;
        if (a.post_rstd) a.post_rstd[row] = rstd;
      }
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      v[j] = x[j] + sc[j] * (g[j] * v[j]);
      if (in && c < a.d) store_vec<T, N, kWhole>(static_cast<T*>(a.y) + row * a.ldy + c, v[j], a.d - c);
    }
    if (a.pre != ABCD_NORM_NONE) {
      joint_stats<G, R, N>(a, v, t, a.pre, red, turn, mean, rstd);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int c = (j * G + t) * N;
        if (in && c < a.d)
          store_vec<T, N, kWhole>(static_cast<T*>(a.z) + row * a.ldz + c, (v[j] - mean) * rstd * wn[j] + bn[j], a.d - c);
      }
      if (t == 0 && in) {
        if (a.pre_mean) a.pre_mean[row] = mean;
        if (a.pre_rstd) a.pre_rstd[row] = rstd;
      }
    }
  }
}

constexpr int kWide = 1024;  // threads of a row too long for registers

// A workgroup per row, in passes over it: f's mean, f's variance, y and its mean, y's variance, z.
template <typename T, bool kWhole>
__global__ __launch_bounds__(kWide) void residual_norm_wide_kernel(JointArgs a) {
  constexpr int N = kPer16<T>;
  __shared__ float red[2][1][kWide / 64 + 1];
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    // the sum over the row of f(its columns c..)
    auto total = [&](auto f) {
      float s[1] = {0.0f};
      for (int c = threadIdx.x * N; c < a.d; c += kWide * N) {
        const Floats<N> v = f(c);
#pragma unroll
        for (int i = 0; i < N; ++i) s[0] += c + i < a.d ? v[i] : 0.0f;
      }
      joint_sums<kWide, 1>(s, red, turn);
      return s[0];
    };
    auto stats = [&](int kind, auto f, float& mean, float& rstd) {
      mean = kind == ABCD_NORM_LAYER ? joint_mean(total(f), (float)a.d, a.inv_d) : 0.0f;
      rstd = joint_rsqrt(total([&](int c) {
                           const Floats<N> e = f(c) - mean;
                           return e * e;
                         }) * a.inv_d + a.eps);
    };
    float pm = 0.0f, pr = 1.0f, mean, rstd;
    auto f = [&](int c) { return joint_load<T, N, kWhole>(a.f, row, a.ldf, c, a); };
    if (a.post != ABCD_NORM_NONE) {
      stats(a.post, f, pm, pr);
      if (threadIdx.x == 0) {
        if (a.post_mean) a.post_mean[row] = pm;
        if (a.post_rstd) a.post_rstd[row] = pr;
      }
    }
    auto y = [&](int c) {
      Floats<N> v = f(c);
      if (a.post != ABCD_NORM_NONE)
        v = (v - pm) * pr * joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f) + joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f);
      if (a.gate_mode == 1) v *= (float)static_cast<const T*>(a.gate)[row * a.ldg];
      if (a.gate_mode == 2) v *= joint_load<T, N, kWhole>(a.gate, row, a.ldg, c, a);
      return joint_load<T, N, kWhole>(a.x, row, a.ldx, c, a) + joint_param<T, N, kWhole>(a, a.scale, c, 1.0f) * v;
    };
    for (int c = threadIdx.x * N; c < a.d; c += kWide * N)
      store_vec<T, N, kWhole>(static_cast<T*>(a.y) + row * a.ldy + c, y(c), a.d - c);
    if (a.pre == ABCD_NORM_NONE) continue;
    stats(a.pre, y, mean, rstd);
    if (threadIdx.x == 0) {
      if (a.pre_mean) a.pre_mean[row] = mean;
      if (a.pre_rstd) a.pre_rstd[row] = rstd;
    }
    for (int c = threadIdx.x * N; c < a.d; c += kWide * N)
      store_vec<T, N, kWhole>(static_cast<T*>(a.z) + row * a.ldz + c,
                              (y(c) - mean) * rstd * joint_param<T, N, kWhole>(a, a.pre_w, c, 1.0f) +
                                  joint_param<T, N, kWhole>(a, a.pre_b, c, 0.0f),
                              a.d - c);
  }
}

// ---------------------------------------------------------------- backward

// The parameters' gradients of columns c.. from the four column sums.
template <typename T, int N, bool kWhole>
__device__ __forceinline__ void put_params(const JointArgs& a, int c, Floats<N> s1, Floats<N> s0, Floats<N> dw, Floats<N> db) {
  if (c >= a.d) return;
  auto put = [&](void* p, Floats<N> v) {
    if (!p) return;
    if (a.wf32)
      store_vec<float, N, kWhole>(static_cast<float*>(p) + c, v, a.d - c);
    else
      store_vec<T, N, kWhole>(static_cast<T*>(p) + c, v, a.d - c);
  };
  const Floats<N> sc = joint_param<T, N, kWhole>(a, a.scale, c, 1.0f);
  put(a.dpost_w, sc * s1);
  put(a.dpost_b, sc * s0);
  put(a.dscale, joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f) * s1 + joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f) * s0);
  put(a.dpre_w, dw);
  put(a.dpre_b, db);
}

template <typename T, int G, int R, bool kWhole>
__global__ __launch_bounds__(kJointThreads<G>) void residual_norm_bwd_kernel(JointArgs a) {
  constexpr int N = kPer16<T>, kThreads = kJointThreads<G>, kRows = kThreads / G, kWaves = kThreads / 64;
  __shared__ float red2[2][2][G / 64 + 1], red3[2][3][G / 64 + 1];
  __shared__ float cols[G <= 64 ? kWaves : 1][G <= 64 ? G * R * N : 1];
  int turn2 = 0, turn3 = 0;
  const int t = threadIdx.x % G;
  const bool has_pre = a.pre != ABCD_NORM_NONE, has_post = a.post != ABCD_NORM_NONE;
  Floats<N> wp[R], bp[R], wn[R], sc[R], s1[R], s0[R], dw[R], db[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int c = (j * G + t) * N;
    wp[j] = joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f);
    bp[j] = joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f);
    wn[j] = joint_param<T, N, kWhole>(a, a.pre_w, c, 1.0f);
    sc[j] = joint_param<T, N, kWhole>(a, a.scale, c, 1.0f);
    s1[j] = s0[j] = dw[j] = db[j] = 0.0f;
  }
  const int64_t step = (int64_t)gridDim.x * kRows;
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += step) {
    const int64_t row = first + threadIdx.x / G;
    const bool in = row < a.n;
    Floats<N> g[R], h[R], v[R], f[R], gate[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      g[j] = v[j] = h[j] = 0.0f;
      if (a.dy) g[j] = joint_load<T, N, kWhole>(a.dy, row, a.lddy, c, a);
      if (has_pre) {
        v[j] = joint_load<T, N, kWhole>(a.dz, row, a.lddz, c, a);
        h[j] = joint_load<T, N, kWhole>(a.y, row, a.ldy, c, a);
      }
      f[j] = joint_load<T, N, kWhole>(a.f, row, a.ldf, c, a);
      gate[j] = 1.0f;
      if (a.gate_mode == 2) gate[j] = joint_load<T, N, kWhole>(a.gate, row, a.ldg, c, a);
    }
    float one = 1.0f;
    if (a.gate_mode == 1) one = in ? (float)static_cast<const T*>(a.gate)[row * a.ldg] : 0.0f;
    if (has_pre) {
      const float mean = in && a.pre == ABCD_NORM_LAYER ? a.pre_mean[row] : 0.0f, rstd = in ? a.pre_rstd[row] : 0.0f;
      float s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int c = (j * G + t) * N;
#pragma unroll
        for (int i = 0; i < N; ++i) h[j][i] = c + i < a.d ? (h[j][i] - mean) * rstd : 0.0f;
        dw[j] += v[j] * h[j];
        db[j] += v[j];
        v[j] *= wn[j];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          s[0] += v[j][i];
          s[1] += v[j][i] * h[j][i];
        }
      }
      joint_sums<G, 2>(s, red2, turn2);
      const float c1 = a.pre == ABCD_NORM_LAYER ? s[0] * a.inv_d : 0.0f, c2 = s[1] * a.inv_d;
#pragma unroll
      for (int j = 0; j < R; ++j) g[j] += rstd * (v[j] - c1 - h[j] * c2);
    }
    const float pm = in && a.post == ABCD_NORM_LAYER ? a.post_mean[row] : 0.0f, pr = has_post && in ? a.post_rstd[row] : 1.0f;
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      if (a.dx && in && c < a.d) store_vec<T, N, kWhole>(static_cast<T*>(a.dx) + row * a.lddx + c, g[j], a.d - c);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const bool there = in && c + i < a.d;
        f[j][i] = there ? (f[j][i] - pm) * pr : 0.0f;
        g[j][i] = there ? g[j][i] : 0.0f;
      }
      if (a.gate_mode == 1) gate[j] = one;
      const Floats<N> by = g[j] * sc[j] * (f[j] * wp[j] + bp[j]);  // the gate's
      if (a.dgate && a.gate_mode == 2 && in && c < a.d)
        store_vec<T, N, kWhole>(static_cast<T*>(a.dgate) + row * a.lddg + c, by, a.d - c);
      g[j] *= gate[j];
      s1[j] += g[j] * f[j];
      s0[j] += g[j];
      g[j] *= sc[j] * wp[j];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[0] += g[j][i];
        s[1] += g[j][i] * f[j][i];
        s[2] += by[i];
      }
    }
    if (has_post || a.gate_mode == 1) joint_sums<G, 3>(s, red3, turn3);
    if (a.dgate && a.gate_mode == 1 && in && t == 0) static_cast<T*>(a.dgate)[row * a.lddg] = (T)s[2];
    if (a.df) {
      const float c1 = a.post == ABCD_NORM_LAYER ? s[0] * a.inv_d : 0.0f, c2 = has_post ? s[1] * a.inv_d : 0.0f;
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int c = (j * G + t) * N;
        if (in && c < a.d)
          store_vec<T, N, kWhole>(static_cast<T*>(a.df) + row * a.lddf + c, pr * (g[j] - c1 - f[j] * c2), a.d - c);
      }
    }
  }
  if (!a.part && gridDim.x > 1) return;  // no parameter's gradient is wanted
  if (G > 64) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int c = (j * G + t) * N;
      if (c >= a.d) continue;
      if (gridDim.x == 1) {
        put_params<T, N, kWhole>(a, c, s1[j], s0[j], dw[j], db[j]);
        continue;
      }
      float* const p = a.part + (int64_t)blockIdx.x * 4 * a.pitch + c;
      store_vec<float, N, true>(p, s1[j], N);
      store_vec<float, N, true>(p + a.pitch, s0[j], N);
      store_vec<float, N, true>(p + 2 * a.pitch, dw[j], N);
      store_vec<float, N, true>(p + 3 * a.pitch, db[j], N);
    }
    return;
  }
  // the wave's groups added across the lanes, then the waves' sums through LDS
  constexpr int kTurns = (G * R * N + kThreads - 1) / kThreads;
  float own[4][kTurns];
#pragma unroll
  for (int which = 0; which < 4; ++which) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const Floats<N> v = which == 0 ? s1[j] : which == 1 ? s0[j] : which == 2 ? dw[j] : db[j];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float e = v[i];
        for (int off = G; off < 64; off *= 2) e += __shfl_xor(e, off, 64);
        if ((threadIdx.x & 63) < G) cols[threadIdx.x >> 6][(j * G + t) * N + i] = e;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
      const int c = k * kThreads + threadIdx.x;
      own[which][k] = 0.0f;
      if (c < a.d && c < G * R * N)
        for (int w = 0; w < kWaves; ++w) own[which][k] += cols[w][c];
    }
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int c = k * kThreads + threadIdx.x;
    if (c >= a.d) continue;
    if (gridDim.x == 1)
      put_params<T, 1, true>(a, c, Floats<1>(own[0][k]), Floats<1>(own[1][k]), Floats<1>(own[2][k]), Floats<1>(own[3][k]));
    else
#pragma unroll
      for (int which = 0; which < 4; ++which) a.part[((int64_t)blockIdx.x * 4 + which) * a.pitch + c] = own[which][k];
  }
}

// Long rows: a workgroup per row in three passes, its column sums kept in its part.
template <typename T, bool kWhole>
__global__ __launch_bounds__(kWide) void residual_norm_bwd_wide_kernel(JointArgs a) {
  constexpr int N = kPer16<T>;
  __shared__ float red2[2][2][kWide / 64 + 1], red3[2][3][kWide / 64 + 1];
  int turn2 = 0, turn3 = 0;
  const bool has_pre = a.pre != ABCD_NORM_NONE, has_post = a.post != ABCD_NORM_NONE;
  for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
    const float mean = a.pre == ABCD_NORM_LAYER ? a.pre_mean[row] : 0.0f, rstd = has_pre ? a.pre_rstd[row] : 0.0f;
    const float pm = a.post == ABCD_NORM_LAYER ? a.post_mean[row] : 0.0f, pr = has_post ? a.post_rstd[row] : 1.0f;
    const float one = a.gate_mode == 1 ? (float)static_cast<const T*>(a.gate)[row * a.ldg] : 1.0f;
    auto hat = [&](Floats<N> v, float m, float r, int c) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = c + i < a.d ? (v[i] - m) * r : 0.0f;
      return v;
    };
    float s[2] = {0.0f, 0.0f};
    if (has_pre) {
      for (int c = threadIdx.x * N; c < a.d; c += kWide * N) {
        const Floats<N> h = hat(joint_load<T, N, kWhole>(a.y, row, a.ldy, c, a), mean, rstd, c);
        const Floats<N> v = joint_load<T, N, kWhole>(a.dz, row, a.lddz, c, a) * joint_param<T, N, kWhole>(a, a.pre_w, c, 1.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          s[0] += v[i];
          s[1] += v[i] * h[i];
        }
      }
      joint_sums<kWide, 2>(s, red2, turn2);
    }
    const float c1 = a.pre == ABCD_NORM_LAYER ? s[0] * a.inv_d : 0.0f, c2 = s[1] * a.inv_d;
    auto grad = [&](int c, Floats<N>& dz, Floats<N>& h) {
      Floats<N> g = 0.0f;
      dz = h = 0.0f;
      if (a.dy) g = joint_load<T, N, kWhole>(a.dy, row, a.lddy, c, a);
      if (has_pre) {
        h = hat(joint_load<T, N, kWhole>(a.y, row, a.ldy, c, a), mean, rstd, c);
        dz = joint_load<T, N, kWhole>(a.dz, row, a.lddz, c, a);
        g += rstd * (dz * joint_param<T, N, kWhole>(a, a.pre_w, c, 1.0f) - c1 - h * c2);
      }
      return hat(g, 0.0f, 1.0f, c);
    };
    auto gate_at = [&](int c) {
      return a.gate_mode == 2 ? joint_load<T, N, kWhole>(a.gate, row, a.ldg, c, a) : Floats<N>(one);
    };
    float s3[3] = {0.0f, 0.0f, 0.0f};
    for (int c = threadIdx.x * N; c < a.d; c += kWide * N) {
      Floats<N> dz, h;
      Floats<N> g = grad(c, dz, h);
      if (a.dx) store_vec<T, N, kWhole>(static_cast<T*>(a.dx) + row * a.lddx + c, g, a.d - c);
      const Floats<N> f = hat(joint_load<T, N, kWhole>(a.f, row, a.ldf, c, a), pm, pr, c);
      const Floats<N> wp = joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f), sc = joint_param<T, N, kWhole>(a, a.scale, c, 1.0f);
      const Floats<N> by = g * sc * (f * wp + joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f));
      if (a.dgate && a.gate_mode == 2) store_vec<T, N, kWhole>(static_cast<T*>(a.dgate) + row * a.lddg + c, by, a.d - c);
      g *= gate_at(c);
      if (a.part) {
        float* const p = a.part + (int64_t)blockIdx.x * 4 * a.pitch + c;
        const Floats<N> add[4] = {g * f, g, dz * h, dz};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          Floats<N> was = 0.0f;
          if (row != (int64_t)blockIdx.x) was = load_vec<float, N, true>(p + k * a.pitch, N);
          store_vec<float, N, true>(p + k * a.pitch, was + add[k], N);
        }
      }
      g *= sc * wp;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s3[0] += g[i];
        s3[1] += g[i] * f[i];
        s3[2] += by[i];
      }
    }
    joint_sums<kWide, 3>(s3, red3, turn3);
    if (a.dgate && a.gate_mode == 1 && threadIdx.x == 0) static_cast<T*>(a.dgate)[row * a.lddg] = (T)s3[2];
    if (!a.df) continue;
    const float c3 = a.post == ABCD_NORM_LAYER ? s3[0] * a.inv_d : 0.0f, c4 = has_post ? s3[1] * a.inv_d : 0.0f;
    for (int c = threadIdx.x * N; c < a.d; c += kWide * N) {
      Floats<N> dz, h;
      const Floats<N> g = grad(c, dz, h) * gate_at(c) * joint_param<T, N, kWhole>(a, a.scale, c, 1.0f) *
                          joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f);
      const Floats<N> f = hat(joint_load<T, N, kWhole>(a.f, row, a.ldf, c, a), pm, pr, c);
      store_vec<T, N, kWhole>(static_cast<T*>(a.df) + row * a.lddf + c, pr * (g - c3 - f * c4), a.d - c);
    }
  }
}

// The workgroups' column sums added up in order: 64 columns a workgroup, the parts dealt
// to its waves.
constexpr int kJointPartWaves = 16;
template <typename T>
__global__ __launch_bounds__(kJointPartWaves* kWave) void residual_norm_sums_kernel(JointArgs a, int64_t parts) {
  __shared__ float red[kJointPartWaves][4][kWave];
  const int w = threadIdx.x / kWave, l = threadIdx.x % kWave, c = (int)blockIdx.x * kWave + l;
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < a.d)
#pragma unroll 4
    for (int64_t p = w; p < parts; p += kJointPartWaves)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += a.part[(p * 4 + k) * a.pitch + c];
#pragma unroll
  for (int k = 0; k < 4; ++k) red[w][k][l] = s[k];
  __syncthreads();
  if (w != 0 || c >= a.d) return;
  for (int v = 1; v < kJointPartWaves; ++v)
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] += red[v][k][l];
  put_params<T, 1, true>(a, c, Floats<1>(s[0]), Floats<1>(s[1]), Floats<1>(s[2]), Floats<1>(s[3]));
}

// Rows of G lanes by R vectors that a kernel is compiled for; f(shape) with the
// smallest that holds nvec, and false if none does.
template <int G, int R>
struct JointShape {
  static constexpr int g = G, r = R;
};
template <typename F>
bool with_joint_shape(int nvec, F f) {
  if (nvec <= 8) return f(JointShape<8, 1>{}), true;
  if (nvec <= 16) return f(JointShape<16, 1>{}), true;
  if (nvec <= 32) return f(JointShape<32, 1>{}), true;
  if (nvec <= 64) return f(JointShape<64, 1>{}), true;
  if (nvec <= 128) return f(JointShape<64, 2>{}), true;
  if (nvec <= 256) return f(JointShape<256, 1>{}), true;
  if (nvec <= 512) return f(JointShape<512, 1>{}), true;
  if (nvec <= 1024) return f(JointShape<1024, 1>{}), true;
  return false;
}

template <typename T>
int32_t run_joint(const JointArgs& a, hipStream_t stream) {
  const int nvec = (int)((a.d + kPer16<T> - 1) / kPer16<T>);
  const bool whole = a.d % kPer16<T> == 0;
  const bool held = with_joint_shape(nvec, [&](auto shape) {
    constexpr int G = decltype(shape)::g, R = decltype(shape)::r, kThreads = kJointThreads<G>;
    const int64_t rows = kThreads / G, blocks = std::min<int64_t>((a.n + rows - 1) / rows, G > 64 ? 4096 : 2048);
    if (whole)
      ABCD_LAUNCH("residual_norm", (residual_norm_kernel<T, G, R, true>), blocks, kThreads, 0, stream, a);
    else
      ABCD_LAUNCH("residual_norm", (residual_norm_kernel<T, G, R, false>), blocks, kThreads, 0, stream, a);
  });
  if (!held) {
    const int64_t blocks = std::min<int64_t>(a.n, 1024);
    if (whole)
      ABCD_LAUNCH("residual_norm", (residual_norm_wide_kernel<T, true>), blocks, kWide, 0, stream, a);
    else
      ABCD_LAUNCH("residual_norm", (residual_norm_wide_kernel<T, false>), blocks, kWide, 0, stream, a);
  }
  ABCD_HIP(hipGetLastError());
  return ABCD_OK;
}

template <typename T>
int32_t run_joint_bwd(const JointArgs& a, int64_t blocks, hipStream_t stream) {
  const int nvec = (int)((a.d + kPer16<T> - 1) / kPer16<T>);
  const bool whole = a.d % kPer16<T> == 0;
  bool summed = blocks == 1;
  if (a.n > 0) {
    const bool held = with_joint_shape(nvec, [&](auto shape) {
      constexpr int G = decltype(shape)::g, R = decltype(shape)::r, kThreads = kJointThreads<G>;
      if (whole)
        ABCD_LAUNCH("residual_norm_bwd", (residual_norm_bwd_kernel<T, G, R, true>), blocks, kThreads, 0, stream, a);
      else
        ABCD_LAUNCH("residual_norm_bwd", (residual_norm_bwd_kernel<T, G, R, false>), blocks, kThreads, 0, stream, a);
    });
    if (!held) {
      summed = false;
      if (whole)
        ABCD_LAUNCH("residual_norm_bwd", (residual_norm_bwd_wide_kernel<T, true>), blocks, kWide, 0, stream, a);
      else
        ABCD_LAUNCH("residual_norm_bwd", (residual_norm_bwd_wide_kernel<T, false>), blocks, kWide, 0, stream, a);
    }
    ABCD_HIP(hipGetLastError());
  }
  if (a.part && (!summed || a.n == 0)) {
    ABCD_LAUNCH("residual_norm_sums", (residual_norm_sums_kernel<T>), (a.d + kWave - 1) / kWave, kJointPartWaves * kWave, 0,
                stream, a, a.n == 0 ? 0 : blocks);
    ABCD_HIP(hipGetLastError());
  }
  return ABCD_OK;
}

}  // namespace

#define ABCD_JOINT_KERNELS(NAME, TYPE)                                                                   \
  int32_t residual_norm_##NAME(const JointArgs& a, hipStream_t s) { return run_joint<TYPE>(a, s); }      \
  int32_t residual_norm_bwd_##NAME(const JointArgs& a, int64_t blocks, hipStream_t s) {                  \
    return run_joint_bwd<TYPE>(a, blocks, s);                                                            \
  }

}  // namespace abcd
