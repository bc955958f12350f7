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
//
// 1M x 64 in bf16 with a gate a row, forward 110 us (530 MB, 4.8 TB/s), backward 158; 8,192 x 4,096
// with a gate an element, backward 115 us and 8 for the column sums (537 MB, 4.7 TB/s).
#pragma once

#include <algorithm>

#include "load_frag.h"
#include "residual_norm_args.h"

namespace abcd {
namespace {

// Threads of a workgroup: forward, and backward, where fewer workgroups of more waves leave
// fewer column sums to be added up.
template <int G>
constexpr int kJointThreads = G > kBlock ? G : kBlock;
template <int G>
constexpr int kJointBwdThreads = G > 512 ? G : 512;

// Sums of K values over the G lanes of a row, returned to each. `turn` alternates
// between the two halves of red, so that a wave that writes one again has met the
// other's barrier, behind all reads.
constexpr int kJointWaves = 16;  // of a workgroup at most
template <int G, int K>
__device__ __forceinline__ void joint_sums(float (&v)[K], float (*red)[K][kJointWaves], int& turn) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = lanes_sum<(G <= 64 ? G : 64)>(v[k]);
  if (G <= 64) return;
  constexpr int kOf = G > 64 ? G / 64 : 1;  // waves of a row
  float(&r)[K][kJointWaves] = red[turn & 1];
  ++turn;
  const int wave = threadIdx.x >> 6, first = wave / kOf * kOf;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) r[k][wave] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kOf; ++w) s += r[k][first + w];
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

// Mean (0 of an RMS norm) and 1 / sd of the row whose columns c.. a lane holds.
template <int G, int N>
__device__ __forceinline__ void joint_stats(const JointArgs& a, Floats<N> v, int c, int kind, float (*red)[1][kJointWaves],
                                            int& turn, float& mean, float& rstd) {
  float s[1];
  mean = 0.0f;
  if (kind == ABCD_NORM_LAYER) {
    s[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) s[0] += c + i < a.d ? v[i] : 0.0f;
    joint_sums<G, 1>(s, red, turn);
    mean = joint_mean(s[0], (float)a.d, a.inv_d);
  }
  s[0] = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float e = c + i < a.d ? v[i] - mean : 0.0f;
    s[0] += e * e;
  }
  joint_sums<G, 1>(s, red, turn);
  rstd = joint_rsqrt(s[0] * a.inv_d + a.eps);
}

template <typename T, int G, bool kWhole>
__global__ __launch_bounds__(kJointThreads<G>) void residual_norm_kernel(JointArgs a) {
  constexpr int N = kPer16<T>, kRows = kJointThreads<G> / G;
  __shared__ float red[2][1][kJointWaves];
  int turn = 0;
  const int t = threadIdx.x % G, c = t * N;
  const bool inside = c < a.d;
  const Floats<N> wp = joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f), bp = joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f);
  const Floats<N> wn = joint_param<T, N, kWhole>(a, a.pre_w, c, 1.0f), bn = joint_param<T, N, kWhole>(a, a.pre_b, c, 0.0f);
  const Floats<N> sc = joint_param<T, N, kWhole>(a, a.scale, c, 1.0f);
  const int64_t step = (int64_t)gridDim.x * kRows;
  const int sub = G >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G;
  // Every lane of a row takes part in its sums: rows past the end are worked on as zeros.
  for (int64_t first = (int64_t)blockIdx.x * kRows; first < a.n; first += step) {
    const int64_t row = first + sub;
    const bool in = row < a.n;
    Floats<N> v = joint_load<T, N, kWhole>(a.f, row, a.ldf, c, a), x = joint_load<T, N, kWhole>(a.x, row, a.ldx, c, a);
    Floats<N> g = 1.0f;
    if (a.gate_mode == 2) g = joint_load<T, N, kWhole>(a.gate, row, a.ldg, c, a);
    if (a.gate_mode == 1) g = in ? (float)static_cast<const T*>(a.gate)[row * a.ldg] : 0.0f;
    float mean, rstd;
    if (a.post != ABCD_NORM_NONE) {
      joint_stats<G, N>(a, v, c, a.post, red, turn, mean, rstd);
      v = (v - mean) * rstd * wp + bp;
      if (t == 0 && in) {
        if (a.post_mean) a.post_mean[row] = mean;
        if (a.post_rstd) a.post_rstd[row] = rstd;
      }
    }
    v = x + sc * (g * v);
    if (in && inside) store_vec<T, N, kWhole>(static_cast<T*>(a.y) + row * a.ldy + c, v, a.d - c);
    if (a.pre != ABCD_NORM_NONE) {
      joint_stats<G, N>(a, v, c, a.pre, red, turn, mean, rstd);
      if (in && inside)
        store_vec<T, N, kWhole>(static_cast<T*>(a.z) + row * a.ldz + c, (v - mean) * rstd * wn + bn, a.d - c);
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
  __shared__ float red[2][1][kJointWaves];
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
  // (without a bias S0 does not count, not even an infinite one, which 0 would make a NaN)
  Floats<N> ds = joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f) * s1;
  if (a.post_b) ds += joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f) * s0;
  put(a.dscale, ds);
  put(a.dpre_w, dw);
  put(a.dpre_b, db);
}

// Rows of G lanes, one vector each. The parameters lie in LDS, in fp32, which leaves registers
// for the next row's values, on their way while one is worked on, and for four waves a SIMD
// (8,192 x 4,096 in bf16 with a gate an element: 249 us without either; values that spill are
// dear: 65,536 x 1,024 159 us, with 16 registers in memory 290).
template <typename T, int G, bool kWhole>
__global__ __launch_bounds__(kJointBwdThreads<G>, 4) void residual_norm_bwd_kernel(JointArgs a) {
  constexpr int N = kPer16<T>, kThreads = kJointBwdThreads<G>, kRows = kThreads / G, kWaves = kThreads / 64;
  constexpr int kGroups = G <= 64 ? kWaves : kRows;  // that hold sums of the same columns
  typedef typename Frag<T>::type F;
  __shared__ float red2[2][2][kJointWaves], red3[2][3][kJointWaves];
  __shared__ __align__(16) float params[4][G * N];  // post's weight and bias, pre's weight, scale
  __shared__ float cols[kGroups > 1 ? kGroups : 1][kGroups > 1 ? G * N : 1];
  int turn2 = 0, turn3 = 0;
  const int t = threadIdx.x % G, c = t * N;
  const bool has_pre = a.pre != ABCD_NORM_NONE, has_post = a.post != ABCD_NORM_NONE, inside = c < a.d;
  if ((int)threadIdx.x < G) {
    store_vec<float, N, true>(&params[0][c], joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f), N);
    store_vec<float, N, true>(&params[1][c], joint_param<T, N, kWhole>(a, a.post_b, c, 0.0f), N);
    store_vec<float, N, true>(&params[2][c], joint_param<T, N, kWhole>(a, a.pre_w, c, 1.0f), N);
    store_vec<float, N, true>(&params[3][c], joint_param<T, N, kWhole>(a, a.scale, c, 1.0f), N);
  }
  __syncthreads();
  auto param = [&](int k) { return *reinterpret_cast<const Floats<N>*>(&params[k][c]); };
  Floats<N> s1 = 0.0f, s0 = 0.0f, dw = 0.0f, db = 0.0f;
  F ndy, ndz, ny, nf;
  float nmean, nrstd, npm, npr, none;
  auto load = [&](const void* p, int64_t row, int64_t ld, bool wanted) {
    const int left = row < a.n && wanted ? a.d - c : 0;
    return load_frag<T, kWhole>(static_cast<const T*>(p) + row * ld + c, left, room_of(a.n, row, ld, left));
  };
  auto fetch = [&](int64_t row) {
    const bool in = row < a.n;
    ndy = load(a.dy, row, a.lddy, a.dy != nullptr);
    ndz = load(a.dz, row, a.lddz, has_pre);
    ny = load(a.y, row, a.ldy, has_pre);
    nf = load(a.f, row, a.ldf, true);
    nmean = in && a.pre == ABCD_NORM_LAYER ? a.pre_mean[row] : 0.0f;
    nrstd = in && has_pre ? a.pre_rstd[row] : 0.0f;
    npm = in && a.post == ABCD_NORM_LAYER ? a.post_mean[row] : 0.0f;
    npr = in && has_post ? a.post_rstd[row] : 1.0f;
    none = a.gate_mode == 1 && in ? (float)static_cast<const T*>(a.gate)[row * a.ldg] : 1.0f;
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t first = (int64_t)blockIdx.x * kRows;
  constexpr bool kAhead = G > 64;  // short rows have waves enough without, and need their registers
  // (of whole waves the row is a scalar, and so are its addresses)
  const int sub = G >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / G) : threadIdx.x / G;
  if (kAhead) fetch(first + sub);
  for (; first < a.n; first += step) {
    const int64_t row = first + sub;
    const bool in = row < a.n && inside;
    if (!kAhead) fetch(row);
    const float mean = nmean, rstd = nrstd, pm = npm, pr = npr, one = none;
    auto value = [&](F v) { return __builtin_convertvector((first_of<T, kWhole>(v, a.d - c)), Floats<N>); };
    Floats<N> g = value(ndy), v = value(ndz), h = value(ny);
    const F rf = nf, rg = load(a.gate, row, a.ldg, a.gate_mode == 2);  // the gate is needed last
    if (kAhead) fetch(row + step);
    if (has_pre) {
      float s[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < N; ++i) h[i] = c + i < a.d ? (h[i] - mean) * rstd : 0.0f;
      dw += v * h;
      db += v;
      v *= param(2);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[0] += v[i];
        s[1] += v[i] * h[i];
      }
      joint_sums<G, 2>(s, red2, turn2);
      const float c1 = a.pre == ABCD_NORM_LAYER ? s[0] * a.inv_d : 0.0f, c2 = s[1] * a.inv_d;
      g += rstd * (v - c1 - h * c2);
    }
    if (a.dx && in) store_vec<T, N, kWhole>(static_cast<T*>(a.dx) + row * a.lddx + c, g, a.d - c);
    Floats<N> f = value(rf);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool there = row < a.n && c + i < a.d;
      f[i] = there ? (f[i] - pm) * pr : 0.0f;
      g[i] = there ? g[i] : 0.0f;
    }
    const Floats<N> wp = param(0), sc = param(3);
    const Floats<N> by = g * sc * (f * wp + param(1));  // the gate's
    if (a.dgate && a.gate_mode == 2 && in) store_vec<T, N, kWhole>(static_cast<T*>(a.dgate) + row * a.lddg + c, by, a.d - c);
    if (a.gate_mode == 2)
      g *= value(rg);
    else
      g *= one;
    s1 += g * f;
    s0 += g;
    g *= sc * wp;
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s[0] += g[i];
      s[1] += g[i] * f[i];
      s[2] += by[i];
    }
    if (has_post || a.gate_mode == 1) joint_sums<G, 3>(s, red3, turn3);
    if (a.dgate && a.gate_mode == 1 && row < a.n && t == 0) static_cast<T*>(a.dgate)[row * a.lddg] = (T)s[2];
    if (a.df && in) {
      const float c1 = a.post == ABCD_NORM_LAYER ? s[0] * a.inv_d : 0.0f, c2 = has_post ? s[1] * a.inv_d : 0.0f;
      // without a norm c2 is 0, which an infinity or a NaN of f has to leave so (with one it is a NaN then)
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = __builtin_amdgcn_fmed3f(f[i], -__FLT_MAX__, __FLT_MAX__);
      store_vec<T, N, kWhole>(static_cast<T*>(a.df) + row * a.lddf + c, pr * (g - c1 - f * c2), a.d - c);
    }
  }
  if (!a.part && gridDim.x > 1) return;  // no parameter's gradient is wanted
  if (kGroups == 1) {
    if (!inside) return;
    if (gridDim.x == 1) {
      put_params<T, N, kWhole>(a, c, s1, s0, dw, db);
      return;
    }
    float* const p = a.part + (int64_t)blockIdx.x * 4 * a.pitch + c;
    store_vec<float, N, true>(p, s1, N);
    store_vec<float, N, true>(p + a.pitch, s0, N);
    store_vec<float, N, true>(p + 2 * a.pitch, dw, N);
    store_vec<float, N, true>(p + 3 * a.pitch, db, N);
    return;
  }
  // a wave's rows added across the lanes, then the groups' sums through LDS
  constexpr int kTurns = (G * N + kThreads - 1) / kThreads;
  float own[4][kTurns];
#pragma unroll
  for (int which = 0; which < 4; ++which) {
    const Floats<N> v = which == 0 ? s1 : which == 1 ? s0 : which == 2 ? dw : db;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e = v[i];
      for (int off = G; off < 64; off *= 2) e += __shfl_xor(e, off, 64);
      if (G > 64)
        cols[threadIdx.x / G][c + i] = e;
      else if ((threadIdx.x & 63) < G)
        cols[threadIdx.x >> 6][c + i] = e;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kTurns; ++k) {
      const int at = k * kThreads + threadIdx.x;
      own[which][k] = 0.0f;
      if (at < a.d && at < G * N)
        for (int w = 0; w < kGroups; ++w) own[which][k] += cols[w][at];
    }
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < kTurns; ++k) {
    const int at = k * kThreads + threadIdx.x;
    if (at >= a.d) continue;
    if (gridDim.x == 1)
      put_params<T, 1, true>(a, at, Floats<1>(own[0][k]), Floats<1>(own[1][k]), Floats<1>(own[2][k]), Floats<1>(own[3][k]));
    else
#pragma unroll
      for (int which = 0; which < 4; ++which) a.part[((int64_t)blockIdx.x * 4 + which) * a.pitch + at] = own[which][k];
  }
}

// Long rows: a workgroup per row in three passes, its column sums kept in its part.
template <typename T, bool kWhole>
__global__ __launch_bounds__(kWide) void residual_norm_bwd_wide_kernel(JointArgs a) {
  constexpr int N = kPer16<T>;
  __shared__ float red2[2][2][kJointWaves], red3[2][3][kJointWaves];
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
    const float c3 = a.post == ABCD_NORM_LAYER ? s3[0] * a.inv_d : 0.0f, c4 = s3[1] * a.inv_d;
    for (int c = threadIdx.x * N; c < a.d; c += kWide * N) {
      Floats<N> dz, h;
      Floats<N> g = grad(c, dz, h) * gate_at(c) * joint_param<T, N, kWhole>(a, a.scale, c, 1.0f) *
                    joint_param<T, N, kWhole>(a, a.post_w, c, 1.0f);
      if (has_post) g = pr * (g - c3 - hat(joint_load<T, N, kWhole>(a.f, row, a.ldf, c, a), pm, pr, c) * c4);
      store_vec<T, N, kWhole>(static_cast<T*>(a.df) + row * a.lddf + c, g, a.d - c);
    }
  }
}

// The workgroups' column sums added up in order: 32 columns (128 bytes) of all four a workgroup,
// the parts dealt to its waves (256 parts of 1,001 columns: 4.2 us, with 64 columns of one
// sum after the other 10.6).
constexpr int kJointPartWaves = 16, kJointPartCols = 32;
template <typename T>
__global__ __launch_bounds__(kJointPartWaves* kWave) void residual_norm_sums_kernel(JointArgs a, int64_t parts) {
  typedef VecOf<float, 2>::type F2;
  constexpr int kLanes = kJointPartCols / 2;
  __shared__ F2 red[kJointPartWaves][kWave];
  const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
  const int first = (int)blockIdx.x * kJointPartCols, c = first + l % kLanes * 2;
  const float* const from = a.part + l / kLanes * a.pitch + c;  // (rows of parts are whole vectors)
  F2 s = 0.0f;
  if (c < a.d) {
    int64_t p = w;
    for (; p + 7 * kJointPartWaves < parts; p += 8 * kJointPartWaves) {
      F2 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const F2*>(from + (p + u * kJointPartWaves) * 4 * a.pitch);
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    for (; p < parts; p += kJointPartWaves) s += *reinterpret_cast<const F2*>(from + p * 4 * a.pitch);
  }
  red[w][l] = s;
  __syncthreads();
  if (w == 0) {
    for (int v = 1; v < kJointPartWaves; ++v) s += red[v][l];
    red[0][l] = s;
  }
  __syncthreads();
  if (threadIdx.x < kJointPartCols) {  // (put_params leaves out what lies past the row's end)
    auto sum = [&](int which) { return Floats<1>(red[0][which * kLanes + threadIdx.x / 2][threadIdx.x % 2]); };
    put_params<T, 1, true>(a, first + (int)threadIdx.x, sum(0), sum(1), sum(2), sum(3));
  }
}

// Lanes of a row that a kernel is compiled for; f with the fewest that hold nvec vectors, and
// false if none do.
template <typename F>
bool with_joint_lanes(int nvec, F f) {
  if (nvec <= 8) return f(std::integral_constant<int, 8>{}), true;
  if (nvec <= 16) return f(std::integral_constant<int, 16>{}), true;
  if (nvec <= 32) return f(std::integral_constant<int, 32>{}), true;
  if (nvec <= 64) return f(std::integral_constant<int, 64>{}), true;
  if (nvec <= 128) return f(std::integral_constant<int, 128>{}), true;
  if (nvec <= 256) return f(std::integral_constant<int, 256>{}), true;
  if (nvec <= 512) return f(std::integral_constant<int, 512>{}), true;
  if (nvec <= 1024) return f(std::integral_constant<int, 1024>{}), true;
  return false;
}

template <typename T>
int32_t run_joint(const JointArgs& a, hipStream_t stream) {
  const int nvec = (int)((a.d + kPer16<T> - 1) / kPer16<T>);
  const bool whole = a.d % kPer16<T> == 0;
  const bool held = with_joint_lanes(nvec, [&](auto lanes) {
    constexpr int G = decltype(lanes)::value, kThreads = kJointThreads<G>;
    const int64_t rows = kThreads / G, blocks = std::min<int64_t>((a.n + rows - 1) / rows, G > 64 ? 4096 : 2048);
    if (whole)
      ABCD_LAUNCH("residual_norm", (residual_norm_kernel<T, G, true>), blocks, kThreads, 0, stream, a);
    else
      ABCD_LAUNCH("residual_norm", (residual_norm_kernel<T, G, false>), blocks, kThreads, 0, stream, a);
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
    const bool held = with_joint_lanes(nvec, [&](auto lanes) {
      constexpr int G = decltype(lanes)::value, kThreads = kJointBwdThreads<G>;
      if (whole)
        ABCD_LAUNCH("residual_norm_bwd", (residual_norm_bwd_kernel<T, G, true>), blocks, kThreads, 0, stream, a);
      else
        ABCD_LAUNCH("residual_norm_bwd", (residual_norm_bwd_kernel<T, G, false>), blocks, kThreads, 0, stream, a);
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
    ABCD_LAUNCH("residual_norm_sums", (residual_norm_sums_kernel<T>), (a.d + kJointPartCols - 1) / kJointPartCols,
                kJointPartWaves * kWave, 0, stream, a, a.n == 0 ? 0 : blocks);
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
