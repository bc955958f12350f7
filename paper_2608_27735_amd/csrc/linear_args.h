// linear_args.h -- arguments of the linear layer's kernels, and their launchers by
// element type.
#pragma once

#include "gated_ffn_args.h"

namespace abcd {

// What a forward keeps of act's derivative: float in fp32; in 16-bit types, as it lies between
// -0.13 and 1.13, a code of 16 bits: 30,800 times its root, with its sign. A slope s is so off by
// up to sqrt(s) / 30,800, half a step: 2^-15 of a slope of 1, 2^-12 of one of 0.02 and 2^-11, which
// float16's half a step is of any, of one of 0.0044; of smaller ones (sigmoid's beyond 5.4, the
// others' tails) it is more, 2^-10 at 0.001 and 2^-5 at 10^-6, and float16's less. Kept in the
// rows' type its rounding would be as large as dz's. -32768 is a NaN.
template <typename T>
using SlopeOf = std::conditional_t<sizeof(T) == 4, float, int16_t>;
constexpr float kSlopeUnit = 30800.0f;
template <int N>
__device__ __forceinline__ void store_slopes(float* p, Floats<N> s) {
  store_vec<float, N, true>(p, s, N);
}
template <int N>
__device__ __forceinline__ void store_slopes(int16_t* p, Floats<N> s) {
  typedef typename VecOf<int16_t, N>::type V;
  V q;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float r = __builtin_rintf(__builtin_amdgcn_sqrtf(fabsf(s[i])) * kSlopeUnit);
    q[i] = s[i] == s[i] ? (int16_t)(int)copysignf(r, s[i]) : (int16_t)-32768;
  }
  *reinterpret_cast<V*>(p) = q;
}
template <int N>
__device__ __forceinline__ Floats<N> slopes_of(typename VecOf<int16_t, N>::type q) {
  Floats<N> s;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float v = (float)q[i];
    s[i] = q[i] == -32768 ? __builtin_nanf("") : v * fabsf(v) * (1.0f / (kSlopeUnit * kSlopeUnit));
  }
  return s;
}
template <int N>
__device__ __forceinline__ Floats<N> load_slopes(const float* p) {
  return load_vec<float, N, true>(p, N);
}
template <int N>
__device__ __forceinline__ Floats<N> load_slopes(const int16_t* p) {
  return slopes_of<N>(*reinterpret_cast<const typename VecOf<int16_t, N>::type*>(p));
}

// y = res + act(x w' + bias); slope: act's derivative, [n][ldslope], columns past o zeros.
struct LinearOut {
  Side x, w;
  const void* bias;
  const void* res;
  void* y;
  void* slope;  // NULL: not kept
  int64_t i, o, ldr, ldy, ldslope;
  int act;
  Tiling t;
  const void* dy = nullptr;  // linear_few: given, y is dz = dy act'(x w' + bias), columns up to ldy zeros
  int64_t lddy = 0;
  // the sums of dz's rows: db itself of up to 16 rows, else part: [few_parts(n)][o], of 16 rows each
  // (both NULL: not wanted)
  void* db = nullptr;
  float* part = nullptr;
};
inline int64_t few_parts(int64_t n) { return n <= 16 ? 1 : n <= 32 ? 2 : 4; }
// dz = dy act'(x w' + bias): [n][lddz], columns past o zeros.
struct LinearDz {
  Side x, w;
  const void* bias;
  const void* dy;
  void* dz;
  int64_t i, o, lddy, lddz;
  int act;
  Tiling t;
};
// dx = dz w
struct LinearDx {
  Side dz, w;
  void* dx;
  int64_t o, i, lddx;
  Tiling t;
};
// dz = dy slope, of n rows; without slopes and dz nothing but the sums: part: [parts][o], the
// sums of dz's rows before it is rounded (NULL: not wanted), or db itself where one part is all
struct LinearSlope {
  const void* dy;
  const void* slope;
  void* dz;
  float* part;
  void* db;
  int64_t n, o, lddy, ldslope, lddz;
  int lanes;  // threads along a row, 8 columns each
};

// Narrow rows, 16-bit types.
struct LinearNarrow {
  const void *x, *w, *bias, *res;
  void *y, *slope;
  int64_t n, i, o, ldx, ldr, ldy, ldslope;
  int act;
};
// x, or q and e; part: [workgroups][o i + o], the sums of dw and db, NULL: neither is wanted
struct LinearNarrowBwd {
  const void* x;
  const int8_t* q;
  const uint8_t* e;
  const void *dy, *slope, *w, *bias;
  void* dx;
  float* part;
  int64_t n, i, o, ldx, lddy, ldslope, lddx;
  int act;
};
inline bool narrow_layer(int64_t i, int64_t o) { return i <= 256 && o <= 256 && (i <= 128 || o <= 128); }
inline bool narrow_layer_bwd(int64_t i, int64_t o) { return i <= 128 && o <= 128 && (i <= 64 || o <= 64); }
int32_t linear_narrow_f16(const LinearNarrow&, int64_t blocks, hipStream_t);
int32_t linear_narrow_bf16(const LinearNarrow&, int64_t blocks, hipStream_t);
int32_t linear_narrow_bwd_f16(const LinearNarrowBwd&, int64_t blocks, hipStream_t);
int32_t linear_narrow_bwd_bf16(const LinearNarrowBwd&, int64_t blocks, hipStream_t);

#define ABCD_LINEAR_DECLARE(NAME)                               \
  int32_t linear_out_##NAME(const LinearOut&, hipStream_t);     \
  int32_t linear_few_##NAME(const LinearOut&, hipStream_t);     \
  int32_t linear_dz_##NAME(const LinearDz&, hipStream_t);       \
  int32_t linear_dx_##NAME(const LinearDx&, hipStream_t);       \
  int32_t linear_dw_##NAME(const FfnDWeight&, hipStream_t);     \
  int32_t linear_slope_##NAME(const LinearSlope&, int64_t parts, hipStream_t);
ABCD_LINEAR_DECLARE(f32)
ABCD_LINEAR_DECLARE(f16)
ABCD_LINEAR_DECLARE(bf16)
#undef ABCD_LINEAR_DECLARE

}  // namespace abcd
