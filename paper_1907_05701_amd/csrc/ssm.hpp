// Shared pieces of the state space operators (ssm_scan.hip, ssm_conv.hip):
// dims validation, 4-wide loads and stores of a row piece, the step size's
// softplus, sums over lane groups.
#pragma once

#include "common.hpp"

// Fills nothing; BLSTM_OK or an error code (message set).
int ssm_check_dims(const ssm_dims* d, const char* fn);

// ---------------------------------------------------------------------------
// Four adjacent elements of a row, as floats.  vec: the address is a multiple
// of four elements and all four exist; otherwise the n that exist are read
// one by one and the others are 0.
// ---------------------------------------------------------------------------
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
template <typename T> struct Vec4;
template <> struct Vec4<float> { typedef f32x4 type; };
template <> struct Vec4<bf16> { typedef bf16x4 type; };

template <typename T>
__device__ __forceinline__ typename Vec4<T>::type ld4_raw(const T* p, int n, bool vec) {
  typedef typename Vec4<T>::type V;
  if (vec && n >= 4) return *(const V*)p;
  V v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : (T)0.f;
  return v;
}
template <typename V>
__device__ __forceinline__ f32x4 widen(V v) {
  f32x4 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = (float)v[i];
  return f;
}
template <typename T>
__device__ __forceinline__ void st4(T* p, f32x4 f, int n, bool vec) {
  typedef typename Vec4<T>::type V;
  V v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = from_f32<T>(f[i]);
  if (vec && n >= 4) {
    *(V*)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = v[i];
  }
}

// softplus(v) = max(v, 0) + log(1 + e), e = e^-|v| in (0, 1].  Steps of 1e-3
// and less are ordinary, where 1 + e has lost e's low bits, so the logarithm
// goes by log(1 + e) = 2 artanh(q), q = e / (2 + e) <= 1/3, and the series
// 2 q (1 + q^2/3 + q^4/5 + ...) whose first term left out is below 9^-8 / 17 of
// the sum: relative accuracy at every v, at about a fifth of log1pf's
// instructions.  A NaN stays one (the maximum is not taken by fmaxf).
__device__ __forceinline__ float softplusf_(float v) {
  const float e = __expf(-fabsf(v));
  const float q = e * __builtin_amdgcn_rcpf(2.f + e), w = q * q;
  float p = 1.f / 15.f;
  p = p * w + 1.f / 13.f;
  p = p * w + 1.f / 11.f;
  p = p * w + 1.f / 9.f;
  p = p * w + 1.f / 7.f;
  p = p * w + 1.f / 5.f;
  p = p * w + 1.f / 3.f;
  return (v < 0.f ? 0.f : v) + 2.f * q * (p * w + 1.f);
}
// silu'(v) = p (1 + v (1 - p)), p = sigmoid(v)
__device__ __forceinline__ float dsiluf_(float v) {
  const float p = sigmoidf_(v);
  return p * (1.f + v * (1.f - p));
}
// v sigmoid(v); where e^-v overflows the sigmoid is 0 and so is the product
__device__ __forceinline__ float siluf_(float v) { return v * sigmoidf_(v); }

// ---------------------------------------------------------------------------
// Sums over lanes within a row of 16 by DPP.
// ---------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// over the LPC adjacent lanes of an aligned group; every lane gets the sum
template <int LPC>
__device__ __forceinline__ float group_sum(float v) {
  if constexpr (LPC >= 2) v = dpp_add<0xB1>(v);    // quad_perm [1,0,3,2]
  if constexpr (LPC >= 4) v = dpp_add<0x4E>(v);    // quad_perm [2,3,0,1]
  if constexpr (LPC >= 8) v = dpp_add<0x141>(v);   // row_half_mirror: the other quad of 8 (each holds its sum)
  if constexpr (LPC >= 16) v = dpp_add<0x140>(v);  // row_mirror: the other half of 16
  return v;
}
// over the lanes of a row that are equal modulo LPC
template <int LPC>
__device__ __forceinline__ float stride_sum(float v) {
  if constexpr (LPC <= 8) v = dpp_add<0x128>(v);   // row_ror 8, 4, 2, 1
  if constexpr (LPC <= 4) v = dpp_add<0x124>(v);
  if constexpr (LPC <= 2) v = dpp_add<0x122>(v);
  if constexpr (LPC <= 1) v = dpp_add<0x121>(v);
  return v;
}
