// Products in 8-bit integers (int8*.hip): what their kernels share.
#pragma once

#include "common.hpp"

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// v_mfma_i32_16x16x64_i8: lane l supplies 16 consecutive k (from 16 (l / 16)) of row l % 16 of A
// and of column l % 16 of B, and receives rows 4 (l / 16) .. + 3 of column l % 16.
__device__ __forceinline__ i32x4 mma_i8(i32x4 a, i32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// ---------------------------------------------------------------------------
// A token's integers: q = 127 x / max |x| to the nearest, ties to the even one,
// scale = max |x| / 127.  The product x (127 / max) is off by less than
// 127 * 3 * 2^-24 < 2.5e-5, so that only within that of a half the nearest one is in doubt; there
// 127 x is compared with the half times max |x| in 64 bits, where both are exact (31 and 32 bits).
// A token with a NaN or an infinite value has a NaN for its scale and integers of 0.
// ---------------------------------------------------------------------------
struct Quant {
  float amax, pre, inv, scale;
  __device__ __forceinline__ explicit Quant(float max_abs) {
    scale = max_abs / 127.0f;
    // far below 1 the inverse would overflow: both sides times 2^64, exactly
    pre = max_abs < 1e-30f ? 0x1p64f : 1.0f;
    amax = max_abs * pre;
    inv = amax > 0.f ? 127.0f / amax : 0.f;
    if (!(max_abs < INFINITY)) {
      scale = NAN;
      inv = 0.f;
    }
  }
  __device__ __forceinline__ int operator()(float x) const {
    const float v = x * pre, t = v * inv;
    float n = rintf(t);
    if (fabsf(t - n) > 0.4999f) {
      const double lo = floor((double)t), a = (double)v * 127.0, b = (double)amax * (lo + 0.5);
      const bool odd = (int)lo & 1;
      n = (float)(a > b || (a == b && odd) ? lo + 1.0 : lo);
    }
    return inv == 0.f ? 0 : (int)n;
  }
};
__device__ __forceinline__ uint32_t pack4(int a, int b, int c, int d) {
  return (uint32_t)(a & 255) | (uint32_t)(b & 255) << 8 | (uint32_t)(c & 255) << 16 | (uint32_t)d << 24;
}

// 16 values of a row from column k on, as an MFMA lane takes them (0 behind column K).
template <typename TI> struct Lane16 { TI v[16]; };
template <typename TI>
__device__ __forceinline__ void lane16_load(Lane16<TI>& o, const TI* row, int k, int K) {
  constexpr int V = 16 / sizeof(TI);
#pragma unroll
  for (int i = 0; i < 16; i += V) {
    if (k + i + V <= K) {
      __builtin_memcpy(o.v + i, row + k + i, 16);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[i + j] = k + i + j < K ? row[k + i + j] : from_f32<TI>(0.f);
    }
  }
}
__device__ __forceinline__ float max_abs(float m, float v) {   // a NaN stays
  const float a = fabsf(v);
  return m > a || m != m ? m : a;
}
template <typename TI>
__device__ __forceinline__ float lane16_max(const Lane16<TI>& x, float m) {
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max_abs(m, to_f32(x.v[i]));
  return m;
}
template <typename TI>
__device__ __forceinline__ i32x4 lane16_ints(const Lane16<TI>& x, const Quant& to) {
  i32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = (int)pack4(to(to_f32(x.v[4 * i])), to(to_f32(x.v[4 * i + 1])), to(to_f32(x.v[4 * i + 2])), to(to_f32(x.v[4 * i + 3])));
  return r;
}

// A sum of products as a number: each step a single float32 rounding.
__device__ __forceinline__ float int8_value(int sum, float scale, float bias) {
#pragma clang fp contract(off)
  return (float)sum * scale + bias;
}
__device__ __forceinline__ float scale_of(float x_scale, float w_scale) {
#pragma clang fp contract(off)
  return x_scale * w_scale;
}

// Before the barrier of a two-stage ring: this wave's loads into the next stage have landed, and its reads of the one that
// is filled next are done.
__device__ __forceinline__ void int8_stage_wait() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// Most columns of a row: 2^14 times them stays within int32.
static constexpr int INT8_MAX_K = (1 << 17) - 16;
// Longest row pitch: 256 rows within a buffer resource's 31 bits.
static constexpr int64_t INT8_MAX_LD = 1 << 22;

// Rows of x (TI) to integers of Kq columns (those from K on zero) and scales.
template <typename TI>
void int8_quantize(const TI* x, int64_t ldx, int64_t M, int32_t K, int8_t* q, int64_t ldq, int32_t Kq, float* scale,
                   hipStream_t stream);

// Log probabilities of a head of K classes from tokens x [M][P] (int8_head.hip); buf: int8_head_bytes.  For up to
// so many columns:
bool int8_head_fits(int32_t Kw);
size_t int8_head_bytes(int64_t M, int32_t K, int32_t Kw);
template <typename TI>
int int8_head(const TI* x, int64_t ldx, int64_t M, int32_t P, const int8_t* w, int64_t ldw, const float* ws, int32_t K,
              int32_t Kw, const float* bias, const softmax_scores& scores, char* buf, hipStream_t stream);
