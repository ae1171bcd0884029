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
// scale = max |x| / 127.  With 127 / max |x| as a float32 and the rest of it, t = x hi + (x lo) is the nearest float32 to
// 127 x / max |x|, or its neighbour; a tie is a float32, so that t is the tie then, and adding MAGIC rounds it to the even integer.
//   bf16 values (8 bits each) are ties or further than 2^-16 from one, and t is within 2^-17: nothing is in doubt.
//   float32 values may lie so near a tie that t is the tie: there 127 x is compared with the half times max |x|, each
//   as a product and its rounding error; both have at most 32 bits and are close, so that the difference is exact.
// (With a rounded quotient alone a tie goes either way, and ties are common: one of about 500 bf16 values, x = max / 2
// for one.)  A token with a NaN or an infinite value has a NaN for its scale and integers of 0.
// ---------------------------------------------------------------------------
struct Quant {
  static constexpr float MAGIC = 12582912.0f;   // 1.5 * 2^23: a sum with it is rounded to a whole number, its low byte the integer's
  float amax, hi, lo, scale;
  bool none, tiny;
  // bits: the largest |x| as a word (as words, magnitudes order as floats do, NaN above infinity)
  __device__ __forceinline__ explicit Quant(uint32_t bits) : amax(__uint_as_float(bits)) {
    none = !(amax > 0.f && amax < INFINITY);
    scale = amax < INFINITY ? amax / 127.0f : NAN;
    tiny = amax < 1e-30f;   // the quotient would overflow: values and their maximum times 2^64, exactly
    if (tiny) amax *= 0x1p64f;
    hi = none ? 0.f : 127.0f / amax;
    lo = none ? 0.f : fmaf(-hi, amax, 127.0f) / amax;
  }
  // the same by comparison with the half next to n
  __device__ __forceinline__ float nearest(float x, float n, float way) const {
#pragma clang fp contract(off)
    const float pre = amax > 1e30f ? 0x1p-64f : 1.f, v = x * pre, am = amax * pre, h = n + 0.5f * way;
    const float p = am * h, pl = __builtin_fmaf(am, h, -p), q = v * 127.0f, ql = __builtin_fmaf(v, 127.0f, -q);
    const float d = ((q - p) + (ql - pl)) * way;   // beyond the half?
    return d > 0.f || (d == 0.f && ((int)n & 1)) ? n + way : n;
  }
  // N adjacent values, 4 a word.
  template <typename TI, int N>
  __device__ __forceinline__ void operator()(const TI (&x)[N], uint32_t (&w)[N / 4]) const {
    float v[N];
    uint32_t q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_f32(x[i]);
    if (tiny) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] *= 0x1p64f;
    }
    float far = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = fmaf(v[i], hi, v[i] * lo), f = t + MAGIC;
      if constexpr (sizeof(TI) == 4) far = fmaxf(far, fabsf(t - (f - MAGIC)));
      q[i] = __float_as_uint(f);
    }
    if constexpr (sizeof(TI) == 4) {
      if (far == 0.5f && !none) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float t = fmaf(v[i], hi, v[i] * lo), n = rintf(t);
          if (fabsf(t - n) == 0.5f) q[i] = (uint32_t)(int)nearest(v[i], n, t < n ? -1.f : 1.f);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      // low bytes: v_perm_b32's selectors 0-3 name its second operand's bytes, 4-7 its first's
      const uint32_t a = __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400), b = __builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x04000c0c);
      w[i] = none ? 0u : a | b;
    }
  }
};

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t m) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  return m;
}
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
// V adjacent values of a row: 16 bytes, 0 behind column K.
template <typename TI> struct Vec16 {
  static constexpr int n = 16 / sizeof(TI);
  TI v[n];
  // Without branches, so that many loads go out before one is waited for: a vector that is not whole reads the row's first
  // one and counts as zeros.  (Where K >= n.)  patch() then gives the one that ends behind K its values.
  __device__ __forceinline__ void load(const TI* row, int c, int K) {
    const bool in = c + n <= K;
    uint32_t w[4];
    __builtin_memcpy(w, row + (in ? c : 0), 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = in ? w[j] : 0;
    __builtin_memcpy(v, w, 16);
  }
  __device__ __forceinline__ void patch(const TI* row, int c, int K) {
    if (c < K && c + n > K) {
#pragma unroll
      for (int j = 0; j < n; ++j) v[j] = c + j < K ? row[c + j] : from_f32<TI>(0.f);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < n; ++j) v[j] = from_f32<TI>(0.f);
  }
  // the largest magnitude so far: m in the type's own words (two of 16 bits side by side), word() as a float's
  __device__ __forceinline__ uint32_t max(uint32_t m) const {
    uint32_t w[4];
    __builtin_memcpy(w, v, 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(TI) == 2) {
        const uint32_t a = w[j] & 0x7fff7fffu;
        m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, a)));
      } else {
        m = ::max(m, w[j] & 0x7fffffffu);
      }
    }
    return m;
  }
  static __device__ __forceinline__ uint32_t word(uint32_t m) {
    return sizeof(TI) == 2 ? ::max(m << 16, m & 0xffff0000u) : m;
  }
};

// A few tokens to integers in LDS, by a workgroup of NW waves: each takes every NW-th row, R of them at a time,
// of up to NV vectors a lane.  Rows of `cols` bytes at a pitch of cols + 16, columns from K on zero; then their scales.
// (A pitch of an odd number of 16-byte pieces: 16 rows' pieces at one column lie in 16 different bank groups.)
template <typename TI, int NW, int R, int NV>
__device__ __forceinline__ void tokens_to_lds(const TI* x, int64_t ldx, int rows, int K, int cols, char* dst, float* scales) {
  constexpr int V = Vec16<TI>::n;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int r0 = wid; r0 < rows; r0 += NW * R) {
    Vec16<TI> v[R][NV];
    const TI* row[R];
#pragma unroll
    for (int i = 0; i < R; ++i) row[i] = x + min(r0 + NW * i, rows - 1) * ldx;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (K >= V) v[i][j].load(row[i], (j * 64 + lane) * V, K);
        else v[i][j].zero();
      }
    if (K % V) {
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < NV; ++j) v[i][j].patch(row[i], (j * 64 + lane) * V, K);
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (r0 + NW * i < rows) {
        uint32_t mx = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) mx = v[i][j].max(mx);
        const Quant to(wave_max_bits(Vec16<TI>::word(mx)));
        if (lane == 0) scales[r0 + NW * i] = to.scale;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = (j * 64 + lane) * V;
          uint32_t w[V / 4];
          to(v[i][j].v, w);
          if (c < cols) __builtin_memcpy(dst + (r0 + NW * i) * (cols + 16) + c, w, V);
        }
      }
  }
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

// 16 integers of a row from column k on; zeros behind column K (at least 16), without a branch.
__device__ __forceinline__ i32x4 ints16(const int8_t* row, int k, int K) {
  const i32x4 v = *(const i32x4*)(row + min(k, K - 16));
  const bool in = k < K;
  return i32x4{in ? v[0] : 0, in ? v[1] : 0, in ? v[2] : 0, in ? v[3] : 0};
}

// Most columns of a row: 2^14 times them stays within int32.
static constexpr int INT8_MAX_K = (1 << 17) - 16;
// Longest row pitch: 256 rows within a buffer resource's 31 bits.
static constexpr int64_t INT8_MAX_LD = 1 << 22;

// Rows of x (TI) to integers of Kq columns (those from K on zero) and scales.
template <typename TI>
void int8_quantize(const TI* x, int64_t ldx, int64_t M, int32_t K, int8_t* q, int64_t ldq, int32_t Kq, float* scale,
                   hipStream_t stream);

// Log probabilities of a head of K classes from tokens x [M][P] (int8_head.hip); buf: int8_head_bytes of as many frames or more.  For up to
// so many columns:
bool int8_head_fits(int32_t Kw);
size_t int8_head_bytes(int64_t M, int32_t K, int32_t Kw);
template <typename TI>
int int8_head(const TI* x, int64_t ldx, int64_t M, int32_t P, const int8_t* w, int64_t ldw, const float* ws, int32_t K,
              int32_t Kw, const float* bias, const softmax_scores& scores, char* buf, hipStream_t stream);
