// Rows of logits, one workgroup a row: how a row is held and read, sums and
// maxima over it, its k largest, and the choice of threads by its length.
#pragma once

#include <float.h>
#include <math.h>

#include <type_traits>

#include "common.hpp"

#define LOG2E_F 1.4426950408889634f
#define LN2_F 0.6931471805599453f
static_assert(SOFTMAX_MAX_CLASSES == 1 << 18, "bits of a class");
static constexpr int RT = 256;             // least threads of a row with MAXK entries (T below: 256, 512 or 1024; 64 with few)
static constexpr int CAND = 1024;          // most candidates kept in LDS
static constexpr int MAXK = SOFTMAX_MAX_TOP;
static_assert(MAXK <= RT && MAXK <= CAND, "an entry a thread; the k-th largest of the threads' maxima bounds the k-th logit");

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// Sum and maximum over the workgroup, in lane and wave order; buf: T / 64 floats.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
template <int T>
__device__ __forceinline__ float row_sum(float v, float* buf) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = buf[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) t += buf[w];
  return t;
}
// a NaN among the values is the maximum
__device__ __forceinline__ float max_nan(float a, float b) { return (a > b || a != a) ? a : b; }
template <int T>
__device__ __forceinline__ float row_max(float v, float* buf) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max_nan(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = buf[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) t = max_nan(t, buf[w]);
  return t;
}

// Adjacent elements that a thread reads at once: 16 bytes.  Rows of any pitch
// and start are read so (global memory takes 16-byte accesses at an element's alignment).
template <typename TI> struct Wide;
template <> struct Wide<float> { typedef f32x4 type; static constexpr int n = 4; };
template <> struct Wide<bf16> { typedef bf16x8 type; static constexpr int n = 8; };

// A row in registers: vector i of thread t holds columns (i T + t) V and on, as
// far as whole vectors go; the fewer than V columns behind them are one a
// thread.  What does not exist is -inf.  bf16 pairs stay packed; again() between passes
// keeps the compiler from carrying widened values and exponentials from one pass to the next.
template <typename TI, int V, int NV, int T> struct Row {
  static constexpr bool PACKED = sizeof(TI) == 2 && V > 1;
  static constexpr int W = PACKED ? V / 2 : V;   // words of a vector
  uint32_t w[NV][W];
  float tail;
  static __device__ __forceinline__ int col(int i) { return (i * T + (int)threadIdx.x) * V; }
  static __device__ __forceinline__ int whole(int K) { return K / V * V; }
  // vector i's address (a base that the workgroup shares and 32 bits of the
  // thread's own), and whether it exists
  template <typename P> static __device__ __forceinline__ P* at(P* s, int i) {
    typedef typename std::conditional<std::is_const<P>::value, const char, char>::type C;
    return (P*)((C*)(s + i * T * V) + (uint32_t)(threadIdx.x * (V * sizeof(P))));
  }
  static __device__ __forceinline__ bool has(int i, int n) { return (int)threadIdx.x * V < n - i * T * V; }
  // the thread's column behind the whole vectors (K or more: none)
  static __device__ __forceinline__ int tail_col(int K) { return V == 1 ? K : whole(K) + (int)threadIdx.x; }
  __device__ __forceinline__ float get(int i, int j) const {
    if constexpr (!PACKED) return __uint_as_float(w[i][j]);
    else return __uint_as_float(j & 1 ? w[i][j >> 1] & 0xffff0000u : w[i][j >> 1] << 16);
  }
  __device__ __forceinline__ void drop(int i, int j) {   // -inf
    if constexpr (!PACKED) w[i][j] = 0xff800000u;
    else w[i][j >> 1] = j & 1 ? (w[i][j >> 1] & 0xffffu) | 0xff800000u : (w[i][j >> 1] & 0xffff0000u) | 0xff80u;
  }
  __device__ __forceinline__ void again() {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) asm volatile("" : "+v"(w[i][j]));
  }
  __device__ __forceinline__ void load(const TI* s, int K) {
    const int n = whole(K);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[i][j] = PACKED ? 0xff80ff80u : 0xff800000u;
      if (has(i, n)) {
        if constexpr (V == 1) w[i][0] = __float_as_uint(to_f32(*at(s, i)));
        else __builtin_memcpy(w[i], at(s, i), V * sizeof(TI));
      }
    }
    tail = tail_col(K) < K ? to_f32(s[tail_col(K)]) : -INFINITY;
  }
};

// Waves of a SIMD that the registers are kept to.  Three rows on a CU instead
// of two hide more of each other's barriers and waits: 2688 bf16 rows of 32000 (64
// values a thread) 4 waves 56.5, 6 waves 49.3 us for the top, 82 and 77 for the loss with labels at
// temperature 1, 95 and 88 at 3, although six waves spill one register at temperature 2 and two at others than
// 1 and 2.  float32 rows of 64 values have no room for it.  (8 waves: the top of 12000 bf16 rows of 9001, 32
// values a thread, 95 us, with 6 114.)
template <typename TI, int T, int V, int NV> constexpr int waves_of() {
  if (NV == 0 || T > 512) return 4;
  if (V * NV * sizeof(TI) <= 64) return 8;
  return V * NV <= 32 || sizeof(TI) == 2 ? 6 : 4;
}

// Rows longer than registers hold: calls f(column, value) for the thread's
// columns, read from memory (the caches) by every pass.
// ONE: element by element, in fewer registers.
template <typename TI, int T, bool ONE = false, typename F>
__device__ __forceinline__ void each(const TI* s, int K, F f) {
  if constexpr (ONE) {
#pragma unroll 4
    for (int c = (int)threadIdx.x; c < K; c += T) f(c, to_f32(s[c]));
    return;
  }
  constexpr int V = Wide<TI>::n;
  const int done = K / V * V;
  for (int c = (int)threadIdx.x * V; c < done; c += 4 * T * V) {   // four loads in flight
    TI v[4][V];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (c + u * T * V < done) __builtin_memcpy(v[u], s + c + u * T * V, V * sizeof(TI));
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (c + u * T * V >= done) break;
#pragma unroll
      for (int i = 0; i < V; ++i) f(c + u * T * V + i, to_f32(v[u][i]));
    }
  }
  const int c = done + (int)threadIdx.x;
  if (c < K) f(c, to_f32(s[c]));
}

// Order of logits as unsigned words: larger logit, larger word; both zeros
// alike, every NaN on top.
__device__ __forceinline__ uint32_t order_word(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);   // -0 + 0 = +0
  if (v != v) return 0xffffffffu;
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t w) {
  return w == 0xffffffffu ? __uint_as_float(0x7fc00000u)
                          : __uint_as_float((w & 0x80000000u) ? w & 0x7fffffffu : ~w);
}

// ---------------------------------------------------------------------------
// The k largest of a row.  Each thread's maximum is one of T; the k-th
// largest of those is no larger than the row's k-th, and few logits lie above
// it (about T ln(T / (T - k)) of them in no particular order), so the
// logits from there on are collected and ranked by counting.  Rows whose
// logits bunch (ties, or all large ones in one thread's columns) can have
// more than CAND candidates: their k-th logit, and the last class that ties
// with it, are then found bit by bit.
// ---------------------------------------------------------------------------
// (T threads; room for C candidates, and for N maxima)
template <int T, int C = CAND, int N = T> struct TopkLds {
  uint32_t tmax[N];
  uint64_t cand[C];   // order word, complement of the class; in the order of arrival
  float left[C];      // logits of the candidates behind the k-th, in their order
  uint32_t thr, count, cnt[2][T / 64], flag;
  uint64_t kth;
  float buf[T / 64];
};
static constexpr uint32_t LOWEST = 0x007fffffu;   // order word of -inf
struct TopkP {
  int64_t ld;
  int K, k;
  float l2t;   // log2 e / temperature
  float *top, *rest;
  int32_t* idx;
};

// A word of LDS that every lane reads alike, as a scalar: a branch on it is one
// for the whole wave, and what lives on past the branch not taken takes no registers from it.
__device__ __forceinline__ uint32_t same(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// The k-th largest of the threads' maxima (order words), down to its bits from
// LOW on; where k is small, of the maxima of groups of 4 or 8 threads, two words a
// lane: a few more logits pass (37 instead of 33 of a row of 32 from 512 threads), and each step of
// the search takes a quarter of the instructions.
template <int LOW, int NW>
__device__ __forceinline__ uint32_t kth_word(const uint32_t (&w)[NW], int k) {
  uint32_t t = 0;
  for (int bit = 31; bit >= LOW; --bit) {
    const uint32_t c = t | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) n += __popcll(__ballot(w[i] >= c));
    if (n >= k) t = c;
  }
  return t;
}
static constexpr int FOLD = 64;   // largest k for groups
// (of one wave, behind a barrier; fold: largest k for groups here)
template <int LOW, int T, int C, int N>
__device__ __forceinline__ uint32_t kth_search(const TopkLds<T, C, N>& l, int k, int fold = FOLD) {
  const int lane = threadIdx.x & 63;
  constexpr int NW = N / 64;
  uint32_t w[NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) w[i] = l.tmax[i * 64 + lane];
  if constexpr (NW > 2) {
    if (k <= fold) {
      uint32_t g[2] = {w[0], w[1]};
#pragma unroll
      for (int i = 2; i < NW; ++i) g[i & 1] = max(g[i & 1], w[i]);
      return kth_word<LOW>(g, k);
    }
  }
  return kth_word<LOW>(w, k);
}
template <int LOW, int T, int C, int N>
__device__ __forceinline__ uint32_t kth_max(TopkLds<T, C, N>& l, int k) {
  __syncthreads();
  if (threadIdx.x < 64) {
    const uint32_t t = kth_search<LOW>(l, k);
    if ((threadIdx.x & 63) == 0) l.thr = t;
  }
  __syncthreads();
  return l.thr;
}
template <int T, int C, int N>
__device__ __forceinline__ void push(TopkLds<T, C, N>& l, float v, int c) {
  const uint32_t at = atomicAdd(&l.count, 1u);
  if (at < (uint32_t)C) l.cand[at] = ((uint64_t)order_word(v) << 32) | (uint32_t)~c;
}
// Writes the k largest of n candidates as value(logit), and what is left to l.left (so that
// sums over it do not depend on who arrived first).
struct Itself {
  __device__ __forceinline__ float operator()(float v) const { return v; }
};
template <int T, int C, int N, typename F = Itself>
__device__ __forceinline__ void rank(TopkLds<T, C, N>& l, int n, int64_t m, const TopkP& p, F value = F()) {
  for (int i = threadIdx.x; i < n; i += T) {
    const uint64_t w = l.cand[i];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) r += l.cand[j] > w;
    if (r < p.k) {
      p.top[m * p.k + r] = value(order_value((uint32_t)(w >> 32)));
      p.idx[m * p.k + r] = (int32_t)~(uint32_t)w;
      if (r == p.k - 1) l.kth = w;
    } else {
      l.left[r - p.k] = order_value((uint32_t)(w >> 32));
    }
  }
}

// The log-sum-exp of what orders behind the k-th, from its own maximum, from memory.
template <typename TI, int T, bool ONE, int C>
__device__ __forceinline__ void rest_of(TopkLds<T, C>& l, const TI* s, int64_t m, const TopkP& p) {
  const int tid = threadIdx.x, K = p.K;
  const uint64_t last = l.kth;
  float rm = -INFINITY;
  each<TI, T, ONE>(s, K, [&](int c, float v) {
    if ((((uint64_t)order_word(v) << 32) | (uint32_t)~c) < last) rm = max_nan(rm, v);
  });
  rm = row_max<T>(rm, l.buf);
  float sum = 0.f;
  if (fabsf(rm) < INFINITY) {
    each<TI, T, ONE>(s, K, [&](int c, float v) {
      if ((((uint64_t)order_word(v) << 32) | (uint32_t)~c) < last) sum += exp2_((v - rm) * p.l2t);
    });
  }
  sum = row_sum<T>(sum, l.buf);
  // the others' largest logit alone where it is infinite or a NaN, or there is none
  if (tid == 0) p.rest[m] = fabsf(rm) < INFINITY ? rm * (p.l2t * LN2_F) + log2f(sum) * LN2_F : rm;
}

// Any row, from memory.
template <typename TI, int T, bool ONE, int C, typename F = Itself>
__device__ __forceinline__ void topk_any(TopkLds<T, C>& l, const TI* s, int64_t m, const TopkP& p, F value = F()) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K;
  uint32_t mx = 0;
  each<TI, T, ONE>(s, K, [&](int, float v) { mx = max(mx, order_word(v)); });
  __syncthreads();
  l.tmax[tid] = mx;
  if (tid == 0) l.count = 0;
  const uint32_t th = kth_max<0>(l, p.k);
  each<TI, T, ONE>(s, K, [&](int c, float v) {
    if (order_word(v) >= th) push(l, v, c);
  });
  __syncthreads();
  int n = (int)min(same(l.count), (uint32_t)C);
  if (same(l.count) > (uint32_t)C) {
    // the k-th: the largest word (and complement of the class) with k of them from it on
    uint64_t t = 0;
    int par = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t c = t | (1ull << bit);
      if (bit < 32 && bit >= 18) {   // set in the complement of every class
        t = c;
        continue;
      }
      uint32_t mine = 0;
      each<TI, T, ONE>(s, K, [&](int col, float v) {
        mine += ((((uint64_t)order_word(v)) << 32) | (uint32_t)~col) >= c;
      });
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
      if (lane == 0) l.cnt[par][wave] = mine;
      __syncthreads();
      uint32_t all = 0;
#pragma unroll
      for (int i = 0; i < T / 64; ++i) all += l.cnt[par][i];
      if (all >= (uint32_t)p.k) t = c;
      par ^= 1;
    }
    if (tid == 0) l.count = 0;
    __syncthreads();
    each<TI, T, ONE>(s, K, [&](int c, float v) {
      if ((((uint64_t)order_word(v) << 32) | (uint32_t)~c) >= t) push(l, v, c);   // exactly k
    });
    __syncthreads();
    n = p.k;
  }
  rank(l, n, m, p, value);
  if (!p.rest) return;
  __syncthreads();
  rest_of<TI, T, ONE>(l, s, m, p);
}

// Joins a wave's values into buf; after a barrier all_sum and all_max join the waves'.
// NAN_MAX: a NaN is the maximum (a teacher's is seen so; a student's is in the sums).
template <bool NAN_MAX = false> __device__ __forceinline__ float max_of(float a, float b) { return NAN_MAX ? max_nan(a, b) : fmaxf(a, b); }
template <bool NAN_MAX = false>
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max_of<NAN_MAX>(v, __shfl_xor(v, o));
  return v;
}
__device__ __forceinline__ void put_wave(float* buf, float v) {
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
}
template <int T>
__device__ __forceinline__ float all_sum(const float* buf) {
  float t = buf[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) t += buf[w];
  return t;
}
template <int T, bool NAN_MAX = false>
__device__ __forceinline__ float all_max(const float* buf) {
  float t = buf[0];
#pragma unroll
  for (int w = 1; w < T / 64; ++w) t = max_of<NAN_MAX>(t, buf[w]);
  return t;
}

// How a row is read.  Short rows go element by element: their few 16-byte
// pieces would leave most threads without a maximum of their own.  Longer ones
// go 16 bytes at a time, 16, 32 or 64 values a thread, since what a thread holds room for
// it also computes, with as few threads as that takes: a row's barriers and searches
// then keep less of the CU waiting.  (12000 bf16 rows, top logits / loss with labels at temperature 1, us: of
// 3500 classes 256 threads 37 / 57, 512 75 / 119; of 6000 51 / 70 and 84 / 116; of 9001 84 / 114 and
// 93 / 137.  Few rows do not gain from more: 256 rows of 32000 logits 11.1 us with 512 threads, 11.6 with
// 1024.)  Packed bf16 pairs go to 128 values in rows of up to PACKED; what no
// registers hold is read by every pass.
// FEW: 256 threads have maxima enough for the threshold, k <= 128 of them (of
// more, the k-th largest would let too many logits pass).
template <typename TI, int PACKED, bool FEW, typename F> static void by_length(int32_t K, F f) {
  constexpr int V = Wide<TI>::n;
#define INT(n) std::integral_constant<int, n>{}
  if constexpr (FEW) {
    if (K <= 8 * 256) return f(INT(256), INT(1), INT(8));
    if (K <= 16 * 256) return f(INT(256), INT(V), INT(16 / V));
    if (K <= 32 * 256) return f(INT(256), INT(V), INT(32 / V));
    if (K <= 64 * 256) return f(INT(256), INT(V), INT(64 / V));
  } else {
    if (K <= 8 * 512) return f(INT(512), INT(1), INT(8));
    if (K <= 32 * 512) return f(INT(512), INT(V), INT(32 / V));
  }
  if (K <= 64 * 512) return f(INT(512), INT(V), INT(64 / V));
  if (K <= 64 * 1024) return f(INT(1024), INT(V), INT(64 / V));
  if constexpr (sizeof(TI) == 2 && PACKED > 64 * 1024)
    if (K <= PACKED) return f(INT(1024), INT(V), INT(128 / V));
  f(INT(1024), INT(V), INT(0));
#undef INT
}
