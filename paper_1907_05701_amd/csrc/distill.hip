// Row operators of distillation: a teacher's top logits, and a student's loss
// and logit gradients against them.  One workgroup per row.
//
// Exponentials are base-2 hardware ones of differences from a row maximum;
// sums are float32 in a fixed order.  Memory bounds both: 2688 bf16 rows of 32000
// logits, the top 32 in 49 us (172 MB, 3.5 TB/s; the vector unit issues 36 us of it,
// and a row's search, candidates and ranks are barriers that only other rows hide), loss and gradients
// with labels in 77 us (344 MB, 4.5 TB/s).
#include <float.h>
#include <math.h>

#include <cmath>
#include <type_traits>

#include "common.hpp"
#include "distill.hpp"

#define LOG2E_F 1.4426950408889634f
#define LN2_F 0.6931471805599453f
static_assert(SOFTMAX_MAX_CLASSES == 1 << 18, "bits of a class");
static constexpr int RT = 256;             // least threads of a row (T below: 256, 512 or 1024)
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
template <int T> struct TopkLds {
  uint32_t tmax[T];
  uint64_t cand[CAND];   // order word, complement of the class; in the order of arrival
  float left[CAND];      // logits of the candidates behind the k-th, in their order
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
template <int LOW, int T>
__device__ __forceinline__ uint32_t kth_max(TopkLds<T>& l, int k) {
  const int lane = threadIdx.x & 63;
  __syncthreads();
  if (threadIdx.x < 64) {
    constexpr int NW = T / 64;
    uint32_t w[NW], t;
#pragma unroll
    for (int i = 0; i < NW; ++i) w[i] = l.tmax[i * 64 + lane];
    if (k <= FOLD) {
      uint32_t g[2] = {w[0], w[1]};
#pragma unroll
      for (int i = 2; i < NW; ++i) g[i & 1] = max(g[i & 1], w[i]);
      t = kth_word<LOW>(g, k);
    } else {
      t = kth_word<LOW>(w, k);
    }
    if (lane == 0) l.thr = t;
  }
  __syncthreads();
  return l.thr;
}
template <int T>
__device__ __forceinline__ void push(TopkLds<T>& l, float v, int c) {
  const uint32_t at = atomicAdd(&l.count, 1u);
  if (at < (uint32_t)CAND) l.cand[at] = ((uint64_t)order_word(v) << 32) | (uint32_t)~c;
}
// Writes the k largest of n candidates, and what is left to l.left (so that sums
// over it do not depend on who arrived first).
template <int T>
__device__ __forceinline__ void rank(TopkLds<T>& l, int n, int64_t m, const TopkP& p) {
  for (int i = threadIdx.x; i < n; i += T) {
    const uint64_t w = l.cand[i];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) r += l.cand[j] > w;
    if (r < p.k) {
      p.top[m * p.k + r] = order_value((uint32_t)(w >> 32));
      p.idx[m * p.k + r] = (int32_t)~(uint32_t)w;
      if (r == p.k - 1) l.kth = w;
    } else {
      l.left[r - p.k] = order_value((uint32_t)(w >> 32));
    }
  }
}

// The log-sum-exp of what orders behind the k-th, from its own maximum, from memory.
template <typename TI, int T, bool ONE>
__device__ __forceinline__ void rest_of(TopkLds<T>& l, const TI* s, int64_t m, const TopkP& p) {
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
template <typename TI, int T, bool ONE>
__device__ __forceinline__ void topk_any(TopkLds<T>& l, const TI* s, int64_t m, const TopkP& p) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K;
  uint32_t mx = 0;
  each<TI, T, ONE>(s, K, [&](int, float v) { mx = max(mx, order_word(v)); });
  __syncthreads();
  l.tmax[tid] = mx;
  if (tid == 0) l.count = 0;
  const uint32_t th = kth_max<0, T>(l, p.k);
  each<TI, T, ONE>(s, K, [&](int c, float v) {
    if (order_word(v) >= th) push(l, v, c);
  });
  __syncthreads();
  int n = (int)min(same(l.count), (uint32_t)CAND);
  if (same(l.count) > (uint32_t)CAND) {
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
  rank(l, n, m, p);
  if (!p.rest) return;
  __syncthreads();
  rest_of<TI, T, ONE>(l, s, m, p);
}

// A longer row than registers hold: read for its threshold, and again for its
// candidates and the sum of the others, which is taken from the threshold as below.
template <typename TI, int T>
__global__ __launch_bounds__(T) void topk_long_kernel(const TI* __restrict__ logits, const TopkP p) {
  __shared__ TopkLds<T> l;
  const int64_t m = blockIdx.x;
  const TI* s = logits + m * p.ld;
  const int tid = threadIdx.x;
  if (tid == 0) {
    l.count = 0;
    l.flag = 0;
  }
  __syncthreads();
  float mx = -INFINITY;
  bool nan = false;
  each<TI, T>(s, p.K, [&](int, float v) {
    mx = fmaxf(mx, v);
    nan |= v != v;
  });
  if (nan) l.flag = 1;
  l.tmax[tid] = order_word(mx);
  const float thr = order_value(max(kth_max<12, T>(l, p.k), LOWEST));
  if (same(l.flag)) {
    topk_any<TI, T, true>(l, s, m, p);
    return;
  }
  const float ref = fabsf(thr) < INFINITY ? thr * p.l2t : 0.f;
  float sum = 0.f;
  each<TI, T>(s, p.K, [&](int c, float v) {
    if (v >= thr) push(l, v, c);
    else sum += exp2_(v * p.l2t - ref);
  });
  __syncthreads();
  const int n = (int)same(l.count);
  if (n > CAND) {
    topk_any<TI, T, true>(l, s, m, p);
    return;
  }
  rank(l, n, m, p);
  if (!p.rest) return;
  __syncthreads();
  for (int i = tid; i < n - p.k; i += T) sum += exp2_(l.left[i] * p.l2t - ref);
  sum = row_sum<T>(sum, l.buf);
  if (same(sum > 1e-20f && sum < 1e30f)) {
    if (tid == 0) p.rest[m] = (ref + log2f(sum)) * LN2_F;
    return;
  }
  rest_of<TI, T, false>(l, s, m, p);
}

// A row in registers, read once.  Candidates leave the registers (-inf in
// their place), so that what stays is of the others; their sum is taken from the threshold,
// which no other exceeds, and again from their own maximum where that leaves
// nothing.  Rows with a NaN, and rows with too many candidates, go the way of any row.
template <typename TI, int T, int V, int NV>
__global__ __launch_bounds__(T, (waves_of<TI, T, V, NV>())) void topk_rows_kernel(const TI* __restrict__ logits, const TopkP p) {
  __shared__ TopkLds<T> l;
  const int64_t m = blockIdx.x;
  const TI* s = logits + m * p.ld;
  const int tid = threadIdx.x;
  Row<TI, V, NV, T> row;
  row.load(s, p.K);
  if (tid == 0) {
    l.count = 0;
    l.flag = 0;
  }
  __syncthreads();
  float vm[NV], mx = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    vm[i] = row.get(i, 0);
#pragma unroll
    for (int j = 1; j < V; ++j) vm[i] = fmaxf(vm[i], row.get(i, j));
    if constexpr (V == 1) nan |= vm[i] != vm[i];
    else {
#pragma unroll
      for (int j = 0; j < V; j += 2) nan |= __builtin_isunordered(row.get(i, j), row.get(i, j + 1));
    }
    mx = fmaxf(mx, vm[i]);
    if constexpr (V > 1) {
      asm volatile("" : "+v"(vm[i]));
      __builtin_amdgcn_sched_barrier(0);   // one vector at a time: fewer registers
    }
  }
  mx = fmaxf(mx, row.tail);
  nan |= row.tail != row.tail;
  if (nan) l.flag = 1;
  l.tmax[tid] = order_word(mx);
  // bf16: the lower 16 bits of all order words are alike; float32: a threshold
  // rounded down to 11 bits lets a few more pass and takes a third fewer steps
  const uint32_t tw = max(kth_max<std::is_same<TI, bf16>::value ? 16 : 12, T>(l, p.k), LOWEST);
  const float thr = order_value(tw);
  row.again();
  if (same(l.flag)) {
    topk_any<TI, T, true>(l, s, m, p);
    return;
  }
  const int whole = row.whole(p.K);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (vm[i] >= thr && row.has(i, whole)) {
      // few vectors come here, most with one value; the others of a vector are
      // read again, so that this is one loop and not a branch per value
      uint32_t bits = 0;
      float v = 0.f;
#pragma unroll
      for (int j = V - 1; j >= 0; --j) {
        const float x = row.get(i, j);
        const bool in = x >= thr;
        bits |= in ? 1u << j : 0u;
        v = in ? x : v;   // ends with the first of them
        if (in) row.drop(i, j);
      }
      push(l, v, row.col(i) + __builtin_ctz(bits));
      bits &= bits - 1;
      for (; bits; bits &= bits - 1) {
        const int c = row.col(i) + __builtin_ctz(bits);
        push(l, to_f32(s[c]), c);
      }
    }
  }
  if (row.tail >= thr && row.tail_col(p.K) < p.K) {
    push(l, row.tail, row.tail_col(p.K));
    row.tail = -INFINITY;
  }
  __syncthreads();
  const int n = (int)same(l.count);
  if (n > CAND) {
    topk_any<TI, T, true>(l, s, m, p);
    return;
  }
  const float ref = fabsf(thr) < INFINITY ? thr * p.l2t : 0.f;
  float sum = 0.f, rm = -INFINITY;
  rank(l, n, m, p);
  if (!p.rest) return;
  __syncthreads();
  for (int i = tid; i < n - p.k; i += T) {
    sum += exp2_(l.left[i] * p.l2t - ref);
    rm = fmaxf(rm, l.left[i]);
  }
  row.again();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < V; ++j) sum += exp2_(row.get(i, j) * p.l2t - ref);
    if constexpr (V > 1) __builtin_amdgcn_sched_barrier(0);   // one vector at a time: fewer registers
  }
  sum += exp2_(row.tail * p.l2t - ref);
  sum = row_sum<T>(sum, l.buf);
  if (same(sum > 1e-20f && sum < 1e30f)) {
    if (tid == 0) p.rest[m] = (ref + log2f(sum)) * LN2_F;
    return;
  }
  // far below the threshold, or infinite
  row.again();
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) rm = fmaxf(rm, row.get(i, j));
  rm = row_max<T>(fmaxf(rm, row.tail), l.buf);
  sum = 0.f;
  if (fabsf(rm) < INFINITY) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) sum += exp2_((row.get(i, j) - rm) * p.l2t);
    sum += exp2_((row.tail - rm) * p.l2t);
    for (int i = tid; i < n - p.k; i += T) sum += exp2_((l.left[i] - rm) * p.l2t);
  }
  sum = row_sum<T>(sum, l.buf);
  if (tid == 0) p.rest[m] = fabsf(rm) < INFINITY ? rm * (p.l2t * LN2_F) + log2f(sum) * LN2_F : rm;
}

// ---------------------------------------------------------------------------
// Loss and gradient.  With u = s / tau, the listed classes' probabilities p
// (equal classes' added up), the others' r, and Z, Zr the sums of e^u over all
// and over the others:
//   KL = sum p (log p - log q) + r (log r - log(Zr / Z)),  q = e^u / Z
//   d(tau^2 KL)/ds = tau (q - p) where listed, tau e^u (1/Z - r/Zr) elsewhere
// The others' sum has a maximum of its own, so that it does not vanish
// beside listed logits however large they are.  Every exponent is a difference of logits,
// scaled: a mask of -1e9 or of the type's lowest value times log2 e / tau would overflow, or
// carry a rounding of its own size into the exponential.  What differences cost (KL = sum p
// (log p + log z - (s - max) / tau)) stays unscaled up to the loss for the same reason.
// ---------------------------------------------------------------------------
struct DistillP {
  int64_t ld, ldd;
  const float *top, *rest, *weights;
  const int32_t *idx, *labels;
  float* row_loss;
  int K, k, pad;
  float it2, tau, soft, hard, scale;   // it2: log2 e / tau
};
// Threads of a row of 32000: 512.  (2688 rows without labels, us: bf16 73, with 256 threads 108, with 1024
// 125; float32 136, 426 and 155.  256 threads spill their 128 values; 1024 leave a CU one row or two.)
template <int T> struct DistillLds {
  float pv[MAXK];
  int32_t iv[MAXK];
  float buf[8][T / 64];
  uint32_t dup;
};

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

// A row's other classes (those that are not listed): in registers, or, NV = 0, read
// from memory by each pass.  others(f) calls f(value) for each, the listed
// ones and what lies behind K as -inf; write(f) stores f(value) in their place.
template <typename TI, typename TO, int T, int V, int NV> struct Others {
  Row<TI, V, NV, T> row;
  __device__ __forceinline__ void load(const TI* s, int K) { row.load(s, K); }
  __device__ __forceinline__ void mask(const uint32_t* listed, int K) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = row.col(i);
      // V columns never straddle a word
      const uint32_t bits = (listed[c >> 5] >> (c & 31)) & ((1u << V) - 1);
      if (bits) {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if ((bits >> j) & 1u) row.drop(i, j);
      }
    }
    const int c = row.tail_col(K);
    if (c < K && ((listed[c >> 5] >> (c & 31)) & 1u)) row.tail = -INFINITY;
  }
  template <typename F> __device__ __forceinline__ void others(const TI*, int, const uint32_t*, F f) {
    row.again();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < V; ++j) f(row.get(i, j));
      if constexpr (V > 1) __builtin_amdgcn_sched_barrier(0);   // one vector at a time: fewer registers
    }
    if constexpr (V > 1) f(row.tail);
  }
  template <typename F> __device__ __forceinline__ void write(const TI*, TO* d, int K, const uint32_t*, F f) {
    row.again();
    const int n = row.whole(K);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      TO o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = from_f32<TO>(f(row.get(i, j)));
      if (row.has(i, n)) __builtin_memcpy(row.at(d, i), o, V * sizeof(TO));
      if constexpr (V > 1) __builtin_amdgcn_sched_barrier(0);
    }
    if (row.tail_col(K) < K) d[row.tail_col(K)] = from_f32<TO>(f(row.tail));
  }
};
template <typename TI, typename TO, int T, int V> struct Others<TI, TO, T, V, 0> {
  __device__ __forceinline__ void load(const TI*, int) {}
  __device__ __forceinline__ void mask(const uint32_t*, int) {}
  static __device__ __forceinline__ float of(const uint32_t* listed, int c, float v) {
    return ((listed[c >> 5] >> (c & 31)) & 1u) ? -INFINITY : v;
  }
  template <typename F> __device__ __forceinline__ void others(const TI* s, int K, const uint32_t* listed, F f) const {
    each<TI, T>(s, K, [&](int c, float v) { f(of(listed, c, v)); });
  }
  template <typename F>
  __device__ __forceinline__ void write(const TI* s, TO* d, int K, const uint32_t* listed, F f) const {
    // a thread writes only where it has read (d may be s)
    const int done = K / V * V;
    for (int c = (int)threadIdx.x * V; c < done; c += T * V) {
      TI v[V];
      TO o[V];
      __builtin_memcpy(v, s + c, V * sizeof(TI));
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = from_f32<TO>(f(of(listed, c + j, to_f32(v[j]))));
      __builtin_memcpy(d + c, o, V * sizeof(TO));
    }
    const int c = done + (int)threadIdx.x;
    if (c < K) d[c] = from_f32<TO>(f(of(listed, c, to_f32(s[c]))));
  }
};

// HARD: how the labels' cross-entropy has e^s of the others, NO: no labels, OWN: an
// exponential of its own, POW1, POW2: from e^u, its first or second power.
// (Temperatures of 1 and 2.  2688 bf16 rows of 32000: NO 72, POW1 77, POW2 78, OWN 90 us: half the
// exponentials of OWN, which the vector unit shares with the rounding and the moves.)
enum { NO, OWN, POW1, POW2 };
template <typename TI, typename TO, int T, int V, int NV, int HARD>
__global__ __launch_bounds__(T, (waves_of<TI, T, V, NV>())) void distill_rows_kernel(const TI* logits, TO* dlogits, const DistillP p) {
  extern __shared__ uint32_t listed[];   // a bit per class, to the end of the registers' columns
  __shared__ DistillLds<T> l;
  const int64_t m = blockIdx.x;
  const TI* s = logits + m * p.ld;
  TO* d = dlogits + m * p.ldd;
  const int tid = threadIdx.x, K = p.K;
  const float weight = p.weights ? p.weights[m] : 1.f;
  for (int c = K + tid; c < K + p.pad; c += T) d[c] = from_f32<TO>(0.f);
  auto nothing = [&]() {   // a row that has no loss
    for (int c = tid; c < K; c += T) d[c] = from_f32<TO>(0.f);
    if (tid == 0) p.row_loss[m] = 0.f;
  };
  if (weight == 0.f) return nothing();
  Others<TI, TO, T, V, NV> row;
  row.load(s, K);   // in flight while the teacher's part runs
  const int words = (NV ? NV * V * T : K + 31) / 32;
  for (int i = tid; i < words; i += T) listed[i] = 0;
  if (tid == 0) l.dup = 0;
  int at = -1;
  float tv = -INFINITY, sv = -INFINITY;   // the entry's teacher logit, student logit
  if (tid < p.k) {
    at = p.idx[m * p.k + tid];
    if (at < 0 || at >= K) at = -1;
    else {
      tv = p.top[m * p.k + tid];
      sv = to_f32(s[at]);
    }
    l.iv[tid] = at;
  }
  const float rest = p.rest ? p.rest[m] : -INFINITY;   // log of the rest: a logit over tau
  const int lab = HARD ? p.labels[m] : -1;
  const bool marked = HARD && lab >= 0 && lab < K;
  const float sl = marked ? to_f32(s[lab]) : 0.f;
  __syncthreads();
  if (at >= 0 && (atomicOr(&listed[at >> 5], 1u << (at & 31)) & (1u << (at & 31)))) l.dup = 1;
  put_wave(l.buf[0], wave_max<true>(tv));
  put_wave(l.buf[1], wave_max(sv));
  __syncthreads();
  // the teacher's probabilities; lt: log2 of the entry's, lr: of the rest's, but for the sum
  const float tmax = all_max<T, true>(l.buf[0]), lm = all_max<T>(l.buf[1]);
  const float tbase = tmax == -INFINITY ? 0.f : tmax;   // of the listed ones; over tau, as far as float32 goes:
  const float ta = fabsf(tmax) < INFINITY ? fminf(fmaxf(tmax / p.tau, -FLT_MAX), FLT_MAX) : tmax;
  const float tm = max_nan(ta, rest);
  // an unwanted loss may be infinite; a teacher's NaN or +inf makes tz, every probability and r a NaN
  const bool taught = p.soft != 0.f && !(tm == -INFINITY);
  if (same(!taught && !marked)) return nothing();   // whatever it holds: below, 0 times its z would count
  const float lt = (tv - tbase) * p.it2 + (ta - tm) * LOG2E_F, lr = (rest - tm) * LOG2E_F;
  const float e = taught ? exp2_(lt) : 0.f, er = taught ? exp2_(lr) : 0.f;
  if (tid < p.k) l.pv[tid] = e;
  put_wave(l.buf[2], wave_sum(e));
  row.mask(listed, K);
  float rm = -INFINITY;
  row.others(s, K, listed, [&](float v) { rm = fmaxf(rm, v); });
  put_wave(l.buf[3], wave_max(rm));
  __syncthreads();
  const float tz = all_sum<T>(l.buf[2]) + er, l2tz = taught ? log2f(tz) : 0.f;
  const float prob = taught ? e / tz : 0.f, r = taught ? er / tz : 0.f;
  float lp = lt - l2tz;     // log2 of the entry's probability
  float own = prob;         // of its class
  bool lead = at >= 0;      // the class's first entry
  if (l.dup && at >= 0) {   // (the sums below are zeros where the row is not taught)
    own = 0.f;
    for (int j = 0; j < p.k; ++j)
      if (l.iv[j] == at) {
        own += l.pv[j];
        if (j < tid) lead = false;
      }
    own = taught ? own / tz : 0.f;
    lp = log2f(own);
  }
  // maxima: the others', the row's; from where their exponents count
  rm = all_max<T>(l.buf[3]);
  const float am = fmaxf(rm, lm), aref = am == -INFINITY ? 0.f : am, rref = rm == -INFINITY ? 0.f : rm;
  const float eo = exp2_((rm - aref) * p.it2);   // the others' sums, from the row's maximum
  float zr = 0.f, z1 = 0.f;
  row.others(s, K, listed, [&](float v) {
    const float y = v - rref, x = exp2_(y * p.it2);
    zr += x;
    if constexpr (HARD == OWN) z1 += exp2_(y * LOG2E_F);
    if constexpr (HARD == POW2) z1 += x * x;
    // or the compiler would sink this sum past the loop, and carry every exponential there
    if constexpr (HARD == OWN || HARD == POW2) asm volatile("" : "+v"(z1));
  });
  const float eh = HARD ? exp2_((rm - aref) * LOG2E_F) : 0.f;   // as eo, of e^s
  z1 = (HARD == POW1 ? zr : z1) * eh;
  const float ez = lead ? exp2_((sv - aref) * p.it2) : 0.f;
  if (HARD && lead) z1 += exp2_((sv - aref) * LOG2E_F);
  put_wave(l.buf[4], wave_sum(zr));
  put_wave(l.buf[5], wave_sum(ez));
  if constexpr (HARD) put_wave(l.buf[6], wave_sum(z1));
  __syncthreads();   // every listed logit and the label's have been read, too
  zr = all_sum<T>(l.buf[4]);
  const float z = all_sum<T>(l.buf[5]) + zr * eo;
  if constexpr (HARD) z1 = all_sum<T>(l.buf[6]);
  const float l2z = log2f(z);
  const float tln = p.tau * LN2_F;
  put_wave(l.buf[7], wave_sum(at >= 0 && prob != 0.f ? prob * ((lp + l2z) * tln + (aref - sv)) : 0.f));   // tau KL
  const float ks = taught ? p.scale * weight * p.soft * p.tau : 0.f, kh = marked ? p.scale * weight * p.hard : 0.f;
  const float cr = ks * (eo / z - (r == 0.f || (r > 0.f && zr == 0.f) ? 0.f : r / zr));   // of x in the others
  const float ch = marked ? kh / z1 : 0.f;
  const float cp = HARD == POW1 ? cr + ch * eh : ch * eh;   // of x at POW1, of the exponential of its own or x^2
  row.write(s, d, K, listed, [&](float v) {
    const float y = v - rref, x = exp2_(y * p.it2);
    if constexpr (HARD == OWN) return cr * x + cp * exp2_(y * LOG2E_F);
    else if constexpr (HARD == POW1) return cp * x;
    else if constexpr (HARD == POW2) return (cr + cp * x) * x;
    else return cr * x;
  });
  __syncthreads();   // the others lie before what replaces the listed ones' and the label's values
  if (lead) {
    float g = ks * (ez / z - own);
    if constexpr (HARD) {
      g += ch * exp2_((sv - aref) * LOG2E_F);
      if (at == lab) g -= kh;
    }
    d[at] = from_f32<TO>(g);
  }
  if (tid != 0) return;
  if (marked && !((listed[lab >> 5] >> (lab & 31)) & 1u))
    d[lab] = from_f32<TO>(cr * exp2_((sl - rref) * p.it2) + ch * exp2_((sl - aref) * LOG2E_F) - kh);
  float loss = 0.f;
  if (taught) {
    float kl = all_sum<T>(l.buf[7]);
    if (r != 0.f) kl += r * ((lr - l2tz - log2f(zr) + l2z) * tln + (aref - rm));
    loss = p.soft * p.tau * kl;
  }
  if (marked) loss += p.hard * ((aref - sl) + log2f(z1) * LN2_F);
  p.row_loss[m] = weight * loss;
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
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

template <typename TI>
int topk_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, int32_t k, float temperature, float* top,
              int32_t* idx, float* rest, hipStream_t stream) {
  const TopkP p{ld, K, k, LOG2E_F / temperature, top, rest, idx};
  auto launch = [&](auto t, auto v, auto nv) {
    constexpr int T = decltype(t)::value, V = decltype(v)::value, NV = decltype(nv)::value;
    if constexpr (NV > 0)
      BLSTM_LAUNCH("softmax_topk_rows", (topk_rows_kernel<TI, T, V, NV>), dim3((unsigned)M), dim3(T), 0, stream, logits, p);
    else
      BLSTM_LAUNCH("softmax_topk_rows", (topk_long_kernel<TI, T>), dim3((unsigned)M), dim3(T), 0, stream, logits, p);
  };
  if (k <= 128) by_length<TI, 0, true>(K, launch);
  else by_length<TI, 0, false>(K, launch);
  return blstm_check_launch("softmax_topk_rows");
}
template int topk_rows<float>(const float*, int64_t, int64_t, int32_t, int32_t, float, float*, int32_t*, float*, hipStream_t);
template int topk_rows<bf16>(const bf16*, int64_t, int64_t, int32_t, int32_t, float, float*, int32_t*, float*, hipStream_t);

template <typename TI, typename TO>
int distill_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, const softmax_teacher* t, float loss_scale,
                 float* row_loss, TO* dlogits, int64_t ldd, int32_t pad, hipStream_t stream) {
  DistillP p{};
  p.ld = ld; p.ldd = ldd; p.top = t->top; p.rest = t->rest; p.weights = t->weights; p.idx = t->idx;
  p.labels = t->hard != 0.f ? t->labels : nullptr;
  p.row_loss = row_loss; p.K = K; p.k = t->k; p.pad = pad;
  p.it2 = LOG2E_F / t->temperature; p.tau = t->temperature; p.soft = t->soft; p.hard = t->hard; p.scale = loss_scale;
  by_length<TI, 128 * 1024, true>(K, [&](auto tt, auto v, auto nv) {
    constexpr int T = decltype(tt)::value, V = decltype(v)::value, NV = decltype(nv)::value;
    const size_t bits = (size_t)(NV ? NV * V * T : rup(K, 32)) / 8;
#define DISTILL(HARD)                                                                                                  \
  BLSTM_LAUNCH("softmax_distill_rows", (distill_rows_kernel<TI, TO, T, V, NV, HARD>), dim3((unsigned)M), dim3(T), bits, \
               stream, logits, dlogits, p)
    if (!p.labels) DISTILL(NO);
    else if (p.tau == 1.f) DISTILL(POW1);
    else if (p.tau == 2.f) DISTILL(POW2);
    else DISTILL(OWN);
  });
  return blstm_check_launch("softmax_distill_rows");
}
template int distill_rows<float, float>(const float*, int64_t, int64_t, int32_t, const softmax_teacher*, float, float*, float*, int64_t, int32_t, hipStream_t);
template int distill_rows<float, bf16>(const float*, int64_t, int64_t, int32_t, const softmax_teacher*, float, float*, bf16*, int64_t, int32_t, hipStream_t);
template int distill_rows<bf16, bf16>(const bf16*, int64_t, int64_t, int32_t, const softmax_teacher*, float, float*, bf16*, int64_t, int32_t, hipStream_t);

static int check_rows(const char* fn, const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision) {
  if (M < 1 || K < 1) return blstm_fail(BLSTM_EINVAL, "%s: M and K must be positive (M=%lld K=%d)", fn, (long long)M, K);
  if (!logits) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (precision != BLSTM_FP32 && precision != BLSTM_BF16)
    return blstm_fail(BLSTM_EINVAL, "%s: precision must be BLSTM_FP32 or BLSTM_BF16", fn);
  if (ld < K) return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  if (M * 1024 > LAUNCH_THREADS) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: too many rows", fn);
  return BLSTM_OK;
}
static int check_k(int32_t k, int32_t K, float temperature, const char* fn) {
  if (K > SOFTMAX_MAX_CLASSES) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: K > %d", fn, SOFTMAX_MAX_CLASSES);
  if (k < 1) return blstm_fail(BLSTM_EINVAL, "%s: k must be positive", fn);
  if (k > MAXK) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: k > %d", fn, MAXK);
  if (!(temperature > 0.f) || !std::isnormal(temperature))
    return blstm_fail(BLSTM_EINVAL, "%s: the temperature must be positive and finite", fn);
  return BLSTM_OK;
}
int check_top(int32_t k, int32_t K, float temperature, const char* fn) {
  const int rc = check_k(k, K, temperature, fn);
  if (rc) return rc;
  return k > K ? blstm_fail(BLSTM_EINVAL, "%s: k=%d above K=%d", fn, k, K) : BLSTM_OK;
}
int check_teacher(const softmax_teacher* t, int32_t K, const char* fn) {
  if (!t || !t->top || !t->idx) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (!std::isfinite(t->soft) || !std::isfinite(t->hard)) return blstm_fail(BLSTM_EINVAL, "%s: soft and hard must be finite", fn);
  return check_k(t->k, K, t->temperature, fn);
}

extern "C" int softmax_topk_rows(const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision, int32_t k,
                                 float temperature, float* top, int32_t* idx, float* rest, hipStream_t stream) {
  int rc = check_rows("softmax_topk_rows", logits, ld, M, K, precision);
  if (!rc) rc = check_top(k, K, temperature, "softmax_topk_rows");
  if (rc) return rc;
  if (!top || !idx) return blstm_fail(BLSTM_EINVAL, "softmax_topk_rows: NULL pointer");
  return precision == BLSTM_BF16 ? topk_rows((const bf16*)logits, ld, M, K, k, temperature, top, idx, rest, stream)
                                 : topk_rows((const float*)logits, ld, M, K, k, temperature, top, idx, rest, stream);
}

extern "C" int softmax_distill_rows(const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision,
                                    const softmax_teacher* teacher, float loss_scale, float* row_loss, void* dlogits,
                                    int64_t ldd, hipStream_t stream) {
  int rc = check_rows("softmax_distill_rows", logits, ld, M, K, precision);
  if (!rc) rc = check_teacher(teacher, K, "softmax_distill_rows");
  if (rc) return rc;
  if (!row_loss || !dlogits) return blstm_fail(BLSTM_EINVAL, "softmax_distill_rows: NULL pointer");
  if (ldd < K) return blstm_fail(BLSTM_EINVAL, "softmax_distill_rows: a row pitch is below its row");
  if (dlogits == logits && ldd != ld)
    return blstm_fail(BLSTM_EINVAL, "softmax_distill_rows: dlogits over logits with another row pitch");
  if (precision == BLSTM_BF16)
    return distill_rows((const bf16*)logits, ld, M, K, teacher, loss_scale, row_loss, (bf16*)dlogits, ldd, 0, stream);
  return distill_rows((const float*)logits, ld, M, K, teacher, loss_scale, row_loss, (float*)dlogits, ldd, 0, stream);
}
