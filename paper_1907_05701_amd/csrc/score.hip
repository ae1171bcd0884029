// Row operators of scoring: log probabilities of given classes, the entropy and
// the most likely classes of rows of logits, and the gradient of the logits.
//
// With y_j = (s_j - max s) log2 e / tau, Z = sum 2^y and T = sum 2^y y:
//   log p_j = (s_j - max s) / tau - ln Z,   H = ln Z - ln 2 T / Z
// Exponents are scaled differences of logits, so that a mask of -1e9 or of the
// type's lowest value is a value like any other.  Sums are float32 in a fixed order.
//
// Memory bounds both: a row is read once, into registers.  2688 bf16 rows of 32000 logits with one listed class, the
// entropy and 8 most likely classes in 39.8 us (172 MB, 4.3 TB/s; the vector unit issues 31 us of it), the gradient in
// 70 us (344 MB, 4.9 TB/s).
#include <cmath>

#include "rows.hpp"
#include "score.hpp"

struct ScoreP {
  int64_t ld;
  int K, n, k;
  float it2, itau;   // log2 e / tau, 1 / tau
  const int32_t* ids;
  float *logprob, *entropy, *top;
  int32_t* idx;
};

// Below this exponent 2^y is 0 in float32: y stops here in products with it, so that a class at -inf adds 0 to T.
static constexpr float Y_MIN = -200.f;

// A row's statistics, its sums from `ref`, the largest logit (0 where there is none above -inf).
// A NaN in the row, or a difference of infinities, makes z a NaN.
struct RowStats {
  float ref, it2, z = 0.f, t = 0.f;
  bool some;   // a class above -inf, or a NaN
  __device__ __forceinline__ RowStats(float largest, float it2_)
      : ref(largest == -INFINITY ? 0.f : largest), it2(it2_), some(!(largest == -INFINITY)) {}
  __device__ __forceinline__ float y_of(float v) const { return (v - ref) * it2; }
  __device__ __forceinline__ void add(float v) {
    const float y = y_of(v), e = exp2_(y);
    z += e;
    t += e * fmaxf(y, Y_MIN);
  }
  // or the compiler would sink the sums past the loop over vectors, and carry every exponential there
  __device__ __forceinline__ void keep() { asm volatile("" : "+v"(z), "+v"(t)); }
  __device__ __forceinline__ bool good() const { return z == z; }
};
// A logit's log probability; every class of a row with none above -inf has log probability -inf,
// every one of a row with a NaN or +inf NaN.
struct LogProb {
  float ref, itau, lz;
  bool some;
  __device__ __forceinline__ LogProb(const RowStats& r, float itau_)
      : ref(r.ref), itau(itau_), lz(log2f(r.z) * LN2_F), some(r.some || !r.good()) {}
  __device__ __forceinline__ float operator()(float v) const { return some ? (v - ref) * itau - lz : -INFINITY; }
};

// The largest of a thread's logits, and (vm) of each vector of them; a NaN counts as none.
template <typename TI, int V, int NV, int T>
__device__ __forceinline__ float largest(const Row<TI, V, NV, T>& row, float (&vm)[NV]) {
  float mx = row.tail;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    vm[i] = row.get(i, 0);
#pragma unroll
    for (int j = 1; j < V; ++j) vm[i] = fmaxf(vm[i], row.get(i, j));
    mx = fmaxf(mx, vm[i]);
    if constexpr (V > 1) {
      asm volatile("" : "+v"(vm[i]));
      __builtin_amdgcn_sched_barrier(0);   // one vector at a time: fewer registers
    }
  }
  return mx;
}
template <typename TI, int V, int NV, int T>
__device__ __forceinline__ void add_row(RowStats& r, Row<TI, V, NV, T>& row) {
  row.again();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < V; ++j) r.add(row.get(i, j));
    r.keep();
    if constexpr (V > 1) __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (V > 1) r.add(row.tail);
}

// The most likely classes of a row whose candidates are too many, or that has a NaN or +inf, read again: all above the
// k-th largest of the threads' maxima, and of those that equal it the first, which are found soon where they are many.
// (175 bf16 rows of 32000 classes, one all at -inf: 22 us, 239 with a search bit by bit for the last of them.)
template <typename TI, int T, int C, typename F>
__device__ __forceinline__ void most_likely(TopkLds<T, C>& l, const TI* s, int64_t m, const TopkP& p, F value) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K;
  uint32_t mx = 0;
  each<TI, T>(s, K, [&](int, float v) { mx = max(mx, order_word(v)); });
  __syncthreads();
  l.tmax[tid] = mx;
  if (tid == 0) l.count = 0;
  const uint32_t t = kth_max<0>(l, p.k);
  each<TI, T>(s, K, [&](int c, float v) {
    if (order_word(v) > t) push(l, v, c);
  });
  __syncthreads();
  int taken = (int)same(l.count);
  if (taken > C) {
    topk_any<TI, T, true>(l, s, m, p, value);
    return;
  }
  const int n = max(taken, p.k);
  __syncthreads();
  for (int c0 = 0, par = 0; taken < p.k && c0 < K; c0 += T, par ^= 1) {
    const int c = c0 + tid;
    const float v = c < K ? to_f32(s[c]) : 0.f;
    const bool tie = c < K && order_word(v) == t;
    const uint64_t ties = __ballot(tie);
    if (lane == 0) l.cnt[par][wave] = __popcll(ties);
    __syncthreads();
    int before = taken + __popcll(ties & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < T / 64; ++w) {
      const int there = (int)l.cnt[par][w];
      before += w < wave ? there : 0;
      taken += there;
    }
    if (tie && before < p.k) push(l, v, c);
  }
  __syncthreads();
  rank(l, n, m, p, value);
}

template <typename TI, int T, int V, int NV, bool TOP>
__global__ __launch_bounds__(T, (waves_of<TI, T, V, NV>())) void score_rows_kernel(
    const TI* __restrict__ logits, const ScoreP p) {
  constexpr int C = T == 64 ? 256 : CAND;   // (a one-wave workgroup's share of the LDS)
  __shared__ TopkLds<TOP ? T : 64, TOP ? C : 64> l;
  __shared__ float buf[3][T / 64];
  const int64_t m = blockIdx.x;
  const TI* s = logits + m * p.ld;
  const int tid = threadIdx.x, K = p.K;
  Row<TI, V, NV ? NV : 1, T> row;
  if constexpr (NV > 0) row.load(s, K);   // in flight while the list is read
  if (TOP && tid == 0) l.count = 0;
  int at = -1;
  float sv = 0.f;
  if (tid < p.n) {
    at = p.ids[m * p.n + tid];
    if (at < 0 || at >= K) at = -1;
    else sv = to_f32(s[at]);
  }
  float vm[NV ? NV : 1], mx = -INFINITY;
  if constexpr (NV > 0) mx = largest(row, vm);
  else each<TI, T>(s, K, [&](int, float v) { mx = fmaxf(mx, v); });
  mx = fmaxf(mx, -INFINITY);   // of NaN alone: none
  put_wave(buf[0], wave_max(mx));
  float thr = INFINITY;
  if constexpr (TOP) {
    l.tmax[tid] = order_word(mx);
    // bf16: the lower 16 bits of all order words are alike; float32: a threshold
    // rounded down to 11 bits lets a few more pass and takes a third fewer steps
    thr = order_value(max(kth_max<std::is_same<TI, bf16>::value ? 16 : 12>(l, p.k), LOWEST));
  } else {
    __syncthreads();
  }
  RowStats r(all_max<T>(buf[0]), p.it2);
  if constexpr (NV > 0) {
    add_row(r, row);
    if constexpr (TOP) {
      row.again();
      const int whole = row.whole(K);
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
            bits |= x >= thr ? 1u << j : 0u;
            v = x >= thr ? x : v;   // ends with the first of them
          }
          push(l, v, row.col(i) + __builtin_ctz(bits));
          bits &= bits - 1;
          for (; bits; bits &= bits - 1) {
            const int c = row.col(i) + __builtin_ctz(bits);
            push(l, to_f32(s[c]), c);
          }
        }
      }
      if (row.tail >= thr && row.tail_col(K) < K) push(l, row.tail, row.tail_col(K));
    }
  } else {
    each<TI, T>(s, K, [&](int c, float v) {
      r.add(v);
      if constexpr (TOP)
        if (v >= thr) push(l, v, c);
    });
  }
  put_wave(buf[1], wave_sum(r.z));
  put_wave(buf[2], wave_sum(r.t));
  __syncthreads();
  r.z = all_sum<T>(buf[1]);
  r.t = all_sum<T>(buf[2]);
  const LogProb lp(r, p.itau);
  if (tid < p.n) p.logprob[m * p.n + tid] = at < 0 ? 0.f : lp(sv);
  if (p.entropy && tid == 0) p.entropy[m] = lp.some ? lp.lz - r.t / r.z * LN2_F : 0.f;
  if constexpr (TOP) {
    TopkP tp{p.ld, K, p.k, p.it2, p.top, nullptr, p.idx};
    const int n = (int)same(l.count);
    if (same(!r.good()) || n > C) most_likely<TI, T>(l, s, m, tp, lp);
    else rank(l, n, m, tp, lp);
  }
}

// ---------------------------------------------------------------------------
// The gradient.  With g_i of the log probability of class id_i and h of the
// entropy, G = sum g:
//   dL/ds_j = (sum_{id_i = j} g_i - p_j (G + h (log p_j + H))) / tau
//           = 2^y_j (A + B y_j) + (sum_{id_i = j} g_i) / tau
// Rows of zeros g and h have a gradient of zeros whatever they hold, and so has
// a row with no class above -inf; one with a NaN or +inf has NaN.
// ---------------------------------------------------------------------------
struct ScoreGradP {
  int64_t ld, ldd;
  int K, n, pad;
  float it2, itau;   // log2 e / tau, 1 / tau
  const int32_t* ids;
  const float *dlogprob, *dentropy;
};

// A row's list: all that is given to a class, for the class's first entry to write.  64 entries a wave; the ballots of each
// bit of their classes say which of them a class equals, so that n entries take n / 64 steps a bit and not n.  (us, so / by
// comparing each with each: 768 float32 rows of 9001 classes with 256 listed 16.3 / 51, 5000 of 700 with 64 8.9 / 24,
// 2688 bf16 rows of 32000 with 256 75 / 154.)
struct Listed {
  bool first;
  float sum;   // in the list's order
};
template <int N> struct ListLds {
  static constexpr int BITS = 18;
  float g[N];
  uint64_t bit[N / 64][BITS], some[N / 64];
  static __device__ __forceinline__ int bits(int K) { return 32 - __builtin_clz(K); }   // of every class, and of K
  __device__ __forceinline__ void put(int at, float v, int n, int K) {
    const int w = threadIdx.x >> 6;
    if (n < 2 || w * 64 >= n) return;
    g[threadIdx.x] = v;
    const uint64_t there = __ballot(at >= 0);
    if ((threadIdx.x & 63) == 0) some[w] = there;
    const int nb = min(bits(K), BITS);
    for (int b = 0; b < nb; ++b) {
      const uint64_t set = __ballot(at >> b & 1);
      if ((threadIdx.x & 63) == 0) bit[w][b] = set;
    }
  }
  // behind a barrier
  __device__ __forceinline__ Listed all_of(int at, float v, int n, int K) const {
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    Listed o{at >= 0, v};
    if (n < 2 || w * 64 >= n) return o;
    o.sum = 0.f;
    const int nb = min(bits(K), BITS);
    for (int c = 0; c * 64 < n; ++c) {
      uint64_t alike = some[c];
#pragma unroll 4
      for (int b = 0; b < nb; ++b) alike &= bit[c][b] ^ (uint64_t)((int64_t)(at >> b & 1) - 1);
      const uint64_t before = c < w ? ~0ull : c == w ? (1ull << lane) - 1 : 0;
      o.first &= !(alike & before);
      for (; alike; alike &= alike - 1) o.sum += g[c * 64 + __builtin_ctzll(alike)];
    }
    return o;
  }
};

template <typename TI, typename TO, int T, int V, int NV>
__global__ __launch_bounds__(T, (waves_of<TI, T, V, NV>())) void score_grad_kernel(const TI* logits, TO* dlogits, const ScoreGradP p) {
  __shared__ ListLds<T == 64 ? 64 : MAXK> list;
  __shared__ float buf[4][T / 64];
  __shared__ uint32_t wanted;
  const int64_t m = blockIdx.x;
  const TI* s = logits + m * p.ld;
  TO* d = dlogits + m * p.ldd;
  const int tid = threadIdx.x, K = p.K;
  Row<TI, V, NV ? NV : 1, T> row;
  if constexpr (NV > 0) row.load(s, K);
  if (tid == 0) wanted = 0;
  int at = -1;
  float sv = 0.f, g = 0.f;
  if (tid < p.n) {
    at = p.ids[m * p.n + tid];
    if (at < 0 || at >= K) at = -1;
    else {
      sv = to_f32(s[at]);
      g = p.dlogprob[m * p.n + tid];
    }
  }
  list.put(at, g, p.n, K);
  const float h = p.dentropy ? p.dentropy[m] : 0.f;
  for (int c = K + tid; c < K + p.pad; c += T) d[c] = from_f32<TO>(0.f);
  __syncthreads();
  const Listed own = list.all_of(at, g, p.n, K);   // (the row is still on its way)
  float vm[NV ? NV : 1], mx = -INFINITY;
  if constexpr (NV > 0) mx = largest(row, vm);
  else each<TI, T>(s, K, [&](int, float v) { mx = fmaxf(mx, v); });
  if (!(g == 0.f)) wanted = 1;
  put_wave(buf[0], wave_max(fmaxf(mx, -INFINITY)));
  put_wave(buf[1], wave_sum(g));
  __syncthreads();
  RowStats r(all_max<T>(buf[0]), p.it2);
  auto nothing = [&]() {
    for (int c = tid; c < K; c += T) d[c] = from_f32<TO>(0.f);
  };
  if (same(!wanted && h == 0.f)) return nothing();
  const float sum_g = all_sum<T>(buf[1]);
  if constexpr (NV > 0) add_row(r, row);
  else each<TI, T>(s, K, [&](int, float v) { r.add(v); });
  put_wave(buf[2], wave_sum(r.z));
  put_wave(buf[3], wave_sum(r.t));
  __syncthreads();   // every listed logit has been read, too
  r.z = all_sum<T>(buf[2]);
  if (same(!r.some && r.good())) return nothing();
  // log p_j + H = ln 2 (y_j - T / Z)
  const float mean = all_sum<T>(buf[3]) / r.z, per = p.itau / r.z;
  const float A = -per * (sum_g - h * LN2_F * mean), B = -per * h * LN2_F;
  auto grad = [&](float v) {
    const float y = r.y_of(v);
    return exp2_(y) * fmaf(B, fmaxf(y, Y_MIN), A);
  };
  if constexpr (NV > 0) {
    row.again();
    const int whole = row.whole(K);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      TO o[V];
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = from_f32<TO>(grad(row.get(i, j)));
      if (row.has(i, whole)) __builtin_memcpy(row.at(d, i), o, V * sizeof(TO));
      if constexpr (V > 1) __builtin_amdgcn_sched_barrier(0);
    }
    if (row.tail_col(K) < K) d[row.tail_col(K)] = from_f32<TO>(grad(row.tail));
  } else {
    // a thread writes only where it has read (d may be s)
    const int done = K / V * V;
    for (int c = tid * V; c < done; c += T * V) {
      TI v[V];
      TO o[V];
      __builtin_memcpy(v, s + c, V * sizeof(TI));
#pragma unroll
      for (int j = 0; j < V; ++j) o[j] = from_f32<TO>(grad(to_f32(v[j])));
      __builtin_memcpy(d + c, o, V * sizeof(TO));
    }
    const int c = done + tid;
    if (c < K) d[c] = from_f32<TO>(grad(to_f32(s[c])));
  }
  __syncthreads();   // the dense part lies before what replaces the listed classes' values
  if (own.first) d[at] = from_f32<TO>(grad(sv) + own.sum * p.itau);
}

// Short rows, four to a workgroup, a wave each without barriers; a class's list entries are added where the class lies in
// registers, one after the other.  (us, so / by a workgroup of one wave each: 20000 bf16 rows of 100 classes with 4 listed
// 8.4 / 16.6, with 16 11.7 / 16.8, with 64 26.8 / 17.3; 20000 of 500 with 4 19.0 / 20.0, with 8 20.3 / 19.4, with 12
// 22.9 / 19.6; 5000 of 1000 with one 8.7 / 7.3.)
static constexpr int WAVE_K = 512, WAVE_LIST = 64;   // most classes; most entries times values a lane

// Class i * 64 + lane of a row in registers, -inf behind the last.
template <typename TI, int NV>
__device__ __forceinline__ void wave_load(const TI* s, int K, float (&v)[NV]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < NV; ++i) v[i] = i * 64 + lane < K ? to_f32(s[i * 64 + lane]) : -INFINITY;
}
template <int NV>
__device__ __forceinline__ RowStats wave_stats(const float (&v)[NV], float it2) {
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) mx = fmaxf(mx, v[i]);
  RowStats r(wave_max(mx), it2);
#pragma unroll
  for (int i = 0; i < NV; ++i) r.add(v[i]);
  r.z = wave_sum(r.z);
  r.t = wave_sum(r.t);
  return r;
}

template <typename TI, typename TO, int NV>
__global__ __launch_bounds__(256) void score_grad_wave_kernel(const TI* logits, TO* dlogits, int64_t M, const ScoreGradP p) {
  const int lane = threadIdx.x & 63, K = p.K;
  const int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= M) return;
  TO* d = dlogits + m * p.ldd;
  float v[NV], own[NV];
  wave_load(logits + m * p.ld, K, v);
  int at = -1;
  float g = 0.f;
  if (lane < p.n) {
    at = p.ids[m * p.n + lane];
    if (at < 0 || at >= K) at = -1;
    else g = p.dlogprob[m * p.n + lane];
  }
  const float h = p.dentropy ? p.dentropy[m] : 0.f;
  const RowStats r = wave_stats(v, p.it2);
  const float sum_g = wave_sum(g);
  const bool zero = (!__any(!(g == 0.f)) && h == 0.f) || (!r.some && r.good());
#pragma unroll
  for (int i = 0; i < NV; ++i) own[i] = 0.f;
  for (int j = 0; j < p.n; ++j) {
    const int c = __builtin_amdgcn_readlane(at, j);
    const float gj = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), j));
#pragma unroll
    for (int i = 0; i < NV; ++i) own[i] += i * 64 + lane == c ? gj : 0.f;
  }
  const float mean = r.t / r.z, per = p.itau / r.z;
  const float A = -per * (sum_g - h * LN2_F * mean), B = -per * h * LN2_F;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = i * 64 + lane;
    const float y = r.y_of(v[i]);
    if (c < K) d[c] = from_f32<TO>(zero ? 0.f : exp2_(y) * fmaf(B, fmaxf(y, Y_MIN), A) + own[i] * p.itau);
  }
  for (int c = K + lane; c < K + p.pad; c += 64) d[c] = from_f32<TO>(0.f);
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// Rows that a wave holds are a workgroup of one wave each: its barriers wait for nobody, and a CU has 32 rows.  A few long
// rows are done sooner by more threads each.  (us, by a wave / by a workgroup of 256; 8 most likely classes: 20000 float32
// rows of 100 13.1 / 38.3, 5000 bf16 rows of 1000 6.9 / 12.9, 12000 of 1500 17.2 / 34.1, of 3500 27.4 / 31.4, one of 3000
// 5.0 / 3.9; gradients: 5000 bf16 rows of 1000 7.3 / 12.6, 12000 of 1500 20.7 / 33.4, 1024 of 2000 4.8 / 5.4.)
static bool one_wave(int64_t M, int32_t K) { return K <= 1024 || (K <= 64 * 64 && M >= 1024); }
template <typename TI, typename F> static void by_wave(int32_t K, F f) {
  constexpr int V = Wide<TI>::n;
  constexpr std::integral_constant<int, 64> t{};
  if (K <= 16 * 64) f(t, std::integral_constant<int, V>{}, std::integral_constant<int, 16 / V>{});
  else if (K <= 32 * 64) f(t, std::integral_constant<int, V>{}, std::integral_constant<int, 32 / V>{});
  else f(t, std::integral_constant<int, V>{}, std::integral_constant<int, 64 / V>{});
}

template <typename TI>
int score_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, const softmax_scores& q, hipStream_t stream) {
  const ScoreP p{ld, K, q.n, q.k, LOG2E_F / q.temperature, 1.f / q.temperature, q.ids, q.logprob, q.entropy, q.top, q.idx};
  auto launch = [&](auto t, auto v, auto nv, auto top) {
    constexpr int T = decltype(t)::value, V = decltype(v)::value, NV = decltype(nv)::value;
    BLSTM_LAUNCH("softmax_logprob_rows", (score_rows_kernel<TI, T, V, NV, decltype(top)::value>), dim3((unsigned)M),
                 dim3(T), 0, stream, logits, p);
  };
  auto with = [&](auto t, auto v, auto nv) {
    if (q.k) launch(t, v, nv, std::true_type{});
    else launch(t, v, nv, std::false_type{});
  };
  // 64 maxima give a threshold for up to 32 classes
  if (q.k <= 32 && q.n <= 64 && one_wave(M, K)) {
    using One = std::integral_constant<int, 1>;
    if (K <= 4 * 64) with(std::integral_constant<int, 64>{}, One{}, std::integral_constant<int, 4>{});
    else if (K <= 8 * 64) with(std::integral_constant<int, 64>{}, One{}, std::integral_constant<int, 8>{});
    else by_wave<TI>(K, with);
    return blstm_check_launch("softmax_logprob_rows");
  }
  if (q.k <= 128) by_length<TI, 128 * 1024, true>(K, with);
  else by_length<TI, 128 * 1024, false>(K, with);
  return blstm_check_launch("softmax_logprob_rows");
}
template int score_rows<float>(const float*, int64_t, int64_t, int32_t, const softmax_scores&, hipStream_t);
template int score_rows<bf16>(const bf16*, int64_t, int64_t, int32_t, const softmax_scores&, hipStream_t);

template <typename TI, typename TO>
int score_grad_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, const softmax_score_grads& q, TO* dlogits,
                    int64_t ldd, int32_t pad, hipStream_t stream) {
  const ScoreGradP p{ld, ldd, K, q.n, pad, LOG2E_F / q.temperature, 1.f / q.temperature, q.ids, q.dlogprob, q.dentropy};
  if (K <= WAVE_K && q.n * cdiv(K, 64) <= WAVE_LIST) {
    auto wave = [&](auto nv) {
      BLSTM_LAUNCH("softmax_logprob_bwd_rows", (score_grad_wave_kernel<TI, TO, decltype(nv)::value>),
                   dim3((unsigned)cdiv(M, 4)), dim3(256), 0, stream, logits, dlogits, M, p);
    };
    if (K <= 2 * 64) wave(std::integral_constant<int, 2>{});
    else if (K <= 4 * 64) wave(std::integral_constant<int, 4>{});
    else wave(std::integral_constant<int, 8>{});
    return blstm_check_launch("softmax_logprob_bwd_rows");
  }
  auto with = [&](auto t, auto v, auto nv) {
    constexpr int T = decltype(t)::value, V = decltype(v)::value, NV = decltype(nv)::value;
    BLSTM_LAUNCH("softmax_logprob_bwd_rows", (score_grad_kernel<TI, TO, T, V, NV>), dim3((unsigned)M), dim3(T), 0,
                 stream, logits, dlogits, p);
  };
  if (q.n <= 64 && one_wave(M, K)) {
    by_wave<TI>(K, with);
    return blstm_check_launch("softmax_logprob_bwd_rows");
  }
  by_length<TI, 128 * 1024, true>(K, with);
  return blstm_check_launch("softmax_logprob_bwd_rows");
}
template int score_grad_rows<float, float>(const float*, int64_t, int64_t, int32_t, const softmax_score_grads&, float*, int64_t, int32_t, hipStream_t);
template int score_grad_rows<float, bf16>(const float*, int64_t, int64_t, int32_t, const softmax_score_grads&, bf16*, int64_t, int32_t, hipStream_t);
template int score_grad_rows<bf16, bf16>(const bf16*, int64_t, int64_t, int32_t, const softmax_score_grads&, bf16*, int64_t, int32_t, hipStream_t);

softmax_scores scores_from(const softmax_scores& q, int64_t r0) {
  softmax_scores o = q;
  if (q.n) { o.ids += r0 * q.n; o.logprob += r0 * q.n; }
  if (q.entropy) o.entropy += r0;
  if (q.k) { o.top += r0 * q.k; o.idx += r0 * q.k; }
  return o;
}
softmax_score_grads score_grads_from(const softmax_score_grads& g, int64_t r0) {
  softmax_score_grads o = g;
  if (g.n) { o.ids += r0 * g.n; o.dlogprob += r0 * g.n; }
  if (g.dentropy) o.dentropy += r0;
  return o;
}

static int check_list(int32_t n, int32_t K, float temperature, const char* what, const char* fn) {
  if (K > SOFTMAX_MAX_CLASSES) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: K > %d", fn, SOFTMAX_MAX_CLASSES);
  if (n < 0) return blstm_fail(BLSTM_EINVAL, "%s: %s is negative", fn, what);
  if (n > MAXK) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: %s > %d", fn, what, MAXK);
  if (!(temperature > 0.f) || !std::isnormal(temperature))
    return blstm_fail(BLSTM_EINVAL, "%s: the temperature must be positive and finite", fn);
  return BLSTM_OK;
}
int check_scores(const softmax_scores* q, int32_t K, const char* fn) {
  if (!q) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  int rc = check_list(q->n, K, q->temperature, "n", fn);
  if (!rc) rc = check_list(q->k, K, q->temperature, "k", fn);
  if (rc) return rc;
  if (q->k > K) return blstm_fail(BLSTM_EINVAL, "%s: k=%d above K=%d", fn, q->k, K);
  if ((q->n && (!q->ids || !q->logprob)) || (q->k && (!q->top || !q->idx)))
    return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (!q->n && !q->k && !q->entropy) return blstm_fail(BLSTM_EINVAL, "%s: nothing is asked for", fn);
  return BLSTM_OK;
}
int check_score_grads(const softmax_score_grads* g, int32_t K, const char* fn) {
  if (!g) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  const int rc = check_list(g->n, K, g->temperature, "n", fn);
  if (rc) return rc;
  if (g->n && (!g->ids || !g->dlogprob)) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (!g->n && !g->dentropy) return blstm_fail(BLSTM_EINVAL, "%s: no gradient is given", fn);
  return BLSTM_OK;
}

static int check_rows(const char* fn, const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision) {
  if (M < 1 || K < 1) return blstm_fail(BLSTM_EINVAL, "%s: M and K must be positive (M=%lld K=%d)", fn, (long long)M, K);
  if (!logits) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (precision != BLSTM_FP32 && precision != BLSTM_BF16)
    return blstm_fail(BLSTM_EINVAL, "%s: precision must be BLSTM_FP32 or BLSTM_BF16", fn);
  if (ld < K) return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  if (M > LAUNCH_THREADS / 1024) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: too many rows", fn);
  return BLSTM_OK;
}

extern "C" int softmax_logprob_rows(const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision,
                                    const softmax_scores* scores, hipStream_t stream) {
  int rc = check_rows("softmax_logprob_rows", logits, ld, M, K, precision);
  if (!rc) rc = check_scores(scores, K, "softmax_logprob_rows");
  if (rc) return rc;
  return precision == BLSTM_BF16 ? score_rows((const bf16*)logits, ld, M, K, *scores, stream)
                                 : score_rows((const float*)logits, ld, M, K, *scores, stream);
}

extern "C" int softmax_logprob_bwd_rows(const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision,
                                        const softmax_score_grads* grads, void* dlogits, int64_t ldd,
                                        hipStream_t stream) {
  int rc = check_rows("softmax_logprob_bwd_rows", logits, ld, M, K, precision);
  if (!rc) rc = check_score_grads(grads, K, "softmax_logprob_bwd_rows");
  if (rc) return rc;
  if (!dlogits) return blstm_fail(BLSTM_EINVAL, "softmax_logprob_bwd_rows: NULL pointer");
  if (ldd < K) return blstm_fail(BLSTM_EINVAL, "softmax_logprob_bwd_rows: a row pitch is below its row");
  if (dlogits == logits && ldd != ld)
    return blstm_fail(BLSTM_EINVAL, "softmax_logprob_bwd_rows: dlogits over logits with another row pitch");
  if (precision == BLSTM_BF16)
    return score_grad_rows((const bf16*)logits, ld, M, K, *grads, (bf16*)dlogits, ldd, 0, stream);
  return score_grad_rows((const float*)logits, ld, M, K, *grads, (float*)dlogits, ldd, 0, stream);
}
