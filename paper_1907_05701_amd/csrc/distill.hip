// Row operators of distillation: a teacher's top logits, and a student's loss
// and logit gradients against them.  One workgroup per row.
//
// Exponentials are base-2 hardware ones of differences from a row maximum;
// sums are float32 in a fixed order.  Memory bounds both: 2688 bf16 rows of 32000
// logits, the top 32 in 49 us (172 MB, 3.5 TB/s; the vector unit issues 36 us of it,
// and a row's search, candidates and ranks are barriers that only other rows hide), loss and gradients
// with labels in 77 us (344 MB, 4.5 TB/s).
#include <cmath>

#include "distill.hpp"
#include "rows.hpp"

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
  const float thr = order_value(max(kth_max<12>(l, p.k), LOWEST));
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
  const uint32_t tw = max(kth_max<std::is_same<TI, bf16>::value ? 16 : 12>(l, p.k), LOWEST);
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
