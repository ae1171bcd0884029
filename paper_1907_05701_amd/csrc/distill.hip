// Row operators of distillation: a teacher's top logits, and a student's loss
// and logit gradients against them.  One workgroup per row.
//
// Exponentials are base-2 hardware ones of differences from a row maximum;
// sums are float32 in a fixed order.
#include <math.h>

#include <cmath>

#include "common.hpp"
#include "distill.hpp"

#define LOG2E_F 1.4426950408889634f
#define LN2_F 0.6931471805599453f
static_assert(SOFTMAX_MAX_CLASSES == 1 << 18, "bits of a class");
static constexpr int RT = 512;             // threads of a row
static constexpr int RW = RT / 64;
static constexpr int CAND = 1024;          // most candidates kept in LDS
static constexpr int MAXK = SOFTMAX_MAX_TOP;
static_assert(MAXK <= RT && MAXK <= CAND, "the k-th largest of the threads' maxima bounds the k-th logit");

__device__ __forceinline__ float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }

// Sum and maximum over the workgroup, in lane and wave order; buf: RW floats.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float row_sum(float v, float* buf) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = buf[0];
#pragma unroll
  for (int w = 1; w < RW; ++w) t += buf[w];
  return t;
}
// a NaN among the values is the maximum
__device__ __forceinline__ float max_nan(float a, float b) { return (a > b || a != a) ? a : b; }
__device__ __forceinline__ float row_max(float v, float* buf) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max_nan(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = buf[0];
#pragma unroll
  for (int w = 1; w < RW; ++w) t = max_nan(t, buf[w]);
  return t;
}

// Calls f(column, value) for the thread's columns of a row.
template <typename TI> struct Wide;
template <> struct Wide<float> { typedef f32x4 type; static constexpr int n = 4; };
template <> struct Wide<bf16> { typedef bf16x8 type; static constexpr int n = 8; };
template <typename TI, typename F>
__device__ __forceinline__ void each(const TI* s, int K, bool vec, F f) {
  constexpr int V = Wide<TI>::n;
  typedef typename Wide<TI>::type W;
  int done = 0;
  if (vec) {
    done = K / V * V;
    for (int c = (int)threadIdx.x * V; c < done; c += RT * V) {
      const W v = *(const W*)(s + c);
#pragma unroll
      for (int i = 0; i < V; ++i) f(c + i, (float)v[i]);
    }
  }
  for (int c = done + (int)threadIdx.x; c < K; c += RT) f(c, to_f32(s[c]));
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
// The k largest of a row.  Each thread's maximum is one of RT; the k-th largest of
// those is no larger than the row's k-th, and few logits lie above it
// (about RT ln(RT / (RT - k)) of them in no particular order), so the logits
// from there on are collected and ranked by counting.  Rows whose logits
// bunch (ties, or all large ones in one thread's columns) can have more
// than CAND candidates: their k-th logit, and the last class that ties with
// it, are then found bit by bit.
// ---------------------------------------------------------------------------
template <typename TI>
__global__ __launch_bounds__(RT) void topk_rows_kernel(const TI* __restrict__ logits, int64_t ld, int K, int k,
                                                       float l2t, float* __restrict__ top, int32_t* __restrict__ idx,
                                                       float* __restrict__ rest, bool vec) {
  __shared__ uint32_t tmax[RT];
  __shared__ uint64_t cand[CAND];
  __shared__ uint32_t thr, count, cnt[2][RW];
  __shared__ uint64_t kth;
  __shared__ float buf[RW];
  const int64_t m = blockIdx.x;
  const TI* s = logits + m * ld;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t mx = 0;
  each(s, K, vec, [&](int, float v) { mx = max(mx, order_word(v)); });
  tmax[tid] = mx;
  if (tid == 0) count = 0;
  __syncthreads();
  if (wave == 0) {
    uint32_t w[RW], t = 0;
#pragma unroll
    for (int i = 0; i < RW; ++i) w[i] = tmax[i * 64 + lane];
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t c = t | (1u << bit);
      int n = 0;
#pragma unroll
      for (int i = 0; i < RW; ++i) n += __popcll(__ballot(w[i] >= c));
      if (n >= k) t = c;
    }
    if (lane == 0) thr = t;
  }
  __syncthreads();
  const uint32_t th = thr;
  each(s, K, vec, [&](int c, float v) {
    const uint32_t w = order_word(v);
    if (w >= th) {
      const uint32_t at = atomicAdd(&count, 1u);
      if (at < (uint32_t)CAND) cand[at] = ((uint64_t)w << 32) | (uint32_t)~c;
    }
  });
  __syncthreads();
  int n = (int)min(count, (uint32_t)CAND);
  if (count > (uint32_t)CAND) {
    // the k-th word: the largest with at least k words from it on
    uint64_t t = 0;   // word, then ~class: the same order as the candidates'
    int par = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t c = t | (1ull << bit);
      if (bit < 32 && bit >= 18) {   // set in the complement of every class
        t = c;
        continue;
      }
      uint32_t mine = 0;
      each(s, K, vec, [&](int col, float v) {
        mine += ((((uint64_t)order_word(v)) << 32) | (uint32_t)~col) >= c;
      });
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mine += __shfl_xor(mine, o);
      if (lane == 0) cnt[par][wave] = mine;
      __syncthreads();
      uint32_t all = 0;
#pragma unroll
      for (int i = 0; i < RW; ++i) all += cnt[par][i];
      if (all >= (uint32_t)k) t = c;
      par ^= 1;
    }
    if (tid == 0) count = 0;
    __syncthreads();
    each(s, K, vec, [&](int c, float v) {
      const uint64_t w = ((uint64_t)order_word(v) << 32) | (uint32_t)~c;
      if (w >= t) cand[atomicAdd(&count, 1u)] = w;   // exactly k
    });
    __syncthreads();
    n = k;
  }
  for (int i = tid; i < n; i += RT) {
    const uint64_t w = cand[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += cand[j] > w;
    if (r < k) {
      top[m * k + r] = order_value((uint32_t)(w >> 32));
      idx[m * k + r] = (int32_t)~(uint32_t)w;
      if (r == k - 1) kth = w;
    }
  }
  if (!rest) return;
  __syncthreads();
  const uint64_t last = kth;
  float rm = -INFINITY;
  each(s, K, vec, [&](int c, float v) {
    if ((((uint64_t)order_word(v) << 32) | (uint32_t)~c) < last) rm = max_nan(rm, v);
  });
  rm = row_max(rm, buf);
  float sum = 0.f;
  if (fabsf(rm) < INFINITY) {
    each(s, K, vec, [&](int c, float v) {
      if ((((uint64_t)order_word(v) << 32) | (uint32_t)~c) < last) sum += exp2_((v - rm) * l2t);
    });
  }
  sum = row_sum(sum, buf);
  // the others' largest logit alone where it is infinite or a NaN, or there is none
  if (tid == 0) rest[m] = fabsf(rm) < INFINITY ? rm * (l2t * LN2_F) + log2f(sum) * LN2_F : rm;
}

// ---------------------------------------------------------------------------
// Loss and gradient.  With u = s / tau, the listed classes' probabilities p
// (equal classes' added up), the others' r, and Z, Zr the sums of e^u over all
// and over the others:
//   KL = sum p (log p - log q) + r (log r - log(Zr / Z)),  q = e^u / Z
//   d(tau^2 KL)/ds = tau (q - p) where listed, tau e^u (1/Z - r/Zr) elsewhere
// The others' sum has a maximum of its own, so that it does not vanish
// beside listed logits however large they are.
// ---------------------------------------------------------------------------
struct DistillP {
  int64_t ld, ldd;
  const float *top, *rest, *weights;
  const int32_t *idx, *labels;
  float* row_loss;
  int K, k, pad;
  float it2, tau, soft, hard, scale;   // it2: log2 e / tau
  bool vec, vecd;
};

template <typename TI, typename TO>
__global__ __launch_bounds__(RT) void distill_rows_kernel(const TI* logits, TO* dlogits, const DistillP p) {
  extern __shared__ uint32_t listed[];   // a bit per class
  __shared__ float pv[MAXK], uv[MAXK];
  __shared__ int32_t iv[MAXK];
  __shared__ float buf[RW];
  __shared__ uint32_t dup;
  const int64_t m = blockIdx.x;
  const TI* s = logits + m * p.ld;
  TO* d = dlogits + m * p.ldd;
  const int tid = threadIdx.x, K = p.K;
  const float weight = p.weights ? p.weights[m] : 1.f;
  for (int c = K + tid; c < K + p.pad; c += RT) d[c] = from_f32<TO>(0.f);
  if (weight == 0.f) {
    for (int c = tid; c < K; c += RT) d[c] = from_f32<TO>(0.f);
    if (tid == 0) p.row_loss[m] = 0.f;
    return;
  }
  const int words = (K + 31) / 32;
  for (int i = tid; i < words; i += RT) listed[i] = 0;
  if (tid == 0) dup = 0;
  __syncthreads();
  // the teacher's probabilities (base-2 exponents throughout)
  int at = -1;
  float t2 = -INFINITY;
  if (tid < p.k) {
    at = p.idx[m * p.k + tid];
    if (at < 0 || at >= K) at = -1;
    else {
      t2 = p.top[m * p.k + tid] * p.it2;
      if (atomicOr(&listed[at >> 5], 1u << (at & 31)) & (1u << (at & 31))) dup = 1;
    }
    iv[tid] = at;
  }
  const float r2 = p.rest ? p.rest[m] * LOG2E_F : -INFINITY;
  const float tm = row_max(max_nan(t2, r2), buf);
  float prob = 0.f, r = 0.f, tz = 1.f;
  const bool taught = !(tm == -INFINITY);
  if (taught) {
    prob = exp2_(t2 - tm);
    r = exp2_(r2 - tm);
  }
  tz = row_sum(prob, buf) + r;
  if (taught) { prob /= tz; r /= tz; }
  float lp = taught ? t2 - tm - log2f(tz) : 0.f;   // log2 of it
  const float lr = taught ? r2 - tm - log2f(tz) : 0.f;
  float own = prob;       // of the entry's class
  bool lead = at >= 0;    // the class's first entry
  if (tid < p.k) pv[tid] = prob;
  __syncthreads();
  if (dup && at >= 0) {
    own = 0.f;
    for (int j = 0; j < p.k; ++j)
      if (iv[j] == at) {
        own += pv[j];
        if (j < tid) lead = false;
      }
    lp = log2f(own);
  }
  // the student's maxima: the others' (times log2 e / tau), the row's
  float rm = -INFINITY, am = -INFINITY;
  each(s, K, p.vec, [&](int c, float v) {
    am = max_nan(am, v);
    if (!((listed[c >> 5] >> (c & 31)) & 1u)) rm = max_nan(rm, v);
  });
  rm = row_max(rm, buf) * p.it2;
  am = row_max(am, buf);
  const float rref = rm == -INFINITY ? 0.f : rm, aref = am == -INFINITY ? 0.f : am;
  float zr = 0.f, z1 = 0.f;
  each(s, K, p.vec, [&](int c, float v) {
    if (!((listed[c >> 5] >> (c & 31)) & 1u)) zr += exp2_(v * p.it2 - rref);
    if (p.labels) z1 += exp2_((v - aref) * LOG2E_F);
  });
  zr = row_sum(zr, buf);
  if (p.labels) z1 = row_sum(z1, buf);
  // the listed logits, before any gradient is written over them
  const float sv = at >= 0 ? to_f32(s[at]) : -INFINITY, u = sv * p.it2;
  const float um = aref * p.it2;   // the row's maximum, as u
  const float ez = lead ? exp2_(u - um) : 0.f;
  const float eo = rm == -INFINITY ? 0.f : exp2_(rref - um);   // the others' sum in the same terms
  const float z = row_sum(ez, buf) + zr * eo;
  const float l2z = log2f(z);
  float kl = 0.f;
  if (at >= 0 && prob > 0.f) kl = prob * (lp - (u - um - l2z));
  kl = row_sum(kl, buf);
  if (r > 0.f) kl += r * (lr - (log2f(zr) + rref - um - l2z));
  const int lab = p.labels ? p.labels[m] : -1;
  const bool marked = lab >= 0 && lab < K;
  const float sl = marked ? to_f32(s[lab]) : 0.f;
  float loss = taught ? p.soft * p.tau * p.tau * kl * LN2_F : 0.f;
  if (marked) loss += p.hard * (aref + log2f(z1) * LN2_F - sl);
  if (tid == 0) p.row_loss[m] = weight * loss;
  const float ks = taught ? p.scale * weight * p.soft * p.tau : 0.f, kh = marked ? p.scale * weight * p.hard : 0.f;
  const float cr = ks * (eo / z - (r > 0.f && zr > 0.f ? r / zr : 0.f));   // of e^(u - rref) in the others
  const float ch = marked ? kh / z1 : 0.f;
  __syncthreads();   // every listed logit and the label's have been read
  {
    // a class's dense part; the listed ones' soft part follows
    auto grad = [&](int c, float v) {
      float g = 0.f;
      if (!((listed[c >> 5] >> (c & 31)) & 1u)) g = cr * exp2_(v * p.it2 - rref);
      if (marked) {
        g += ch * exp2_((v - aref) * LOG2E_F);
        if (c == lab) g -= kh;
      }
      return g;
    };
    constexpr int V = Wide<TI>::n;
    typedef typename Wide<TI>::type W;
    int done = 0;
    if (p.vec && p.vecd) {
      done = K / V * V;
      for (int c = tid * V; c < done; c += RT * V) {
        const W v = *(const W*)(s + c);
        TO o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = from_f32<TO>(grad(c + i, (float)v[i]));
        __builtin_memcpy(__builtin_assume_aligned(d + c, V * sizeof(TO)), o, V * sizeof(TO));
      }
    }
    for (int c = done + tid; c < K; c += RT) d[c] = from_f32<TO>(grad(c, to_f32(s[c])));
  }
  __syncthreads();   // the dense parts lie before the listed ones' values
  if (lead) {
    float g = ks * (ez / z - own);
    if (marked) {
      g += ch * exp2_((sv - aref) * LOG2E_F);
      if (at == lab) g -= kh;
    }
    d[at] = from_f32<TO>(g);
  }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
template <typename TI>
int topk_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, int32_t k, float temperature, float* top,
              int32_t* idx, float* rest, hipStream_t stream) {
  constexpr int V = Wide<TI>::n;
  const bool vec = ((uintptr_t)logits % 16) == 0 && ld % V == 0;
  BLSTM_LAUNCH("softmax_topk_rows", topk_rows_kernel<TI>, dim3((unsigned)M), dim3(RT), 0, stream, logits, ld, K, k,
               LOG2E_F / temperature, top, idx, rest, vec);
  return blstm_check_launch("softmax_topk_rows");
}
template int topk_rows<float>(const float*, int64_t, int64_t, int32_t, int32_t, float, float*, int32_t*, float*, hipStream_t);
template int topk_rows<bf16>(const bf16*, int64_t, int64_t, int32_t, int32_t, float, float*, int32_t*, float*, hipStream_t);

template <typename TI, typename TO>
int distill_rows(const TI* logits, int64_t ld, int64_t M, int32_t K, const softmax_teacher* t, float loss_scale,
                 float* row_loss, TO* dlogits, int64_t ldd, int32_t pad, hipStream_t stream) {
  constexpr int V = Wide<TI>::n;
  DistillP p{};
  p.ld = ld; p.ldd = ldd; p.top = t->top; p.rest = t->rest; p.weights = t->weights; p.idx = t->idx;
  p.labels = t->hard != 0.f ? t->labels : nullptr;
  p.row_loss = row_loss; p.K = K; p.k = t->k; p.pad = pad;
  p.it2 = LOG2E_F / t->temperature; p.tau = t->temperature; p.soft = t->soft; p.hard = t->hard; p.scale = loss_scale;
  p.vec = ((uintptr_t)logits % 16) == 0 && ld % V == 0;
  p.vecd = ((uintptr_t)dlogits % (V * sizeof(TO))) == 0 && ldd % V == 0;
  BLSTM_LAUNCH("softmax_distill_rows", (distill_rows_kernel<TI, TO>), dim3((unsigned)M), dim3(RT),
               (size_t)cdiv(K, 32) * 4, stream, logits, dlogits, p);
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
  if (M > 0x7fffffff) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: too many rows", fn);
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
