// Products in 8-bit integers with a scale for each token and each channel:
//   y[m][n] = float(sum_k q[m][k] w[n][k]) (x_scale[m] w_scale[n]) + bias[n]
// The sum is exact, and each step behind it one float32 rounding, so that every kernel here gives the same bits.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "int8_tile.hpp"
#include "score.hpp"

// ---------------------------------------------------------------------------
// Tokens to integers.  T threads a row (a wave, or a workgroup of 256); a row
// of up to NV vectors a thread is read once, longer ones (NV = 0) twice.
// ---------------------------------------------------------------------------
template <typename TI, int T, int NV>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const TI* __restrict__ x, int64_t ldx, int64_t M, int K,
                                                            int8_t* __restrict__ q, int64_t ldq, int Kq,
                                                            float* __restrict__ scale) {
  constexpr int V = Vec16<TI>::n, NR = NV ? NV : 1;
  __shared__ uint32_t buf[4];
  const int tid = T == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t m = T == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (T == 64 && m >= M) return;   // no barrier there
  const TI* s = x + m * ldx;
  int8_t* d = q + m * ldq;
  Vec16<TI> v[NR];
  uint32_t mx = 0;
  auto read = [&](Vec16<TI>& o, int c) {   // (q may have many more columns than a short row)
    if (K >= V) o.load(s, c, K);
    else o.zero();
    if (K % V) o.patch(s, c, K);
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (K >= V) v[i].load(s, (i * T + tid) * V, K);
      else v[i].zero();
    }
    if (K % V) {
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i].patch(s, (i * T + tid) * V, K);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) mx = v[i].max(mx);
  } else {
    for (int c = tid * V; c < K; c += T * V) {
      read(v[0], c);
      mx = v[0].max(mx);
    }
  }
  mx = wave_max_bits(Vec16<TI>::word(mx));
  if constexpr (T == 256) {
    if ((tid & 63) == 0) buf[tid >> 6] = mx;
    __syncthreads();
    mx = max(max(buf[0], buf[1]), max(buf[2], buf[3]));
  }
  const Quant to(mx);
  if (tid == 0) scale[m] = to.scale;
  auto store = [&](int c, const Vec16<TI>& o) {
    if (c >= Kq) return;   // Kq is a multiple of V
    uint32_t w[V / 4];
    to(o.v, w);
    __builtin_memcpy(d + c, w, V);
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) store((i * T + tid) * V, v[i]);
  } else {
    for (int c = tid * V; c < Kq; c += T * V) {
      read(v[0], c);
      store(c, v[0]);
    }
  }
}

template <typename TI>
void int8_quantize(const TI* x, int64_t ldx, int64_t M, int32_t K, int8_t* q, int64_t ldq, int32_t Kq, float* scale,
                   hipStream_t stream) {
  constexpr int V = Vec16<TI>::n;
  auto launch = [&](auto t, auto nv) {
    constexpr int T = decltype(t)::value, NV = decltype(nv)::value;
    BLSTM_LAUNCH("int8_quantize_rows", (quantize_rows_kernel<TI, T, NV>), dim3((unsigned)(T == 64 ? cdiv(M, 4) : M)),
                 dim3(256), 0, stream, x, ldx, M, (int)K, q, ldq, (int)Kq, scale);
  };
#define INT(n) std::integral_constant<int, n>{}
  if (Kq <= 64 * V) launch(INT(64), INT(1));
  else if (Kq <= 2 * 64 * V) launch(INT(64), INT(2));
  else if (Kq <= 4 * 64 * V) launch(INT(64), INT(4));
  else if (Kq <= 2 * 256 * V) launch(INT(256), INT(2));
  else if (Kq <= 4 * 256 * V) launch(INT(256), INT(4));
  else launch(INT(256), INT(0));
#undef INT
}
template void int8_quantize<float>(const float*, int64_t, int64_t, int32_t, int8_t*, int64_t, int32_t, float*, hipStream_t);
template void int8_quantize<bf16>(const bf16*, int64_t, int64_t, int32_t, int8_t*, int64_t, int32_t, float*, hipStream_t);

// ---------------------------------------------------------------------------
// The product.
// ---------------------------------------------------------------------------
// The same for up to 16 FN tokens of floats (TO, also y's), quantised on the way by every workgroup for itself while
// its weights are in flight; NW waves, each with every NW-th 64 of K.
struct Int8FewP {
  Int8P p;
  const void* x;
  int64_t ldx;
  int K, cols;   // columns of x, p.K those of the weights; in LDS
};
// Of all tokens, whom every workgroup quantises: 64 tokens of 1024 take 13.4 us in one launch, and 3.2 + 6.2 in two.
static constexpr int64_t FEW_VALUES = 1 << 15;
template <typename TO, int FN, int NW, int NV>
__global__ __launch_bounds__(NW * 64) void int8_few_tokens_kernel(const Int8FewP a) {
  const Int8P& p = a.p;
  constexpr int U = 4;
  extern __shared__ __attribute__((aligned(16))) char tokens[];
  __shared__ float xs[16 * FN];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, fr = lane & 15, fc = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int8_t* wr = p.w + min(n0 + fr, p.N - 1) * p.ldw;   // rows past the last: any, dropped at the end
  const int k0 = wid * 64 + fc * 16;
  i32x4 w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) w[u] = ints16(wr, k0 + u * NW * 64, p.K);
  tokens_to_lds<TO, NW, NV < 8 ? 8 / NV : 1, NV>((const TO*)a.x, a.ldx, (int)p.M, a.K, a.cols, tokens, xs);
  __syncthreads();
  const char* xr[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) xr[j] = tokens + (j * 16 + fr < p.M ? j * 16 + fr : 0) * (a.cols + 16);   // past the last token: any
  i32x4 acc[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) acc[j] = i32x4{0, 0, 0, 0};
  auto add = [&](i32x4 v, int k) {
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[j] = mma_i8(v, *(const i32x4*)(xr[j] + k), acc[j]);
  };
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (wid * 64 + u * NW * 64 < a.cols) add(w[u], k0 + u * NW * 64);
  for (int k = U * NW * 64; k < a.cols; k += U * NW * 64) {
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = ints16(wr, k0 + k + u * NW * 64, p.K);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (wid * 64 + k + u * NW * 64 < a.cols) add(w[u], k0 + k + u * NW * 64);
  }
  __syncthreads();   // the tokens are done with
  i32x4* part = (i32x4*)tokens;
#pragma unroll
  for (int j = 0; j < FN; ++j) part[(wid * FN + j) * 64 + lane] = acc[j];
  __syncthreads();
  if (wid >= FN) return;   // a wave for each 16 tokens
  i32x4 sum{0, 0, 0, 0};
#pragma unroll
  for (int v = 0; v < NW; ++v) sum += part[(v * FN + wid) * 64 + lane];
  put4<TO>(p, wid * 16 + fr, n0 + 4 * fc, sum, xs[wid * 16 + fr]);
}
static int few_fragments(int64_t M) { return M <= 16 ? 1 : M <= 32 ? 2 : 4; }   // of 16 tokens
static bool few_tokens_ok(int64_t M, int32_t Kw) {
  return M <= 64 && 16 * few_fragments(M) * rup(Kw, 64) <= FEW_VALUES;
}
// NV vectors a lane hold a token; longer ones take twice as many, up to the longest that few_tokens_ok lets pass.
template <typename TO, int FN, int NW, int NV = 1>
static void few_tokens(const Int8FewP& a, hipStream_t s) {
  constexpr int COLS = NV * 64 * Vec16<TO>::n, MOST = FEW_VALUES / (16 * FN);
  if constexpr (COLS < MOST) {
    if (a.cols > COLS) return few_tokens<TO, FN, NW, 2 * NV>(a, s);
  }
  auto kernel = int8_few_tokens_kernel<TO, FN, NW, NV>;
  constexpr size_t most = FEW_VALUES + 64 * 16;
  const size_t bytes = std::max<size_t>((size_t)rup(a.p.M, 16) * (a.cols + 16), NW * FN * 1024);
  static std::atomic<uint64_t> raised{0};
  kc_raise_lds_limit((const void*)kernel, most, raised);
  BLSTM_LAUNCH("int8_linear_few", kernel, dim3((unsigned)cdiv(a.p.N, 16)), dim3(NW * 64), bytes, s, a);
}
template <typename TO>
static void few_tokens_rows(Int8FewP a, hipStream_t s) {
  a.cols = (int)rup(a.p.K, 64);
  switch (few_fragments(a.p.M)) {
    case 1: return few_tokens<TO, 1, 4>(a, s);
    case 2: return few_tokens<TO, 2, 8>(a, s);
    default: return few_tokens<TO, 4, 8>(a, s);
  }
}

template <typename TO>
static void product(Int8P p, hipStream_t s) {
  if (p.M <= 64) {
    const int fn = (int)cdiv(p.M, 16);
    const dim3 grid((unsigned)cdiv(p.N, 16), 1);
    if (fn == 1) BLSTM_LAUNCH("int8_linear_few", (int8_few_kernel<TO, 1>), grid, dim3(256), 0, s, p);
    else if (fn == 2) BLSTM_LAUNCH("int8_linear_few", (int8_few_kernel<TO, 2>), grid, dim3(256), 0, s, p);
    else BLSTM_LAUNCH("int8_linear_few", (int8_few_kernel<TO, 4>), grid, dim3(256), 0, s, p);
    return;
  }
  // 256x256 blocks stage and read the fewest bytes a product, one a CU: where they fill whole rounds of the chip and
  // their start and end count little.  128x192 ones, two a CU, where they leave few CUs idle; else 64x64 ones, with a
  // deeper ring where two a CU hold them all.  (us on uniform integers, 256x256 / 128x192 / 64x64 with two stages / with four.
  // 16384 x 4096 x 4096 237 / 264 / 407 / 440, 8192 x 4096 x 1024 44 / 48 / 66 / 74, 5000 x 4096 x 1024 37 / 32 / 43 / 47,
  // 2688 x 32000 x 256 61 / 59 / 74 / 93, 2688 x 4096 x 1024 20.7 / 18.2 / 22.3 / 26.9, 2688 x 2048 x 1024 18.5 / 11.3 / 13.5 /
  // 15.3, 2688 x 1024 x 4096 46 / 27.0 / 21.1 / 24.6, 1000 x 1000 x 8192 81 / 47 / 31.9 / 20.2, 1000 x 2048 x 1024
  // 17.5 / 10.2 / 6.3 / 6.4.  The values decide the clock: the first takes 191 on zeros.)
  const int64_t big = cdiv(p.M, 256) * cdiv(p.N, 256), rounds = cdiv(big, 256) * 256;
  if (p.K >= 1024 && 5 * big >= 4 * rounds) int8_tile_launch<TO, 256, 256, 4, 4, 128, 2>(p, s);
  else if (cdiv(p.M, 192) * cdiv(p.N, 128) >= 192) int8_tile_launch<TO, 128, 192, 2, 4, 128, 2>(p, s);
  else if (cdiv(p.M, 64) * cdiv(p.N, 64) > 512) int8_tile_launch<TO, 64, 64, 2, 2, 128, 2>(p, s);
  else int8_tile_launch<TO, 64, 64, 2, 2, 128, 4>(p, s);
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

static int check_precision(const char* fn, int32_t precision) {
  return precision == BLSTM_FP32 || precision == BLSTM_BF16
             ? BLSTM_OK
             : blstm_fail(BLSTM_EINVAL, "%s: precision must be BLSTM_FP32 or BLSTM_BF16", fn);
}
// Rows of integers: K columns, a multiple of 16, at a pitch of 16-byte pieces.
static int check_ints(const char* fn, const char* what, const int8_t* q, int64_t ld, int32_t K) {
  if (!q) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (K % 16 || ld % 16 || !aligned16(q))
    return blstm_fail(BLSTM_EINVAL, "%s: %s's columns and row pitch must be multiples of 16, its address 16-byte aligned", fn, what);
  if (ld < K) return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  if (K > INT8_MAX_K || ld > INT8_MAX_LD)
    return blstm_fail(BLSTM_EUNSUPPORTED, "%s: %s's rows are too long", fn, what);
  return BLSTM_OK;
}
static int check_sizes(const char* fn, int64_t M, int64_t N, int64_t K) {
  if (M < 1 || N < 1 || K < 1)
    return blstm_fail(BLSTM_EINVAL, "%s: sizes must be positive (%lld, %lld, %lld)", fn, (long long)M, (long long)N, (long long)K);
  if (M > LAUNCH_THREADS / 1024 || N >= 1 << 24 || cdiv(M, 128) * cdiv(N, 128) > LAUNCH_THREADS / 1024)
    return blstm_fail(BLSTM_EUNSUPPORTED, "%s: too many rows", fn);
  return BLSTM_OK;
}

extern "C" int int8_quantize_rows(const void* x, int64_t ldx, int64_t M, int32_t K, int32_t precision, int8_t* q,
                                  int64_t ldq, int32_t Kq, float* scale, hipStream_t stream) {
  const char* fn = "int8_quantize_rows";
  int rc = check_sizes(fn, M, 1, K);
  if (!rc) rc = check_precision(fn, precision);
  if (!rc) rc = check_ints(fn, "q", q, ldq, Kq);
  if (rc) return rc;
  if (!x || !scale) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (ldx < K || Kq < K) return blstm_fail(BLSTM_EINVAL, "%s: a row is longer than its pitch or q's columns", fn);
  if (precision == BLSTM_BF16) int8_quantize((const bf16*)x, ldx, M, K, q, ldq, Kq, scale, stream);
  else int8_quantize((const float*)x, ldx, M, K, q, ldq, Kq, scale, stream);
  return blstm_check_launch(fn);
}

extern "C" int int8_linear(const int8_t* q, int64_t ldq, const float* x_scale, int64_t M, const int8_t* w, int64_t ldw,
                           const float* w_scale, int32_t N, int32_t K, const float* bias, void* y, int64_t ldy,
                           int32_t precision, hipStream_t stream) {
  const char* fn = "int8_linear";
  int rc = check_sizes(fn, M, N, K);
  if (!rc) rc = check_precision(fn, precision);
  if (!rc) rc = check_ints(fn, "q", q, ldq, K);
  if (!rc) rc = check_ints(fn, "w", w, ldw, K);
  if (rc) return rc;
  if (!x_scale || !w_scale || !y) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (ldy < N) return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  Int8P p{};
  p.x = q; p.w = w; p.ldx = ldq; p.ldw = ldw; p.ldy = ldy; p.M = M; p.N = N; p.K = K;
  p.xs = x_scale; p.ws = w_scale; p.bias = bias; p.y = y;
  if (precision == BLSTM_BF16) product<bf16>(p, stream);
  else product<float>(p, stream);
  return blstm_check_launch(fn);
}

// ws: the tokens' integers [M][Kw], then their scales
static size_t tokens_bytes(int64_t M, int64_t Kw) { return (size_t)(rup(M * Kw, 256) + rup(M * 4, 256)); }

extern "C" int int8_linear_ws_bytes(int64_t M, int32_t K, size_t* bytes) {
  const int rc = check_sizes("int8_linear_ws_bytes", M, 1, K);
  if (rc) return rc;
  if (K > INT8_MAX_K) return blstm_fail(BLSTM_EUNSUPPORTED, "int8_linear_ws_bytes: K > %d", INT8_MAX_K);
  if (bytes) *bytes = tokens_bytes(M, rup(K, 16));
  return BLSTM_OK;
}

// Everything that the two calls behind it check, before either launches.
static int check_tokens(const char* fn, const void* x, int64_t ldx, int64_t M, int32_t K, int32_t precision,
                        const int8_t* w, int64_t ldw, const float* w_scale, int32_t N, int32_t Kw, const void* ws) {
  int rc = check_sizes(fn, M, N, K);
  if (!rc) rc = check_precision(fn, precision);
  if (!rc) rc = check_ints(fn, "w", w, ldw, Kw);
  if (rc) return rc;
  if (!x || !w_scale || !ws) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (ldx < K || Kw < K) return blstm_fail(BLSTM_EINVAL, "%s: a row is longer than its pitch or w's columns", fn);
  if (!aligned16(ws)) return blstm_fail(BLSTM_EINVAL, "%s: ws must be 16-byte aligned", fn);
  return BLSTM_OK;
}

extern "C" int int8_linear_rows(const void* x, int64_t ldx, int64_t M, int32_t K, int32_t precision, const int8_t* w,
                                int64_t ldw, const float* w_scale, int32_t N, int32_t Kw, const float* bias, void* y,
                                int64_t ldy, void* ws, hipStream_t stream) {
  const char* fn = "int8_linear_rows";
  int rc = check_tokens(fn, x, ldx, M, K, precision, w, ldw, w_scale, N, Kw, ws);
  if (rc) return rc;
  if (!y) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (ldy < N) return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  if (few_tokens_ok(M, Kw)) {
    Int8FewP a{};
    a.p.w = w; a.p.ldw = ldw; a.p.ldy = ldy; a.p.M = M; a.p.N = N; a.p.K = Kw; a.p.ws = w_scale; a.p.bias = bias; a.p.y = y;
    a.x = x; a.ldx = ldx; a.K = K;
    if (precision == BLSTM_BF16) few_tokens_rows<bf16>(a, stream);
    else few_tokens_rows<float>(a, stream);
    return blstm_check_launch(fn);
  }
  int8_t* q = (int8_t*)ws;
  float* scale = (float*)((char*)ws + rup(M * Kw, 256));
  rc = int8_quantize_rows(x, ldx, M, K, precision, q, Kw, Kw, scale, stream);
  if (rc) return rc;
  return int8_linear(q, Kw, scale, M, w, ldw, w_scale, N, Kw, bias, y, ldy, precision, stream);
}

// ---------------------------------------------------------------------------
// The head (int8_head.hip); tokens of more columns than that holds: logits of rows at a time, scored.
// ---------------------------------------------------------------------------
// Frames that the head takes at a time: equal parts, of at most about 180 MB of group maxima (K / 4 bytes a frame) and tokens.
static int64_t head_most(int64_t K, int64_t Kw) { return (180 << 20) / (Kw + 16 * cdiv(K, 64) + 64); }
static int64_t head_frames(int64_t M, int64_t K, int64_t Kw) { return cdiv(M, cdiv(M, head_most(K, Kw))); }
static int64_t logit_rows(int64_t M, int64_t K) { return std::min(M, std::max<int64_t>(64, (180 << 20) / (4 * rup(K, 4)))); }

extern "C" int int8_logprob_ws_bytes(int64_t M, int32_t K, int32_t Kw, size_t* bytes) {
  const int rc = check_sizes("int8_logprob_ws_bytes", M, K, Kw);
  if (rc) return rc;
  if (K > SOFTMAX_MAX_CLASSES || Kw > INT8_MAX_K) return blstm_fail(BLSTM_EUNSUPPORTED, "int8_logprob_ws_bytes: too many classes or columns");
  if (!bytes) return BLSTM_OK;
  const int32_t cols = (int32_t)rup(Kw, 16);
  *bytes = int8_head_fits(Kw) ? int8_head_bytes(std::min(M, head_most(K, cols)), K, cols)
                              : tokens_bytes(M, cols) + (size_t)logit_rows(M, K) * rup(K, 4) * 4;
  return BLSTM_OK;
}

extern "C" int int8_logprob_rows(const void* x, int64_t ldx, int64_t M, int32_t P, int32_t precision, const int8_t* w,
                                 int64_t ldw, const float* w_scale, int32_t K, int32_t Kw, const float* bias,
                                 const softmax_scores* scores, void* ws, hipStream_t stream) {
  const char* fn = "int8_logprob_rows";
  int rc = check_tokens(fn, x, ldx, M, P, precision, w, ldw, w_scale, K, Kw, ws);
  if (!rc) rc = check_scores(scores, K, fn);
  if (rc) return rc;
  int8_t* q = (int8_t*)ws;
  float* scale = (float*)((char*)ws + rup(M * Kw, 256));
  char* rest = (char*)ws + tokens_bytes(M, Kw);
  if (int8_head_fits(Kw)) {
    const int64_t step = head_frames(M, K, Kw);
    for (int64_t r0 = 0; !rc && r0 < M; r0 += step) {
      const int64_t n = std::min(step, M - r0);
      const softmax_scores sc = scores_from(*scores, r0);
      rc = precision == BLSTM_BF16
               ? int8_head((const bf16*)x + r0 * ldx, ldx, n, P, w, ldw, w_scale, K, Kw, bias, sc, (char*)ws, stream)
               : int8_head((const float*)x + r0 * ldx, ldx, n, P, w, ldw, w_scale, K, Kw, bias, sc, (char*)ws, stream);
    }
    return rc;
  }
  rc = int8_quantize_rows(x, ldx, M, P, precision, q, Kw, Kw, scale, stream);
  float* logits = (float*)rest;
  const int64_t ld = rup(K, 4), step = logit_rows(M, K);
  for (int64_t r0 = 0; !rc && r0 < M; r0 += step) {
    const int64_t n = std::min(step, M - r0);
    rc = int8_linear(q + r0 * Kw, Kw, scale + r0, n, w, ldw, w_scale, K, Kw, bias, logits, ld, BLSTM_FP32, stream);
    if (!rc) rc = score_rows<float>(logits, ld, n, K, scores_from(*scores, r0), stream);
  }
  return rc;
}
