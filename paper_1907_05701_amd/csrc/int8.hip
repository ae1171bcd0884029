// Products in 8-bit integers with a scale for each token and each channel:
//   y[m][n] = float(sum_k q[m][k] w[n][k]) (x_scale[m] w_scale[n]) + bias[n]
// The sum is exact, and each step behind it one float32 rounding, so that every kernel here gives the same bits.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "gemm_kc.hpp"
#include "int8.hpp"
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
  __shared__ float buf[4];
  const int tid = T == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t m = T == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (T == 64 && m >= M) return;   // no barrier there
  const TI* s = x + m * ldx;
  int8_t* d = q + m * ldq;
  Vec16<TI> v[NR];
  float mx = 0.f;
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i].load(s, (i * T + tid) * V, K);
#pragma unroll
    for (int i = 0; i < NV; ++i) mx = v[i].max(mx);
  } else {
    for (int c = tid * V; c < K; c += T * V) {
      v[0].load(s, c, K);
      mx = v[0].max(mx);
    }
  }
  mx = wave_max_abs(mx);
  if constexpr (T == 256) {
    if ((tid & 63) == 0) buf[tid >> 6] = mx;
    __syncthreads();
    mx = max_abs(max_abs(max_abs(buf[0], buf[1]), buf[2]), buf[3]);
  }
  const Quant to(mx);
  if (tid == 0) scale[m] = to.scale;
  auto store = [&](int c, const Vec16<TI>& o) {
    if (c >= Kq) return;   // Kq is a multiple of V
    uint32_t w[V / 4];
    quantize(to, o.v, w);
    __builtin_memcpy(d + c, w, V);
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) store((i * T + tid) * V, v[i]);
  } else {
    for (int c = tid * V; c < Kq; c += T * V) {
      v[0].load(s, c, K);
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
  else if (Kq <= 4 * 256 * V) launch(INT(256), INT(4));
  else launch(INT(256), INT(0));
#undef INT
}
template void int8_quantize<float>(const float*, int64_t, int64_t, int32_t, int8_t*, int64_t, int32_t, float*, hipStream_t);
template void int8_quantize<bf16>(const bf16*, int64_t, int64_t, int32_t, int8_t*, int64_t, int32_t, float*, hipStream_t);

// ---------------------------------------------------------------------------
// The product.
// ---------------------------------------------------------------------------
struct Int8P {
  const int8_t *x, *w;
  int64_t ldx, ldw, ldy, M, N;   // M tokens, N channels
  int K;
  const float *xs, *ws, *bias;
  void* y;
  // tiles
  int ntm, ntn, gm, total;
};

// Four channels of a token, from n on.
template <typename TO>
__device__ __forceinline__ void put4(const Int8P& p, int64_t m, int64_t n, i32x4 a, float xs) {
  if (m >= p.M || n >= p.N) return;
  TO* y = (TO*)p.y + m * p.ldy + n;
  TO o[4];
  if (n + 4 <= p.N) {
    float w[4], b[4] = {0.f, 0.f, 0.f, 0.f};
    __builtin_memcpy(w, p.ws + n, 16);
    if (p.bias) __builtin_memcpy(b, p.bias + n, 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = from_f32<TO>(int8_value(a[j], scale_of(xs, w[j]), b[j]));
    __builtin_memcpy(y, o, sizeof o);
  } else {
    for (int j = 0; j < 4 && n + j < p.N; ++j)
      y[j] = from_f32<TO>(int8_value(a[j], scale_of(xs, p.ws[n + j]), p.bias ? p.bias[n + j] : 0.f));
  }
}

// 128-byte rows of 8 chunks in LDS, chunk c of row r in slot kc_slot<64>(c, r).
template <int ROWS, int NW>
__device__ __forceinline__ void stage(const int8_t* base, int64_t ld, int64_t rows, int k0, int K, char* tile, int wid,
                                      int lane) {
  const __amdgpu_buffer_rsrc_t r = dma_rsrc(base);
  constexpr int LOADS = ROWS / 8 / NW;
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = (i * NW + wid) * 8 + lane / 8;
    const int k = k0 + kc_slot<64>(lane % 8, row) * 16;
    dma16(r, row < rows && k < K ? (uint32_t)(row * ld + k) : DMA_OFF_NONE, tile + (i * NW + wid) * 1024);
  }
}

// BM channels x BN tokens a workgroup of WM x WN waves, 128 k at a time, two stages.
template <typename TO, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void int8_tile_kernel(const Int8P p) {
  constexpr int NW = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16, STAGE = (BM + BN) * 128;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, wm = wid % WM, wn = wid / WM;
  int z, tm, tn;
  kc_tile_of(p, blockIdx.x, p.gm, z, tm, tn);
  const int64_t n0 = (int64_t)tm * BM, m0 = (int64_t)tn * BN;
  const int steps = (p.K + 127) / 128;
  const int8_t *wb = p.w + n0 * p.ldw, *xb = p.x + m0 * p.ldx;
  auto issue = [&](int j) {
    char* st = lds + (j & 1) * STAGE;
    stage<BM, NW>(wb, p.ldw, p.N - n0, j * 128, p.K, st, wid, lane);
    stage<BN, NW>(xb, p.ldx, p.M - m0, j * 128, p.K, st + BM * 128, wid, lane);
  };
  i32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const int fr = lane & 15, fc = lane >> 4;
  issue(0);
  for (int it = 0; it < steps; ++it) {
    int8_stage_wait();
    kc_barrier();
    if (it + 1 < steps) issue(it + 1);
    const char* st = lds + (it & 1) * STAGE;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      i32x4 a[FM], b[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i)
        a[i] = *(const i32x4*)(st + (wm * (BM / WM) + i * 16 + fr) * 128 + kc_slot<64>(ks * 4 + fc, fr) * 16);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        b[j] = *(const i32x4*)(st + BM * 128 + (wn * (BN / WN) + j * 16 + fr) * 128 + kc_slot<64>(ks * 4 + fc, fr) * 16);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mma_i8(a[i], b[j], acc[i][j]);
    }
  }
  float xs[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) xs[j] = p.xs[min(m0 + wn * (BN / WN) + j * 16 + fr, p.M - 1)];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      put4<TO>(p, m0 + wn * (BN / WN) + j * 16 + fr, n0 + wm * (BM / WM) + i * 16 + 4 * fc, acc[i][j], xs[j]);
}

// Few tokens: 16 channels and up to 16 FN tokens a workgroup, whose four waves
// each take every fourth 64 of K, both operands straight from memory.
template <typename TO, int FN>
__global__ __launch_bounds__(256) void int8_few_kernel(const Int8P p) {
  __shared__ i32x4 part[3][FN][64];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, fr = lane & 15, fc = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * 16 * FN;
  const int8_t* wr = p.w + min(n0 + fr, p.N - 1) * p.ldw;   // rows past the last: any, dropped at the end
  const int8_t* xr[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) xr[j] = p.x + min(m0 + j * 16 + fr, p.M - 1) * p.ldx;
  i32x4 acc[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) acc[j] = i32x4{0, 0, 0, 0};
#pragma unroll 4
  for (int k = wid * 64 + fc * 16; k < p.K + fc * 16; k += 256) {
    const bool in = k < p.K;   // both operands zero behind K
    const i32x4 a = in ? *(const i32x4*)(wr + k) : i32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const i32x4 b = in ? *(const i32x4*)(xr[j] + k) : i32x4{0, 0, 0, 0};
      acc[j] = mma_i8(a, b, acc[j]);
    }
  }
  if (wid > 0) {
#pragma unroll
    for (int j = 0; j < FN; ++j) part[wid - 1][j][lane] = acc[j];
  }
  __syncthreads();
  if (wid > 0) return;
#pragma unroll
  for (int j = 0; j < FN; ++j)
    put4<TO>(p, m0 + j * 16 + fr, n0 + 4 * fc, acc[j] + part[0][j][lane] + part[1][j][lane] + part[2][j][lane],
             p.xs[min(m0 + j * 16 + fr, p.M - 1)]);
}

// The same for up to 16 tokens of floats (TO, also y's), quantised on the way by every workgroup for itself while its
// weights are in flight.
struct Int8FewP {
  Int8P p;
  const void* x;
  int64_t ldx;
  int K, cols;   // columns of x, p.K those of the weights; in LDS
};
static constexpr int FEW_COLS = 4096;   // of 16 tokens in LDS
template <typename TO, int NV>
__global__ __launch_bounds__(256) void int8_few_tokens_kernel(const Int8FewP a) {
  const Int8P& p = a.p;
  constexpr int U = 4;
  extern __shared__ __attribute__((aligned(16))) char tokens[];
  __shared__ i32x4 part[3][64];
  __shared__ float xs[16];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, fr = lane & 15, fc = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int8_t* wr = p.w + min(n0 + fr, p.N - 1) * p.ldw;   // rows past the last: any, dropped at the end
  const int k0 = wid * 64 + fc * 16;
  auto weights = [&](int k) { return k < p.K ? *(const i32x4*)(wr + k) : i32x4{0, 0, 0, 0}; };
  i32x4 w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) w[u] = weights(k0 + u * 256);
  tokens_to_lds<TO, NV < 8 ? 8 / NV : 1, NV>((const TO*)a.x, a.ldx, (int)p.M, a.K, a.cols, tokens, xs);
  __syncthreads();
  const char* xr = tokens + (fr < p.M ? fr : 0) * (a.cols + 16);   // columns past the last token: any
  i32x4 acc{0, 0, 0, 0};
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (wid * 64 + u * 256 < a.cols) acc = mma_i8(w[u], *(const i32x4*)(xr + k0 + u * 256), acc);
#pragma unroll 4
  for (int k = wid * 64 + U * 256; k < a.cols; k += 256) acc = mma_i8(weights(k + fc * 16), *(const i32x4*)(xr + k + fc * 16), acc);
  if (wid > 0) part[wid - 1][lane] = acc;
  __syncthreads();
  if (wid > 0) return;
  put4<TO>(p, fr, n0 + 4 * fc, acc + part[0][lane] + part[1][lane] + part[2][lane], xs[fr]);
}
template <typename TO>
static void few_tokens(Int8FewP a, hipStream_t s) {
  constexpr int V = Vec16<TO>::n;
  a.cols = (int)rup(a.p.K, 64);
  const size_t bytes = 16 * (size_t)(a.cols + 16);
  auto launch = [&](auto nv) {
    auto fn = int8_few_tokens_kernel<TO, decltype(nv)::value>;
    static std::atomic<uint64_t> raised{0};
    kc_raise_lds_limit((const void*)fn, 16 * (FEW_COLS + 16), raised);
    BLSTM_LAUNCH("int8_linear_few", fn, dim3((unsigned)cdiv(a.p.N, 16)), dim3(256), bytes, s, a);
  };
#define INT(n) std::integral_constant<int, n>{}
  if (a.cols <= 64 * V) launch(INT(1));
  else if (a.cols <= 2 * 64 * V) launch(INT(2));
  else if (a.cols <= 4 * 64 * V) launch(INT(4));
  else if (a.cols <= 8 * 64 * V) launch(INT(8));
  else launch(INT(FEW_COLS / (64 * V)));
#undef INT
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
  auto tile = [&](auto bm, auto bn, auto wm, auto wn) {
    constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value, WM = decltype(wm)::value, WN = decltype(wn)::value;
    constexpr size_t bytes = 2 * (BM + BN) * 128;
    auto fn = int8_tile_kernel<TO, BM, BN, WM, WN>;
    static std::atomic<uint64_t> raised{0};
    kc_raise_lds_limit((const void*)fn, bytes, raised);
    p.ntm = (int)cdiv(p.N, BM);
    p.ntn = (int)cdiv(p.M, BN);
    p.gm = kc_group_rows;
    p.total = p.ntm * p.ntn;
    BLSTM_LAUNCH("int8_linear", fn, dim3((unsigned)p.total), dim3(WM * WN * 64), bytes, s, p);
  };
#define INT(n) std::integral_constant<int, n>{}
  if (cdiv(p.M, 256) * cdiv(p.N, 256) >= 256) tile(INT(256), INT(256), INT(2), INT(4));
  else tile(INT(128), INT(128), INT(2), INT(4));
#undef INT
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
  if (M <= 16 && Kw <= FEW_COLS) {
    Int8FewP a{};
    a.p.w = w; a.p.ldw = ldw; a.p.ldy = ldy; a.p.M = M; a.p.N = N; a.p.K = Kw; a.p.ws = w_scale; a.p.bias = bias; a.p.y = y;
    a.x = x; a.ldx = ldx; a.K = K;
    if (precision == BLSTM_BF16) few_tokens<bf16>(a, stream);
    else few_tokens<float>(a, stream);
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
static int64_t logit_rows(int64_t M, int64_t K) { return std::min(M, std::max<int64_t>(64, (180 << 20) / (4 * rup(K, 4)))); }

extern "C" int int8_logprob_ws_bytes(int64_t M, int32_t K, int32_t Kw, size_t* bytes) {
  const int rc = check_sizes("int8_logprob_ws_bytes", M, K, Kw);
  if (rc) return rc;
  if (K > SOFTMAX_MAX_CLASSES || Kw > INT8_MAX_K) return blstm_fail(BLSTM_EUNSUPPORTED, "int8_logprob_ws_bytes: too many classes or columns");
  if (bytes)
    *bytes = int8_head_fits(Kw) ? int8_head_bytes(M, K, (int32_t)rup(Kw, 16))
                                : tokens_bytes(M, rup(Kw, 16)) + (size_t)logit_rows(M, K) * rup(K, 4) * 4;
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
  if (int8_head_fits(Kw))
    return precision == BLSTM_BF16
               ? int8_head((const bf16*)x, ldx, M, P, w, ldw, w_scale, K, Kw, bias, *scores, (char*)ws, stream)
               : int8_head((const float*)x, ldx, M, P, w, ldw, w_scale, K, Kw, bias, *scores, (char*)ws, stream);
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
