// Short causal convolution of the state space block, per channel:
//   pre[t] = bias + sum_j w[j] x[t - W + 1 + j],  y = silu(pre) or pre
//   dpre = dy silu'(pre),  dx[i] = sum_j w[j] dpre[i + W - 1 - j]
//   dw[j] = sum_t dpre[t] x[t - W + 1 + j],  dbias = sum_t dpre[t]
// A thread has SEG frames of one sequence and four adjacent channels: it
// issues every load (the W - 1 frames on either side among them, which
// neighbours read too and the caches serve) before it computes, so one trip to memory is all that
// it waits for.  (Frame after frame, 128 chunks of 21 frames of 1024 channels: forward
// 9.7 us, backward 17.)  The backward computes dpre of W - 1 frames again in
// each stretch, and still shorter ones, which are more waves at a time, cost less there: 8
// frames 72, 4 frames 62 us at 16 sequences of 1500; the forward 28.3, 31.1 at 1024 of 21.
// Memory bounds both at length (1024 chunks of 21 frames: forward 28 us, 3.1 TB/s, backward 52
// us, 2.5 TB/s, with three waves a SIMD to hide the loads); 128 chunks, 7 + 12 + 3 us, are one trip
// to memory, the arithmetic behind it and the launches.
#include "ssm.hpp"

static constexpr int SEG = 8, BSEG = 4;   // frames of a thread, forward and backward

struct ConvP {
  const void *x, *dy, *state, *dsto;
  int64_t ldx, lddy, ldy, lddx;
  const float *w, *bias;
  const int32_t* lens;
  void *y, *sto, *dx, *dstate;
  float* part;   // [row blocks][W + 1][D]: dw by taps, then dbias
  int T, B, D, C4, nseg, silu;
  bool vx, vdy, vy, vdx, vs, vw;   // 4-wide accesses possible (vs: state rows, vw: weights)
  int tx, ncb;   // forward: threads along the channels, workgroups along them
};

__device__ __forceinline__ int conv_len(const ConvP& p, int b) {
  return p.lens ? max(0, min(p.T, p.lens[b])) : p.T;
}
// Input i of sequence b as it lies in memory (i < 0: from the state before the
// first frame), zeros where there is none.
template <typename T, int W>
__device__ __forceinline__ typename Vec4<T>::type conv_input(const ConvP& p, int i, int b, int len, int c, int nv) {
  typename Vec4<T>::type z{};
  if (i >= 0 && i < len) return ld4_raw((const T*)p.x + ((int64_t)i * p.B + b) * p.ldx + c, nv, p.vx);
  if (i < 0 && i >= 1 - W && p.state)
    return ld4_raw((const T*)p.state + ((int64_t)b * (W - 1) + W - 1 + i) * p.D + c, nv, p.vs);
  return z;
}
template <int W>
__device__ __forceinline__ void conv_weights(const ConvP& p, int c, int nv, f32x4* w, f32x4& bias) {
  bias = f32x4{0.f, 0.f, 0.f, 0.f};
  if (p.vw && nv >= 4) {   // the four channels' taps are adjacent
    f32x4 raw[W];
#pragma unroll
    for (int j = 0; j < W; ++j) raw[j] = *(const f32x4*)(p.w + (int64_t)c * W + 4 * j);
    if (p.bias) bias = *(const f32x4*)(p.bias + c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][i] = raw[(i * W + j) / 4][(i * W + j) % 4];
    return;
  }
#pragma unroll
  for (int j = 0; j < W; ++j) w[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < nv; ++i) {
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][i] = p.w[(int64_t)(c + i) * W + j];
    if (p.bias) bias[i] = p.bias[c + i];
  }
}

template <typename T, int W>
__global__ __launch_bounds__(256) void ssm_conv_fwd_kernel(const ConvP p) {
  const unsigned tx = (unsigned)p.tx, ncb = (unsigned)p.ncb;   // tx: a power of two
  const int c = (int)((blockIdx.x % ncb) * tx + (threadIdx.x & (tx - 1))) * 4;
  const unsigned r = blockIdx.x / ncb * (256u / tx) + threadIdx.x / tx;   // at most T * B of them
  const int b = (int)(r % (unsigned)p.B), sg = (int)(r / (unsigned)p.B);
  if (sg >= p.nseg || c >= p.D) return;
  const int nv = min(4, p.D - c), len = conv_len(p, b);
  const int t0 = sg * SEG;
  typename Vec4<T>::type in[SEG + W - 1], last[W > 1 ? W - 1 : 1];
#pragma unroll
  for (int j = 0; j < SEG + W - 1; ++j) in[j] = conv_input<T, W>(p, t0 - W + 1 + j, b, len, c, nv);
  const bool ends = p.sto && sg == 0;
  if (ends) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) last[j] = conv_input<T, W>(p, len - W + 1 + j, b, len, c, nv);
  }
  f32x4 w[W], bias;
  conv_weights<W>(p, c, nv, w, bias);
#pragma unroll
  for (int t = 0; t < SEG; ++t) {
    if (t0 + t >= p.T) break;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    if (t0 + t < len) {
      o = bias;
#pragma unroll
      for (int j = 0; j < W; ++j) o += w[j] * widen(in[t + j]);
      if (p.silu) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = siluf_(o[i]);
      }
    }
    st4((T*)p.y + ((int64_t)(t0 + t) * p.B + b) * p.ldy + c, o, nv, p.vy);
  }
  if (ends) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) st4((T*)p.sto + ((int64_t)b * (W - 1) + j) * p.D + c, widen(last[j]), nv, p.vs);
  }
}

// 64 threads a row of 256 channels, 4 rows a workgroup; a row takes every
// gridDim.y * 4-th stretch of BSEG frames.  There are as many workgroups as run at
// a time, so that none waits behind the others and the partial sums are few.
// workgroups of a CU: what the registers hold (but for 6 that float32 with 8 taps spills)
static constexpr int conv_resident(int W) { return W <= 4 ? 3 : 2; }
template <typename T, int W>
__global__ __launch_bounds__(256, conv_resident(W)) void ssm_conv_bwd_kernel(const ConvP p) {
  const int cl = threadIdx.x & 63, rl = threadIdx.x >> 6;
  const int c = ((int)blockIdx.x * 64 + cl) * 4, nv = min(4, p.D - c);
  f32x4 w[W], bias, dw[W], db{0.f, 0.f, 0.f, 0.f};
  conv_weights<W>(p, c, nv, w, bias);
#pragma unroll
  for (int j = 0; j < W; ++j) dw[j] = db;
  const int items = p.nseg * p.B;   // at most T * B
  for (int it = (int)blockIdx.y * 4 + rl; it < items && nv > 0; it += (int)gridDim.y * 4) {
    const int b = (int)((unsigned)it % (unsigned)p.B), t0 = (int)((unsigned)it / (unsigned)p.B) * BSEG, t1 = min(p.T, t0 + BSEG);
    const int len = conv_len(p, b);
    // inputs t0 - W + 1 .. t0 + BSEG + W - 2, gradients t0 .. t0 + BSEG + W - 2
    typename Vec4<T>::type in[BSEG + 2 * W - 2], gy[BSEG + W - 1];
#pragma unroll
    for (int j = 0; j < BSEG + 2 * W - 2; ++j) in[j] = conv_input<T, W>(p, t0 - W + 1 + j, b, len, c, nv);
#pragma unroll
    for (int j = 0; j < BSEG + W - 1; ++j) {
      gy[j] = typename Vec4<T>::type{};
      if (t0 + j < len) gy[j] = ld4_raw((const T*)p.dy + ((int64_t)(t0 + j) * p.B + b) * p.lddy + c, nv, p.vdy);
    }
    f32x4 dp[W];   // the last W dpre, oldest first
#pragma unroll
    for (int j = 0; j < W; ++j) dp[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < BSEG + W - 1; ++t) {
#pragma unroll
      for (int j = 0; j < W - 1; ++j) dp[j] = dp[j + 1];
      f32x4 g = widen(gy[t]);   // zero behind the end
      if (p.silu) {
        f32x4 pre = bias;
#pragma unroll
        for (int j = 0; j < W; ++j) pre += w[j] * widen(in[t + j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] *= dsiluf_(pre[i]);
      }
      if (t0 + t >= len) g = f32x4{0.f, 0.f, 0.f, 0.f};
      if (t < BSEG) {
        db += g;
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j] += g * widen(in[t + j]);
      }
      dp[W - 1] = g;
      // input i is complete: every frame that it meets has passed
      const int i = t0 + t - W + 1;
      if ((t < W - 1 && t0 > 0) || i >= t1) continue;
      f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < W; ++j) o += w[j] * dp[W - 1 - j];
      if (p.dsto && i < len && i >= len - W + 1)
        o += widen(ld4_raw((const T*)p.dsto + ((int64_t)b * (W - 1) + i - (len - W + 1)) * p.D + c, nv, p.vs));
      if (i >= 0) st4((T*)p.dx + ((int64_t)i * p.B + b) * p.lddx + c, o, nv, p.vdx);
      else if (p.dstate) st4((T*)p.dstate + ((int64_t)b * (W - 1) + W - 1 + i) * p.D + c, o, nv, p.vs);
    }
  }
  __shared__ f32x4 sh[4][64];
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    sh[rl][cl] = j < W ? dw[j] : db;
    __syncthreads();
    if (rl == 0) {
      const f32x4 v = ((sh[0][cl] + sh[1][cl]) + sh[2][cl]) + sh[3][cl];
      for (int i = 0; i < nv; ++i) p.part[((int64_t)blockIdx.y * (W + 1) + j) * p.D + c + i] = v[i];
    }
    __syncthreads();
  }
}

// dw [D][W] and dbias [D]: the row blocks' sums, 16 ranges in order.
__global__ __launch_bounds__(256) void ssm_conv_sum_kernel(const float* __restrict__ part, int rows, int D, int W,
                                                           float* __restrict__ dw, float* __restrict__ dbias) {
  __shared__ float sh[16][17];
  const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int64_t cols = (int64_t)(W + 1) * D, c = (int64_t)blockIdx.x * 16 + cl;
  const int per = (rows + 15) / 16, r0 = rg * per, r1 = min(rows, r0 + per);
  float v = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int r = r0; r < r1; ++r) v += part[r * cols + c];
  }
  sh[rg][cl] = v;
  __syncthreads();
  if (rg || c >= cols) return;
  float t = 0.f;
  for (int i = 0; i < 16; ++i) t += sh[i][cl];
  const int j = (int)(c / D), d = (int)(c % D);
  if (j < W) dw[(int64_t)d * W + j] = t;
  else if (dbias) dbias[d] = t;
}

template <typename T, int W>
__global__ __launch_bounds__(256) void ssm_conv_step_kernel(const ConvP p, const int32_t* __restrict__ slots,
                                                            int n_slots, T* state) {
  const int tiles = (p.C4 + 255) / 256;
  const int b = (int)(blockIdx.x / (unsigned)tiles);
  const int c = ((int)(blockIdx.x % (unsigned)tiles) * 256 + (int)threadIdx.x) * 4;
  __shared__ int taken;
  int slot = b;
  if (slots) {
    slot = slots[b];
    if (threadIdx.x == 0) taken = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < b; i += 256)
      if (slots[i] == slot) taken = 1;   // every writer writes the same
    __syncthreads();
    if (taken || slot < 0 || slot >= n_slots) slot = -1;
  }
  const int nv = min(4, p.D - c);
  if (nv <= 0) return;
  f32x4 o{0.f, 0.f, 0.f, 0.f};
  if (slot >= 0) {
    f32x4 w[W], win[W];
    conv_weights<W>(p, c, nv, w, o);
    T* s = state + (int64_t)slot * (W - 1) * p.D + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j] = widen(ld4_raw(s + (int64_t)j * p.D, nv, p.vs));
    win[W - 1] = widen(ld4_raw((const T*)p.x + (int64_t)b * p.ldx + c, nv, p.vx));
#pragma unroll
    for (int j = 0; j < W; ++j) o += w[j] * win[j];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) st4(s + (int64_t)j * p.D, win[j + 1], nv, p.vs);
    if (p.silu) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = siluf_(o[i]);
    }
  }
  st4((T*)p.y + (int64_t)b * p.ldy + c, o, nv, p.vy);
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// Row blocks of the backward, on 256 CUs.  (16 sequences of 1500 frames of 1024 channels, bf16,
// 4 taps: 512 workgroups 62, 768 53, 1024 62 us; 8 taps, two a CU: 512 best.)
static int conv_rows(const ssm_dims* d) {
  const int64_t items = cdiv(d->T, BSEG) * d->B, most = 256 * conv_resident(d->W) / cdiv(d->D, 256);
  return (int)std::min(std::max<int64_t>(1, most), cdiv(items, 4));
}
size_t ssm_conv_bwd_bytes(const ssm_dims* d) { return (size_t)conv_rows(d) * (d->W + 1) * d->D * 4; }

static bool four(const void* p, int64_t ld, size_t es) { return ((uintptr_t)p % (4 * es)) == 0 && ld % 4 == 0; }

static int conv_args(const ssm_dims* d, const char* fn, const void* x, int64_t ldx, const float* w, const float* bias,
                     const int32_t* lens, const void* state, uint32_t flags, ConvP* p) {
  int rc = ssm_check_dims(d, fn);
  if (rc) return rc;
  if (!x || !w) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (flags & ~(uint32_t)SSM_SILU) return blstm_fail(BLSTM_EINVAL, "%s: unknown flags", fn);
  if (ldx < d->D) return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  const size_t es = d->precision == BLSTM_BF16 ? 2 : 4;
  *p = ConvP{};
  p->x = x; p->ldx = ldx; p->w = w; p->bias = bias; p->lens = lens; p->state = state;
  p->T = d->T; p->B = d->B; p->D = d->D; p->C4 = (int)cdiv(d->D, 4);
  p->nseg = (int)cdiv(d->T, SEG);
  p->silu = flags & SSM_SILU;
  p->vw = (uintptr_t)w % 16 == 0 && (uintptr_t)bias % 16 == 0;
  p->vx = four(x, ldx, es);
  p->vs = d->D % 4 == 0 && ((uintptr_t)state % (4 * es)) == 0;
  return BLSTM_OK;
}

#define CONV_BY_TAPS(T, LAUNCH)        \
  switch (dims->W) {                   \
    case 1: LAUNCH(T, 1); break;       \
    case 2: LAUNCH(T, 2); break;       \
    case 3: LAUNCH(T, 3); break;       \
    case 4: LAUNCH(T, 4); break;       \
    case 5: LAUNCH(T, 5); break;       \
    case 6: LAUNCH(T, 6); break;       \
    case 7: LAUNCH(T, 7); break;       \
    default: LAUNCH(T, 8); break;      \
  }
#define CONV_DISPATCH(LAUNCH)                                       \
  if (dims->precision == BLSTM_BF16) { CONV_BY_TAPS(bf16, LAUNCH) } \
  else { CONV_BY_TAPS(float, LAUNCH) }

extern "C" int ssm_conv_fwd(const ssm_dims* dims, const void* x, int64_t ldx, const float* w, const float* bias,
                            const int32_t* lens, const void* state, void* y, int64_t ldy, void* state_out,
                            uint32_t flags, hipStream_t stream) {
  ConvP p;
  int rc = conv_args(dims, "ssm_conv_fwd", x, ldx, w, bias, lens, state, flags, &p);
  if (rc) return rc;
  if (!y) return blstm_fail(BLSTM_EINVAL, "ssm_conv_fwd: NULL pointer");
  if (ldy < dims->D) return blstm_fail(BLSTM_EINVAL, "ssm_conv_fwd: a row pitch is below its row");
  if (state_out && state_out == state) return blstm_fail(BLSTM_EINVAL, "ssm_conv_fwd: state_out is state");
  const size_t es = dims->precision == BLSTM_BF16 ? 2 : 4;
  p.y = y; p.ldy = ldy; p.sto = state_out;
  p.vy = four(y, ldy, es);
  p.vs = p.vs && ((uintptr_t)state_out % (4 * es)) == 0;
  p.tx = 1;
  while (p.tx < 256 && p.tx < p.C4) p.tx *= 2;
  p.ncb = (int)cdiv(p.C4, p.tx);
  const int64_t blocks = cdiv((int64_t)p.B * p.nseg, 256 / p.tx) * p.ncb;
  if (blocks * 256 > LAUNCH_THREADS) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_conv_fwd: T*B*D too large");
#define FWD(T, W) \
  BLSTM_LAUNCH("ssm_conv_fwd", (ssm_conv_fwd_kernel<T, W>), dim3((unsigned)blocks), dim3(256), 0, stream, p)
  CONV_DISPATCH(FWD)
  return blstm_check_launch("ssm_conv_fwd");
}

extern "C" int ssm_conv_bwd(const ssm_dims* dims, const void* x, int64_t ldx, const float* w, const float* bias,
                            const int32_t* lens, const void* state, const void* dy, int64_t lddy,
                            const void* dstate_out, void* dx, int64_t lddx, float* dw, float* dbias, void* dstate,
                            void* ws, uint32_t flags, hipStream_t stream) {
  ConvP p;
  int rc = conv_args(dims, "ssm_conv_bwd", x, ldx, w, bias, lens, state, flags, &p);
  if (rc) return rc;
  if (!dy || !dx || !dw || !ws) return blstm_fail(BLSTM_EINVAL, "ssm_conv_bwd: NULL pointer");
  if (lddy < dims->D || lddx < dims->D) return blstm_fail(BLSTM_EINVAL, "ssm_conv_bwd: a row pitch is below its row");
  const size_t es = dims->precision == BLSTM_BF16 ? 2 : 4;
  p.dy = dy; p.lddy = lddy; p.dsto = dstate_out; p.dx = dx; p.lddx = lddx; p.dstate = dstate; p.part = (float*)ws;
  p.vdy = four(dy, lddy, es);
  p.vdx = four(dx, lddx, es);
  p.vs = p.vs && ((uintptr_t)dstate_out % (4 * es)) == 0 && ((uintptr_t)dstate % (4 * es)) == 0;
  p.nseg = (int)cdiv(dims->T, BSEG);
  const int rows = conv_rows(dims);
#define BWD(T, W)                                                                                          \
  BLSTM_LAUNCH("ssm_conv_bwd", (ssm_conv_bwd_kernel<T, W>), dim3((unsigned)cdiv(p.C4, 64), (unsigned)rows), \
               dim3(256), 0, stream, p)
  CONV_DISPATCH(BWD)
  BLSTM_LAUNCH("ssm_conv_sum", ssm_conv_sum_kernel, dim3((unsigned)cdiv((int64_t)(dims->W + 1) * dims->D, 16)),
               dim3(256), 0, stream, (const float*)ws, rows, dims->D, dims->W, dw, dbias);
  return blstm_check_launch("ssm_conv_bwd");
}

extern "C" int ssm_conv_step(const ssm_dims* dims, const void* x, int64_t ldx, const float* w, const float* bias,
                             const int32_t* slots, int32_t n_slots, void* state, void* y, int64_t ldy, uint32_t flags,
                             hipStream_t stream) {
  ConvP p;
  int rc = conv_args(dims, "ssm_conv_step", x, ldx, w, bias, nullptr, state, flags, &p);
  if (rc) return rc;
  if (!y || (!state && dims->W > 1)) return blstm_fail(BLSTM_EINVAL, "ssm_conv_step: NULL pointer");
  if (dims->T != 1) return blstm_fail(BLSTM_EINVAL, "ssm_conv_step: T must be 1");
  if (n_slots < 1 || (!slots && n_slots < dims->B))
    return blstm_fail(BLSTM_EINVAL, "ssm_conv_step: %d slots for %d streams", n_slots, dims->B);
  if (ldy < dims->D) return blstm_fail(BLSTM_EINVAL, "ssm_conv_step: a row pitch is below its row");
  p.y = y; p.ldy = ldy;
  p.vy = four(y, ldy, dims->precision == BLSTM_BF16 ? 2 : 4);
  const int64_t blocks = (int64_t)dims->B * cdiv(p.C4, 256);
  if (blocks * 256 > LAUNCH_THREADS) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_conv_step: B*D too large");
#define STEP(T, W)                                                                                            \
  BLSTM_LAUNCH("ssm_conv_step", (ssm_conv_step_kernel<T, W>), dim3((unsigned)blocks), dim3(256), 0, stream, p, \
               slots, n_slots, (T*)state)
  CONV_DISPATCH(STEP)
  return blstm_check_launch("ssm_conv_step");
}
