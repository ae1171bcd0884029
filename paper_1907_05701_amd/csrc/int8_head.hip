// The 8-bit head: log probabilities without the logits in memory.
//
// Pass 1 multiplies a tile of frames with a range of classes and keeps, per
// frame and lane, the softmax sums so far and the largest logit of every group
// of classes that the lane sees.  Pass 2 joins a frame's sums; the few groups
// that reach the k-th largest of the groups' maxima hold its k most likely
// classes, whose logits it computes again, as it does the listed classes': sums
// of integers are exact, so these are the same bits.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "gemm_kc.hpp"
#include "int8.hpp"
#include "rows.hpp"
#include "score.hpp"

static constexpr int CT = 64;             // classes of a tile: one stage in LDS
static constexpr int PAIR = 2 * CT;       // classes over which group maxima are taken
static constexpr float FLOOR = -1e30f;    // sums start from here; logits below count as nothing (second pass)
static constexpr float SLACK = 30.f;      // how far above its reference a lane's largest exponent may get

struct HeadP {
  const int8_t *q, *w;
  int64_t ldw;
  const float *xs, *ws, *bias;
  int64_t M;
  int K, Kw, ksteps;       // classes, columns, 64-column steps
  int nf, ranges, ppr;     // frame tiles, class ranges, pairs of tiles a range
  int nstat, ngroup;       // a frame's sums and group maxima
  float it2, itau;         // log2 e / tau, 1 / tau
  float4* stats;           // [M][nstat]: reference (an exponent of 2), Z, T
  float* gmax;             // [M][ngroup], or null
};

// Sums from a reference exponent: z = sum 2^(y - rc), t = sum 2^(y - rc) (y - rc).
struct Sums {
  float rc, z, t;
  __device__ __forceinline__ void rise(float to) {   // to >= rc
    const float d = to - rc, f = exp2_(-d);
    t = f * (t - d * z);
    z *= f;
    rc = to;
  }
  __device__ __forceinline__ void join(Sums o) {
    const float to = fmaxf(rc, o.rc);
    rise(to);
    o.rise(to);
    z += o.z;
    t += o.t;
  }
};

// 16-byte chunk c of row r of a tile of NCH chunks a row: the slot it lies in (16 rows' chunk c in 16 different
// bank groups).
template <int NCH>
__device__ __forceinline__ int head_slot(int c, int r) {
  return c ^ (NCH >= 16 ? r & 15 : (r * NCH / 16) & (NCH - 1));
}

// KS: most 64-column steps; 16 FN frames a wave; FW waves side by side along the
// frames, the other 4 / FW along the classes of a tile.
template <int KS, int FN, int FW>
__global__ __launch_bounds__(256, KS > 8 ? 1 : 2) void int8_head_kernel(const HeadP p) {
  constexpr int WC = 4 / FW, NI = 4 / WC, NCH = KS * 4, TILE = CT * KS * 64, STAGE = TILE + 512;
  constexpr int LOADS = TILE / 1024 / 4;   // of a wave
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fc = lane >> 4;
  const int wf = wid % FW, wc = wid / FW;
  // workgroup w runs on XCD w % 8: each takes a run of ranges, whose weights its L2 then holds
  const int total = p.nf * p.ranges, share = total / 8;
  const int at = (int)blockIdx.x < 8 * share ? blockIdx.x % 8 * share + blockIdx.x / 8 : blockIdx.x, range = at / p.nf;
  const int64_t f0 = (int64_t)(at % p.nf) * (16 * FN * FW) + wf * 16 * FN;
  const int tile0 = range * p.ppr * 2, tiles = min((int)((p.K + CT - 1) / CT) - tile0, p.ppr * 2);
  const int8_t* wb = p.w + (int64_t)tile0 * CT * p.ldw;
  const int rows = p.K - tile0 * CT;   // classes from the range's first on

  const __amdgpu_buffer_rsrc_t rws = __builtin_amdgcn_make_buffer_rsrc((void*)(p.ws + tile0 * CT), (short)0, rows * 4, 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc((void*)(p.bias + (p.bias ? tile0 * CT : 0)), (short)0,
                                                                     p.bias ? rows * 4 : 0, 0x00020000);
  auto issue = [&](int j) {
    char* st = lds + (j & 1) * STAGE;
    const __amdgpu_buffer_rsrc_t r = dma_rsrc(wb + (int64_t)j * CT * p.ldw);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int pos = (i * 4 + wid) * 64 + lane, row = pos / NCH, c = head_slot<NCH>(pos % NCH, row);
      const bool in = j * CT + row < rows && c * 16 < p.Kw;
      dma16(r, in ? (uint32_t)(row * p.ldw + c * 16) : DMA_OFF_NONE, st + (i * 4 + wid) * 1024);
    }
    // scales and biases, 64 of each (0 behind the last class)
    if (wid < 2)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wid ? rb : rws, (lds_ptr_t)(st + TILE + wid * 256), 4, (j * CT + lane) * 4, 0, 0, 0);
  };
  issue(0);

  i32x4 b[FN][KS];
  float xs[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int64_t f = min(f0 + j * 16 + fr, p.M - 1);   // frames past the last: any, not stored
    xs[j] = p.xs[f];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int k = ks * 64 + fc * 16;
      b[j][ks] = k < p.Kw ? *(const i32x4*)(p.q + f * p.Kw + k) : i32x4{0, 0, 0, 0};
    }
  }
  Sums s[FN];
  float lim[FN], gm[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    s[j] = Sums{FLOOR * p.it2, 0.f, 0.f};
    lim[j] = FLOOR;
    gm[j] = -INFINITY;
  }
  const float slack = SLACK / p.it2;

  for (int it = 0; it < tiles; ++it) {
    int8_stage_wait();
    kc_barrier();
    if (it + 1 < tiles) issue(it + 1);
    const char* st = lds + (it & 1) * STAGE;
    float l[NI][FN][4];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = (wc * NI + i) * 16;
      i32x4 acc[FN];
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[j] = i32x4{0, 0, 0, 0};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if (ks >= p.ksteps) continue;
        const i32x4 a = *(const i32x4*)(st + (row + fr) * (NCH * 16) + head_slot<NCH>(ks * 4 + fc, row + fr) * 16);
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[j] = mma_i8(a, b[j][ks], acc[j]);
      }
      const f32x4 w4 = *(const f32x4*)(st + TILE + (row + 4 * fc) * 4), b4 = *(const f32x4*)(st + TILE + 256 + (row + 4 * fc) * 4);
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) l[i][j][r] = int8_value(acc[j][r], scale_of(xs[j], w4[r]), b4[r]);
    }
    if ((it + 1) * CT > rows) {   // the last tile's classes past the last
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (it * CT + (wc * NI + i) * 16 + 4 * fc + r >= rows) {
#pragma unroll
            for (int j = 0; j < FN; ++j) l[i][j][r] = -INFINITY;
          }
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      float mb = l[0][j][0];
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) mb = fmaxf(mb, l[i][j][r]);
      if (__any(mb > lim[j])) {
        const float to = fmaxf(s[j].rc, mb * p.it2);
        s[j].rise(to);
        lim[j] = fmaxf(lim[j], mb + slack);
      }
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float y = fmaf(l[i][j][r], p.it2, -s[j].rc), e = exp2_(y);
          s[j].z += e;
          s[j].t += e * fmaxf(y, -200.f);
        }
      gm[j] = fmaxf(gm[j], mb);
      if (p.gmax && ((it & 1) || it + 1 == tiles)) {
        const int64_t f = f0 + j * 16 + fr;
        if (f < p.M) p.gmax[f * p.ngroup + ((tile0 + it) / 2 * WC + wc) * 4 + fc] = gm[j];
        gm[j] = -INFINITY;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < FN; ++j) {
#pragma unroll
    for (int o = 16; o < 64; o <<= 1)
      s[j].join(Sums{__shfl_xor(s[j].rc, o), __shfl_xor(s[j].z, o), __shfl_xor(s[j].t, o)});
    const int64_t f = f0 + j * 16 + fr;
    if (fc == 0 && f < p.M) p.stats[f * p.nstat + range * WC + wc] = float4{s[j].rc, s[j].z, s[j].t, 0.f};
  }
}

// ---------------------------------------------------------------------------
// Second pass: a workgroup a frame.
// ---------------------------------------------------------------------------
struct HeadOut {
  const int32_t* ids;
  float *logprob, *entropy, *top;
  int32_t* idx;
  int n, k, wc;   // wc: waves along the classes in the first pass
};
static constexpr int FT_ = 256;          // threads
static constexpr int GROUPS = 512;       // most groups computed again
static constexpr int WIDE = 64;          // largest k for threads' maxima

// A class's logit, the bits of the first pass.
struct Logit {
  const int8_t* w;
  int64_t ldw;
  const float *ws, *bias;
  const i32x4* x;   // the frame's integers, in LDS
  int chunks;
  float xs;
  __device__ __forceinline__ float operator()(int c) const {
    const i32x4* r = (const i32x4*)(w + c * ldw);
    int a = 0;
#pragma unroll 4
    for (int i = 0; i < chunks; ++i) {
      const i32x4 u = r[i], v = x[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) a = __builtin_amdgcn_sdot4(u[j], v[j], a, false);
    }
    return int8_value(a, scale_of(xs, ws[c]), bias ? bias[c] : 0.f);
  }
};

struct HeadLds {
  TopkLds<FT_> l;
  float buf[3][FT_ / 64];
  int32_t groups[GROUPS];
  uint32_t ngroups, hist[256], want;
};

// A log probability from joined sums.
struct HeadLogProb {
  float rc, l2z, it2, itau;
  __device__ __forceinline__ float operator()(float v) const {
    // far out the exponent could overflow, and what it is compared with does not count
    return fabsf(v) > 1e30f ? v * itau : (fmaf(v, it2, -rc) - l2z) * LN2_F;
  }
};

// Any row, its logits computed again in every pass: one with a NaN or infinities, with nothing
// above FLOOR, or with too many classes that reach the threshold.
__device__ __attribute__((noinline)) void head_any(HeadLds& h, const Logit& logit, const HeadP& p, const HeadOut& o, int64_t m) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K;
  float mx = -INFINITY;
  bool nan = false;
  for (int c = tid; c < K; c += FT_) {
    const float v = logit(c);
    mx = fmaxf(mx, v);
    nan |= v != v;
  }
  nan = __syncthreads_or(nan);
  mx = row_max<FT_>(fmaxf(mx, -INFINITY), h.buf[0]);
  const bool some = nan || !(mx == -INFINITY);
  const float ref = some ? mx : 0.f;
  float z = 0.f, t = 0.f;
  for (int c = tid; c < K; c += FT_) {
    const float y = (logit(c) - ref) * p.it2, e = exp2_(y);
    z += e;
    t += e * fmaxf(y, -200.f);
  }
  z = row_sum<FT_>(z, h.buf[1]);
  t = row_sum<FT_>(t, h.buf[2]);
  const float lz = log2f(z) * LN2_F;   // a NaN where there is one, or +inf
  auto value = [&](float v) { return some ? (v - ref) * p.itau - lz : -INFINITY; };
  if (tid < o.n) {
    const int at = o.ids[m * o.n + tid];
    o.logprob[m * o.n + tid] = at < 0 || at >= K ? 0.f : value(logit(at));
  }
  if (o.entropy && tid == 0) o.entropy[m] = some ? lz - t / z * LN2_F : 0.f;
  if (!o.k) return;
  // the k-th largest order word, eight bits at a time, and how many of its ties are taken
  uint32_t word = 0;
  int want = o.k;   // among the words that agree with `word` so far
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    h.hist[tid] = 0;
    __syncthreads();
    for (int c = tid; c < K; c += FT_) {
      const uint32_t u = order_word(logit(c));
      if (shift == 24 || (u >> (shift + 8)) == (word >> (shift + 8))) atomicAdd(&h.hist[(u >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid == 0) {
      int left = want, d = 255;
      for (; d > 0 && (int)h.hist[d] < left; --d) left -= (int)h.hist[d];
      h.want = (uint32_t)left | (uint32_t)d << 16;
    }
    __syncthreads();
    want = (int)(h.want & 0xffff);
    word |= (h.want >> 16) << shift;
  }
  // those above it, and the first `want` of those that equal it
  __syncthreads();
  if (tid == 0) h.l.count = 0;
  int taken = 0;
  for (int c0 = 0; c0 < K; c0 += FT_) {
    const int c = c0 + tid;
    const float v = c < K ? logit(c) : 0.f;
    const uint32_t u = c < K ? order_word(v) : 0;
    const uint64_t same_ = __ballot(c < K && u == word);
    __syncthreads();
    if (lane == 0) h.hist[wave] = __popcll(same_);
    __syncthreads();
    int before = taken;
    for (int i = 0; i < FT_ / 64; ++i) {
      if (i < wave) before += (int)h.hist[i];
      taken += (int)h.hist[i];
    }
    before += __popcll(same_ & ((1ull << lane) - 1));
    if (c < K && (u > word || (u == word && before < want))) push(h.l, v, c);
  }
  __syncthreads();
  TopkP tp{0, K, o.k, p.it2, o.top, nullptr, o.idx};
  rank(h.l, o.k, m, tp, value);
}

__global__ __launch_bounds__(FT_) void int8_head_finish_kernel(const HeadP p, const HeadOut o) {
  extern __shared__ __attribute__((aligned(16))) char xl[];
  __shared__ HeadLds h;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K;
  const int64_t m = blockIdx.x;
  for (int i = tid; i < p.Kw / 16; i += FT_) ((i32x4*)xl)[i] = ((const i32x4*)(p.q + m * p.Kw))[i];
  const Logit logit{p.w, p.ldw, p.ws, p.bias, (const i32x4*)xl, p.Kw / 16, p.xs[m]};
  // the sums, in a fixed order
  Sums s{FLOOR * p.it2, 0.f, 0.f};
  for (int i = tid; i < p.nstat; i += FT_) {
    const float4 v = p.stats[m * p.nstat + i];
    s.join(Sums{v.x, v.y, v.z});
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s.join(Sums{__shfl_xor(s.rc, off), __shfl_xor(s.z, off), __shfl_xor(s.t, off)});
  if (lane == 0) {
    h.buf[0][wave] = s.rc;
    h.buf[1][wave] = s.z;
    h.buf[2][wave] = s.t;
  }
  if (tid == 0) h.ngroups = h.l.count = 0;
  const float* gmax = p.gmax + m * p.ngroup;
  uint32_t mx = 0;
  if (o.k) {
    for (int g = tid; g < p.ngroup; g += FT_) mx = max(mx, order_word(gmax[g]));
    h.l.tmax[tid] = mx;
  }
  __syncthreads();
  s = Sums{h.buf[0][0], h.buf[1][0], h.buf[2][0]};
#pragma unroll
  for (int i = 1; i < FT_ / 64; ++i) s.join(Sums{h.buf[0][i], h.buf[1][i], h.buf[2][i]});
  // (a NaN fails both)
  if (same(!(s.z > 0.f && s.z < INFINITY))) {
    head_any(h, logit, p, o, m);
    return;
  }
  const HeadLogProb lp{s.rc, log2f(s.z), p.it2, p.itau};
  if (o.k) {
    uint32_t tw;
    if (o.k <= WIDE) {
      tw = kth_max<12, FT_>(h.l, o.k);
    } else {
      // over all groups, bit by bit
      tw = 0;
      for (int bit = 31; bit >= 12; --bit) {
        const uint32_t c = tw | (1u << bit);
        int n = 0;
        for (int g = tid; g < p.ngroup; g += FT_) n += order_word(gmax[g]) >= c;
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
        __syncthreads();
        if (lane == 0) h.hist[wave] = n;
        __syncthreads();
        n = 0;
        for (int i = 0; i < FT_ / 64; ++i) n += (int)h.hist[i];
        if (n >= o.k) tw = c;
      }
    }
    tw = max(tw, LOWEST);
    const float thr = order_value(tw);
    if (mx >= tw) {
      for (int g = tid; g < p.ngroup; g += FT_)
        if (gmax[g] >= thr) {
          const uint32_t at = atomicAdd(&h.ngroups, 1u);
          if (at < GROUPS) h.groups[at] = g;
        }
    }
    __syncthreads();
    const int ng = (int)same(h.ngroups), size = 32 / o.wc, ni = 4 / o.wc;
    if (ng > GROUPS) {
      head_any(h, logit, p, o, m);
      return;
    }
    for (int e = tid; e < ng * size; e += FT_) {
      const int g = h.groups[e / size], q = g % 4, w = g / 4 % o.wc, pair = g / 4 / o.wc;
      const int u = e % size / (4 * ni), i = e % (4 * ni) / 4, r = e % 4;
      const int c = pair * PAIR + u * CT + (w * ni + i) * 16 + 4 * q + r;
      if (c < K) {
        const float v = logit(c);
        if (v >= thr) push(h.l, v, c);
      }
    }
    __syncthreads();
    const int n = (int)same(h.l.count);
    if (n > CAND) {
      head_any(h, logit, p, o, m);
      return;
    }
    TopkP tp{0, K, o.k, p.it2, o.top, nullptr, o.idx};
    rank(h.l, n, m, tp, lp);
  }
  if (tid < o.n) {
    const int at = o.ids[m * o.n + tid];
    o.logprob[m * o.n + tid] = at < 0 || at >= K ? 0.f : lp(logit(at));
  }
  if (o.entropy && tid == 0) o.entropy[m] = (lp.l2z - s.t / s.z) * LN2_F;
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct HeadPlan {
  int fn, fw, ks;                 // frames / 16 of a wave, waves along the frames, column steps
  int nf, ranges, ppr, nstat, ngroup;
  size_t stats, gmax, bytes;      // behind the tokens
};
static constexpr int HEAD_MAX_STEPS = 16;

static HeadPlan head_plan(int64_t M, int32_t K, int32_t Kw) {
  HeadPlan h{};
  h.ks = (int)cdiv(Kw, 64);
  h.fn = h.ks > 8 ? 1 : 2;
  const int per = 16 * h.fn;
  h.fw = M <= per ? 1 : M <= 2 * per ? 2 : 4;
  h.nf = (int)cdiv(M, per * h.fw);
  const int64_t pairs = cdiv(K, PAIR), slots = h.ks > 8 ? 256 : 512;
  // as many ranges as take least: whole rounds of the chip, each as long as a range and its start
  int64_t best = -1;
  for (int64_t r = 1; r <= pairs && r <= std::max<int64_t>(1, 2 * slots / h.nf); ++r) {
    const int64_t ppr = cdiv(pairs, r), t = cdiv(cdiv(pairs, ppr) * h.nf, slots) * (2 * ppr + 1);
    if (best < 0 || t < best) {
      best = t;
      h.ppr = (int)ppr;
    }
  }
  h.ranges = (int)cdiv(pairs, h.ppr);
  const int wc = 4 / h.fw;
  h.nstat = h.ranges * wc;
  h.ngroup = (int)pairs * wc * 4;
  h.stats = 0;
  h.gmax = (size_t)rup(M * h.nstat * 16, 256);
  h.bytes = h.gmax + (size_t)rup(M * h.ngroup * 4, 256);
  return h;
}

bool int8_head_fits(int32_t Kw) { return cdiv(Kw, 64) <= HEAD_MAX_STEPS; }
size_t int8_head_bytes(int64_t M, int32_t K, int32_t Kw) { return head_plan(M, K, Kw).bytes; }

int int8_head(const int8_t* q, const float* xs, int64_t M, const int8_t* w, int64_t ldw, const float* ws, int32_t K,
              int32_t Kw, const float* bias, const softmax_scores& sc, char* buf, hipStream_t s) {
  const HeadPlan h = head_plan(M, K, Kw);
  HeadP p{};
  p.q = q; p.w = w; p.ldw = ldw; p.xs = xs; p.ws = ws; p.bias = bias; p.M = M; p.K = K; p.Kw = Kw; p.ksteps = h.ks;
  p.nf = h.nf; p.ranges = h.ranges; p.ppr = h.ppr; p.nstat = h.nstat; p.ngroup = h.ngroup;
  p.it2 = LOG2E_F / sc.temperature; p.itau = 1.f / sc.temperature;
  p.stats = (float4*)(buf + h.stats);
  p.gmax = sc.k ? (float*)(buf + h.gmax) : nullptr;
  auto launch = [&](auto ks, auto fn, auto fw) {
    constexpr int KS = decltype(ks)::value, FN = decltype(fn)::value, FW = decltype(fw)::value;
    constexpr size_t bytes = 2 * (CT * KS * 64 + 512);
    auto kernel = int8_head_kernel<KS, FN, FW>;
    static std::atomic<uint64_t> raised{0};
    kc_raise_lds_limit((const void*)kernel, bytes, raised);
    BLSTM_LAUNCH("int8_head", kernel, dim3((unsigned)(h.ranges * h.nf)), dim3(256), bytes, s, p);
  };
#define INT(n) std::integral_constant<int, n>{}
  auto waves = [&](auto ks, auto fn) {
    if (h.fw == 1) launch(ks, fn, INT(1));
    else if (h.fw == 2) launch(ks, fn, INT(2));
    else launch(ks, fn, INT(4));
  };
  if (h.ks <= 1) waves(INT(1), INT(2));
  else if (h.ks <= 2) waves(INT(2), INT(2));
  else if (h.ks <= 4) waves(INT(4), INT(2));
  else if (h.ks <= 8) waves(INT(8), INT(2));
  else waves(INT(16), INT(1));
#undef INT
  int rc = blstm_check_launch("int8_head");
  if (rc) return rc;
  const HeadOut o{sc.ids, sc.logprob, sc.entropy, sc.top, sc.idx, sc.n, sc.k, 4 / h.fw};
  BLSTM_LAUNCH("int8_head_finish", int8_head_finish_kernel, dim3((unsigned)M), dim3(FT_), (size_t)Kw, s, p, o);
  return blstm_check_launch("int8_head_finish");
}
