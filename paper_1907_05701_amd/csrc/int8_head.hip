// The 8-bit head: log probabilities without the logits in memory.
//
// Pass 1 multiplies a tile of frames with a range of classes and keeps, per
// frame and lane, the softmax sums so far and the largest logit of every group
// of classes that the lane sees.  Pass 2 joins a frame's sums; the few groups
// that reach the k-th largest of the groups' maxima hold its k most likely
// classes, whose logits it computes again, as it does the listed classes': sums
// of integers are exact, so these are the same bits.
//
// 2688 bf16 frames of 256 columns, 32000 classes, 8 of them most likely: 47 us the first pass, which the vector unit bounds
// (9.5 instructions a logit beside the products: conversion, two scalings, bias, exponent, exponential, two sums, half a
// maximum; 27 us of issue at 2.4 GHz with three waves a SIMD, the matrix unit busy for 9), 20 us the second (8 KB of group
// maxima and some 37 KB of weights a frame).  Written out and read back the logits would be 344 MB twice (258 us so).
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "gemm_kc.hpp"
#include "int8.hpp"
#include "rows.hpp"
#include "score.hpp"

static constexpr int CT = 64;             // classes of a tile: one stage in LDS
// Tiles over which a lane's group maxima are taken: 16 classes a group, 8 where four waves share a tile.  (Larger groups
// mean fewer maxima, and more classes to compute again: with 32, the second pass of 2688 frames reads 172 MB of weights.)
__host__ __device__ constexpr int group_tiles(int fw) { return fw == 4 ? 1 : 2; }
// Biases below FLOOR count as FLOOR in the first pass, and sums start from a reference above it, so that such a class
// adds 0; rows that have no other, or not k others, are for the second pass alone.
static constexpr float FLOOR = -1e30f, START = 0.5f * FLOOR;
// That holds as long as no product comes near FLOOR: with scales below SCALE_MAX it is at most 2^24 * 10^20.  A class of a
// larger scale is a NaN in the first pass, and leaves every frame to the second; so does a frame's own scale its frame.
static constexpr float SCALE_MAX = 1e10f;
// How far above its reference a lane's largest exponent may get: a reference that follows every new maximum takes
// its branch in most tiles, one that follows far behind makes T large and its rounding with it (30: the entropy's
// error 1.8e-6).
static constexpr float SLACK = 4.f;
// Largest reference, as an exponent, that the sums are good for: its rounding, at most 8 below that, shifts all of a frame's
// exponents alike.  That of larger ones could reach float32's ends, and logits that large are no masks; such
// frames are for the second pass alone.
static constexpr float REF_MAX = 0x1p28f;

struct HeadP {
  const void* x;           // tokens, where the first pass quantises them itself
  int64_t ldx;
  int P;
  int8_t* q;               // their integers [M][Kw] and scales
  float* xs;
  const int8_t* w;
  int64_t ldw;
  const float *ws, *bias;
  int64_t M;
  int K, Kw;               // classes, columns
  int nf, ranges, per;     // frame tiles, class ranges, tiles a range
  int ngroup;              // a frame's group maxima
  float it2, itau;         // log2 e / tau, 1 / tau
  float4* stats;           // [M][ranges]: reference (an exponent of 2), Z, T
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

__device__ __forceinline__ float fmax_nan(float v, float least) { return v < least ? least : v; }   // a NaN stays

// 16-byte chunk c of row r of a tile of NCH chunks a row: the slot it lies in (16 rows' chunk c in 16 different
// bank groups).
template <int NCH>
__device__ __forceinline__ int head_slot(int c, int r) {
  return c ^ (NCH >= 16 ? r & 15 : (r * NCH / 16) & (NCH - 1));
}

// KS: most 64-column steps; 16 FN frames a wave; FW waves side by side along the
// frames, the other 4 / FW along the classes of a tile.  TI: tokens of this type are quantised here, by every workgroup
// for itself (a launch less), and left for the second pass by the first range's; void: their integers lie in memory.
constexpr int head_per_cu(int ks) { return ks > 8 ? 1 : ks > 4 ? 2 : 3; }   // workgroups, by their registers
template <int KS, int FN, int FW, typename TI>
__global__ __launch_bounds__(256, head_per_cu(KS)) void int8_head_kernel(const HeadP p) {
  constexpr int WC = 4 / FW, NI = 4 / WC, TG = group_tiles(FW), NCH = KS * 4, TILE = CT * KS * 64, STAGE = TILE + 512;
  constexpr int LOADS = TILE / 1024 / 4;   // of a wave
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fc = lane >> 4;
  const int wf = wid % FW, wc = wid / FW;
  // workgroup w runs on XCD w % 8: each takes a run of ranges, whose weights its L2 then holds
  const int total = p.nf * p.ranges, share = total / 8;
  const int at = (int)blockIdx.x < 8 * share ? blockIdx.x % 8 * share + blockIdx.x / 8 : blockIdx.x, range = at / p.nf;
  const int64_t f0 = (int64_t)(at % p.nf) * (16 * FN * FW) + wf * 16 * FN;
  const int tile0 = range * p.per, tiles = min((int)((p.K + CT - 1) / CT) - tile0, p.per);
  const int8_t* wb = p.w + (int64_t)tile0 * CT * p.ldw;
  const int rows = p.K - tile0 * CT;   // classes from the range's first on

  // a tile's scales and biases, one a lane of the first two waves, go through registers: a bias of -inf would make 0 times
  // -inf of a class that adds nothing
  float next = 0.f;
  auto fetch = [&](int j) {
    const int c = j * CT + lane;
    if (wid == 0) next = c < rows ? p.ws[tile0 * CT + c] : 0.f;
    if (wid == 1) next = c < rows ? (p.bias ? p.bias[tile0 * CT + c] : 0.f) : FLOOR;
  };
  auto put = [&](int j) {
    if (wid < 2) *(float*)(lds + (j & 1) * STAGE + TILE + wid * 256 + lane * 4) = wid ? fmax_nan(next, FLOOR) : fabsf(next) < SCALE_MAX ? next : NAN;
  };
  // a tile's rows end with the last class: what lies behind it, and behind a row's columns, reads as zeros
  uint32_t off[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int pos = (i * 4 + wid) * 64 + lane, row = pos / NCH, c = head_slot<NCH>(pos % NCH, row);
    off[i] = c * 16 < p.Kw ? (uint32_t)(row * p.ldw + c * 16) : DMA_OFF_NONE;
  }
  auto issue = [&](int j) {
    char* st = lds + (j & 1) * STAGE;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(wb + (int64_t)j * CT * p.ldw), (short)0, (int)(min(CT, rows - j * CT) * p.ldw), 0x00020000);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) dma16(r, off[i], st + (i * 4 + wid) * 1024);
  };
  // both stages are on their way before anything is waited for
  issue(0);
  fetch(0);
  const float first = next;
  if (tiles > 1) {
    issue(1);
    fetch(1);
  }

  const int own = (int)min((int64_t)16 * FN * FW, p.M - (f0 - wf * 16 * FN));   // frames of the workgroup
  float* scales = (float*)(lds + 2 * STAGE + 16 * FN * FW * (KS * 64 + 16));
  if constexpr (!std::is_void<TI>::value) {
    constexpr int V = 16 / sizeof(TI), NV = KS > V ? KS / V : 1;
    tokens_to_lds<TI, 4, NV < 4 ? 4 : 2, NV>((const TI*)p.x + (f0 - wf * 16 * FN) * p.ldx, p.ldx, own, p.P, KS * 64, lds + 2 * STAGE, scales);
    __syncthreads();
  }
  i32x4 b[FN][KS];
  float xs[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int64_t f = min(f0 + j * 16 + fr, p.M - 1);   // frames past the last: any, not stored
    if constexpr (std::is_void<TI>::value) {
      xs[j] = p.xs[f];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int k = ks * 64 + fc * 16;
        b[j][ks] = ints16(p.q + f * p.Kw, k, p.Kw);
      }
    } else {
      const int row = (wf * FN + j) * 16 + fr;
      const char* t = lds + 2 * STAGE + (row < own ? row : 0) * (KS * 64 + 16);   // frames past the last: any
      xs[j] = scales[row < own ? row : 0];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int k = ks * 64 + fc * 16;
        b[j][ks] = *(const i32x4*)(t + k);
        if (range == 0 && wc == 0 && row < own && k < p.Kw) *(i32x4*)(p.q + f * p.Kw + k) = b[j][ks];
      }
      if (range == 0 && wc == 0 && row < own && fc == 0) p.xs[f] = xs[j];
    }
  }
  Sums s[FN];
  float lim[FN], gm[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    s[j] = Sums{START * p.it2, 0.f, 0.f};
    lim[j] = START;
    gm[j] = -INFINITY;
  }
  const float slack = SLACK / p.it2;
  {
    const float second = next;
    next = first;
    put(0);
    next = second;
    if (tiles > 1) put(1);
  }
  uint32_t at_k[KS];   // of a lane's piece in the first 16 rows of its wave (the slot depends on the row in 16 alone)
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) at_k[ks] = (wc * NI * 16 + fr) * (NCH * 16) + head_slot<NCH>(ks * 4 + fc, fr) * 16;

  for (int it = 0; it < tiles; ++it) {
    int8_stage_wait();
    kc_barrier();
    const bool more = it > 0 && it + 1 < tiles;
    if (more) {
      issue(it + 1);
      fetch(it + 1);
    }
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
        const i32x4 a = *(const i32x4*)(st + at_k[ks] + i * 16 * NCH * 16);
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[j] = mma_i8(a, b[j][ks], acc[j]);
      }
      const f32x4 w4 = *(const f32x4*)(st + TILE + (row + 4 * fc) * 4), b4 = *(const f32x4*)(st + TILE + 256 + (row + 4 * fc) * 4);
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) l[i][j][r] = int8_value(acc[j][r], scale_of(xs[j], w4[r]), b4[r]);
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
      float z = 0.f, t = 0.f;   // of the tile: shorter chains of additions
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float y = fmaf(l[i][j][r], p.it2, -s[j].rc), e = exp2_(y);
          z += e;
          t += e * y;
        }
      s[j].z += z;
      s[j].t += t;
      gm[j] = fmaxf(gm[j], mb);
      if (p.gmax && (it % TG == TG - 1 || it + 1 == tiles)) {
        const int64_t f = f0 + j * 16 + fr;
        if (f < p.M) p.gmax[f * p.ngroup + ((tile0 + it) / TG * WC + wc) * 4 + fc] = gm[j];
        gm[j] = -INFINITY;
      }
    }
    if (more) put(it + 1);
  }
  // a frame's lanes, then its waves
#pragma unroll
  for (int j = 0; j < FN; ++j) {
#pragma unroll
    for (int o = 16; o < 64; o <<= 1)
      s[j].join(Sums{__shfl_xor(s[j].rc, o), __shfl_xor(s[j].z, o), __shfl_xor(s[j].t, o)});
  }
  if constexpr (WC > 1) {
    static_assert(4 * FN * 16 * sizeof(Sums) <= STAGE, "the first stage is done with");
    __syncthreads();
    Sums* part = (Sums*)lds;
    if (fc == 0) {
#pragma unroll
      for (int j = 0; j < FN; ++j) part[(wid * FN + j) * 16 + fr] = s[j];
    }
    __syncthreads();
    if (wc > 0) return;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int w = 1; w < WC; ++w) s[j].join(part[((w * FW + wf) * FN + j) * 16 + fr]);
  }
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    const int64_t f = f0 + j * 16 + fr;
    if (fc == 0 && f < p.M) p.stats[f * p.ranges + range] = float4{s[j].rc, s[j].z, s[j].t, 0.f};
  }
}

// ---------------------------------------------------------------------------
// Second pass: a workgroup a frame.
// ---------------------------------------------------------------------------
struct HeadOut {
  const int32_t* ids;
  float *logprob, *entropy, *top;
  int32_t* idx;
  int n, k, fw;   // fw: waves along the frames in the first pass
};
static constexpr int FT = 128;           // threads: the workgroups of 2688 frames then run all at once
static constexpr int FCAND = 512;        // most candidates
static constexpr int GROUPS = 512;       // most groups computed again

// A class's logit, the bits of the first pass.
struct Logit {
  const int8_t* w;
  int64_t ldw;
  const float *ws, *bias;
  const i32x4* x;   // the frame's integers, in LDS
  int chunks;
  float xs;
  __device__ __forceinline__ float value(int sum, int c) const { return int8_value(sum, scale_of(xs, ws[c]), bias ? bias[c] : 0.f); }
  __device__ __forceinline__ int dot(const i32x4* r, int i) const {
    const i32x4 u = r[i], v = x[i];
    int a = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) a = __builtin_amdgcn_sdot4(u[j], v[j], a, false);
    return a;
  }
  __device__ __forceinline__ float operator()(int c) const {   // by one lane
    const i32x4* r = (const i32x4*)(w + c * ldw);
    int a = 0;
#pragma unroll 4
    for (int i = 0; i < chunks; ++i) a += dot(r, i);
    return value(a, c);
  }
  // by four adjacent lanes, U classes at once; each lane has the results
  template <int U>
  __device__ __forceinline__ void four(const int (&c)[U], float (&v)[U]) const {
    int a[U];
    float s[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      a[u] = 0;
      s[u] = ws[c[u]];
      b[u] = bias ? bias[c[u]] : 0.f;
    }
#pragma unroll 4
    for (int i = threadIdx.x & 3; i < chunks; i += 4)
#pragma unroll
      for (int u = 0; u < U; ++u) a[u] += dot((const i32x4*)(w + c[u] * ldw), i);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      a[u] += __shfl_xor(a[u], 1);
      a[u] += __shfl_xor(a[u], 2);
      v[u] = int8_value(a[u], scale_of(xs, s[u]), b[u]);
    }
  }
};

struct HeadLds {
  TopkLds<FT, FCAND, 4 * FT> l;   // four maxima a thread
  float buf[4][4];
  float listed[SOFTMAX_MAX_TOP];   // the listed classes' logits
  int32_t groups[GROUPS];
  uint32_t ngroups, hist[256], want;
};

// A log probability from joined sums.
struct HeadLogProb {
  float rc, l2z, it2, itau;
  __device__ __forceinline__ float operator()(float v) const {
    // a mask's exponent could overflow; the reference, at most 2^28 / it2 <= 2^-21.8 of it, does not count beside it
    return v < -1e30f ? v * itau : (fmaf(v, it2, -rc) - l2z) * LN2_F;
  }
};

// Any row, its logits computed again in every pass: one with a NaN or infinities, with a scale beyond SCALE_MAX or a
// reference beyond REF_MAX, with fewer than k classes above FLOOR, or with too many that reach the threshold.  (3.0 ms for up
// to 16 frames of 32000 classes and 256 columns, 17.5 for 2688: a lane computes a class, seven times.)
__device__ __forceinline__ void head_any(HeadLds& h, const Logit& logit, const HeadP& p, const HeadOut& o, int64_t m) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K;
  float mx = -INFINITY;
  bool nan = false;
  for (int c = tid; c < K; c += FT) {
    const float v = logit(c);
    mx = fmaxf(mx, v);
    nan |= v != v;
  }
  nan = __syncthreads_or(nan);
  mx = row_max<FT>(fmaxf(mx, -INFINITY), h.buf[0]);
  const bool some = nan || !(mx == -INFINITY);
  const float ref = some ? mx : 0.f;
  float z = 0.f, t = 0.f;
  for (int c = tid; c < K; c += FT) {
    const float y = (logit(c) - ref) * p.it2, e = exp2_(y);
    z += e;
    t += e * fmaxf(y, -200.f);
  }
  z = row_sum<FT>(z, h.buf[1]);
  t = row_sum<FT>(t, h.buf[2]);
  const float lz = log2f(z) * LN2_F;   // a NaN where there is one, or +inf
  auto value = [&](float v) { return some ? (v - ref) * p.itau - lz : -INFINITY; };
  for (int i = tid; i < o.n; i += FT) {
    const int at = o.ids[m * o.n + i];
    o.logprob[m * o.n + i] = at < 0 || at >= K ? 0.f : value(logit(at));
  }
  if (o.entropy && tid == 0) o.entropy[m] = some ? lz - t / z * LN2_F : 0.f;
  if (!o.k) return;
  // the k-th largest order word, eight bits at a time, and how many of its ties are taken
  uint32_t word = 0;
  int want = o.k;   // among the words that agree with `word` so far
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = tid; i < 256; i += FT) h.hist[i] = 0;
    __syncthreads();
    for (int c = tid; c < K; c += FT) {
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
  for (int c0 = 0; c0 < K; c0 += FT) {
    const int c = c0 + tid;
    const float v = c < K ? logit(c) : 0.f;
    const uint32_t u = c < K ? order_word(v) : 0;
    const uint64_t same_ = __ballot(c < K && u == word);
    __syncthreads();
    if (lane == 0) h.hist[wave] = __popcll(same_);
    __syncthreads();
    int before = taken;
    for (int i = 0; i < FT / 64; ++i) {
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

__global__ __launch_bounds__(FT, 6) void int8_head_finish_kernel(const HeadP p, const HeadOut o) {
  extern __shared__ __attribute__((aligned(16))) char xl[];
  __shared__ HeadLds h;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = p.K;
  const int64_t m = blockIdx.x;
  // every first load goes out before any is waited for
  for (int i = tid; i < p.Kw / 16; i += FT) ((i32x4*)xl)[i] = ((const i32x4*)(p.q + m * p.Kw))[i];
  const Logit logit{p.w, p.ldw, p.ws, p.bias, (const i32x4*)xl, p.Kw / 16, p.xs[m]};
  if (tid == 0) h.ngroups = h.l.count = 0;
  constexpr int NS = 4;
  const float4* st = p.stats + m * p.ranges;
  float4 sv[NS];
  if (wave == 1) {
#pragma unroll
    for (int i = 0; i < NS; ++i) sv[i] = st[min(lane + i * 64, p.ranges - 1)];
  }
  const int first = (1 - wave) * 16 + lane / 4;   // of the list: the first wave has the threshold to find
  int at = first < o.n ? o.ids[m * o.n + first] : -1;
  // group maxima: up to NG quads a thread in registers, others read again
  constexpr int NG = 8;
  const f32x4* gmax = (const f32x4*)(p.gmax + m * p.ngroup);
  const int quads = p.ngroup / 4;
  const f32x4 low{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  f32x4 mx = low, gv[NG];
  auto larger = [&](const f32x4& v) {
#pragma unroll
    for (int j = 0; j < 4; ++j) mx[j] = fmaxf(mx[j], v[j]);
  };
  if (o.k) {
#pragma unroll
    for (int i = 0; i < NG; ++i) gv[i] = tid + i * FT < quads ? gmax[tid + i * FT] : low;
#pragma unroll
    for (int i = 0; i < NG; ++i) larger(gv[i]);
    for (int g = tid + NG * FT; g < quads; g += FT) larger(gmax[g]);
#pragma unroll
    for (int j = 0; j < 4; ++j) h.l.tmax[j * FT + tid] = order_word(mx[j]);
  }
  __syncthreads();
  if (wave == 0) {
    if (o.k) {
      // where a thread has one quad at most these are the groups' maxima themselves, too few to be joined (1671 frames of
      // 1000 classes, 30 of them: 38 us, 394 by groups of four of them, of which there are 16)
      const uint32_t t = kth_search<12>(h.l, o.k, quads <= FT ? 0 : FOLD);
      if (lane == 0) h.l.thr = t;
    }
  } else {
    float rc = START * p.it2;
#pragma unroll
    for (int i = 0; i < NS; ++i) rc = fmaxf(rc, sv[i].x);
    for (int i = lane + NS * 64; i < p.ranges; i += 64) rc = fmaxf(rc, st[i].x);
    rc = wave_max(rc);
    float z = 0.f, t = 0.f;
    auto add = [&](float4 v) {
      Sums s{v.x, v.y, v.z};
      s.rise(rc);
      z += s.z;
      t += s.t;
    };
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (lane + i * 64 < p.ranges) add(sv[i]);
    for (int i = lane + NS * 64; i < p.ranges; i += 64) add(st[i]);
    z = wave_sum(z);
    t = wave_sum(t);
    if (lane == 0) {
      // (as a term of the condition behind the barrier it costs 27 spilled registers: 2688 frames 73 us, 66 so)
      h.buf[0][0] = logit.xs < SCALE_MAX ? rc : INFINITY;
      h.buf[0][1] = z;
      h.buf[0][2] = t;
    }
  }
  for (int e = first; e < o.n; e += FT / 4) {   // the four lanes of an entry stay together
    if (e > first) at = o.ids[m * o.n + e];
    const int c[1] = {at < 0 || at >= K ? 0 : at};
    float v[1];
    logit.four(c, v);
    h.listed[e] = v[0];
  }
  __syncthreads();
  const float rc = h.buf[0][0], z = h.buf[0][1], t = h.buf[0][2];
  // (a NaN fails all; a temperature beyond that would bring FLOOR's classes back in, and one below about 2e-9, where START's
  // exponent is -inf, leaves t a NaN)
  if (same(!(z > 0.f && z < INFINITY && fabsf(t) < INFINITY && fabsf(rc) < REF_MAX && p.it2 > 1e-15f))) {
    head_any(h, logit, p, o, m);
    return;
  }
  const HeadLogProb lp{rc, log2f(z), p.it2, p.itau};
  if (o.k) {
    const uint32_t tw = max(same(h.l.thr), order_word(START));
    const float thr = order_value(tw);
    if (fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) >= thr) {
      auto reach = [&](const f32x4& v, int g) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (v[j] >= thr) {
            const uint32_t at = atomicAdd(&h.ngroups, 1u);
            if (at < GROUPS) h.groups[at] = 4 * g + j;
          }
      };
#pragma unroll
      for (int i = 0; i < NG; ++i) reach(gv[i], tid + i * FT);
      for (int g = tid + NG * FT; g < quads; g += FT) reach(gmax[g], g);
    }
    __syncthreads();
    // a group's classes: 4 adjacent ones of every 16 that its wave has in a tile
    const int ng = (int)same(h.ngroups), tg = group_tiles(o.fw), wc = 4 / o.fw, ni = o.fw, size = 4 * ni * tg;
    constexpr int U = 2;
    if (ng <= GROUPS) {
      for (int e0 = 0; e0 < ng * size; e0 += U * FT / 4) {
        int c[U];
        float v[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int e = e0 + u * (FT / 4) + tid / 4;
          in[u] = e < ng * size;
          const int g = in[u] ? h.groups[e / size] : 0, q = g % 4, w = g / 4 % wc, tile = g / 4 / wc * tg;
          const int b = e % size / (4 * ni), i = e % (4 * ni) / 4, r = e % 4;
          c[u] = (tile + b) * CT + (w * ni + i) * 16 + 4 * q + r;
          in[u] = in[u] && c[u] < K;
          c[u] = in[u] ? c[u] : 0;
        }
        logit.four(c, v);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (in[u] && (tid & 3) == 0 && v[u] >= thr) push(h.l, v[u], c[u]);
      }
      __syncthreads();
    }
    int n = (int)same(h.l.count);
    // where groups are few they bound the k-th badly, and ranking takes n^2 steps: the k-th of the candidates' own maxima then
    // (1671 float32 frames of 256 columns, 319 classes, 30 of them: 31 us, 49 without)
    if (n <= FCAND && n > 2 * o.k + 64) {
      static_assert(FCAND == 4 * FT, "four candidates a thread");
      uint64_t own[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        own[j] = j * FT + tid < n ? h.l.cand[j * FT + tid] : 0;
        h.l.tmax[j * FT + tid] = (uint32_t)(own[j] >> 32);
      }
      __syncthreads();
      if (wave == 0) {
        const uint32_t t = kth_search<0>(h.l, o.k);
        if (lane == 0) {
          h.l.thr = t;
          h.l.count = 0;
        }
      }
      __syncthreads();
      const uint32_t t = h.l.thr;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if ((uint32_t)(own[j] >> 32) >= t && own[j]) h.l.cand[atomicAdd(&h.l.count, 1u)] = own[j];
      __syncthreads();
      n = (int)same(h.l.count);
    }
    // too many reach the threshold, or, where fewer than k classes lie above FLOOR, too few
    if (ng > GROUPS || n > FCAND || n < o.k) {
      head_any(h, logit, p, o, m);
      return;
    }
    TopkP tp{0, K, o.k, p.it2, o.top, nullptr, o.idx};
    rank(h.l, n, m, tp, lp);
  }
  for (int i = tid; i < o.n; i += FT) {
    const int id = o.ids[m * o.n + i];
    o.logprob[m * o.n + i] = id < 0 || id >= K ? 0.f : lp(h.listed[i]);
  }
  if (o.entropy && tid == 0) o.entropy[m] = (lp.l2z - t / z) * LN2_F;
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct HeadPlan {
  int fn, fw, ks;                 // frames / 16 of a wave, waves along the frames, most column steps
  int nf, ngroup, ranges, per;
  int64_t units, slots, most;     // runs of classes that may not be parted; workgroups at a time; most ranges
  size_t stats, gmax;             // behind the tokens
};
static constexpr int HEAD_MAX_STEPS = 16;

// Whether the first pass quantises its tokens itself: where they are few, and beside two stages of long rows there is room.
static constexpr bool quantised_here(int fw, int ks) { return fw == 1 || (fw == 2 && ks <= 8); }
static constexpr size_t head_lds(int fn, int fw, int ks) {
  return 2 * (CT * ks * 64 + 512) + (quantised_here(fw, ks) ? 16 * fn * fw * (ks * 64 + 16 + 4) : 0);
}
// Workgroups of the first pass that run at a time.  (512 columns of 17 to 64 frames have LDS for one a CU.  us, planned for
// one / for the two that the registers hold: 17 frames of 45000 classes 28.0 / 34.6, of 131072 43.0 / 50.8; 64 frames 40.2 / 53.3
// and 50.0 / 65.8.)
static int head_slots(int fn, int fw, int ks) {
  return 256 * (int)std::min<size_t>(head_per_cu(ks), 160 * 1024 / head_lds(fn, fw, ks));
}

static HeadPlan head_shape(int64_t M, int32_t K, int32_t Kw) {
  HeadPlan h{};
  h.ks = Kw <= 64 ? 1 : Kw <= 128 ? 2 : Kw <= 256 ? 4 : Kw <= 512 ? 8 : HEAD_MAX_STEPS;
  h.fn = h.ks > 8 || M <= 16 ? 1 : 2;
  const int frames = 16 * h.fn;
  h.fw = M <= frames ? 1 : M <= 2 * frames ? 2 : 4;
  h.nf = (int)cdiv(M, frames * h.fw);
  const int tg = group_tiles(h.fw);
  h.units = cdiv(K, CT * tg);
  h.slots = head_slots(h.fn, h.fw, h.ks);
  h.ngroup = (int)h.units * (4 / h.fw) * 4;
  // (of one tile of frames, two rounds are never shorter than one of ranges twice as long)
  h.most = std::min(h.units, std::max<int64_t>(1, (h.nf == 1 ? 1 : 2) * h.slots / h.nf));
  return h;
}
static HeadPlan head_plan(int64_t M, int32_t K, int32_t Kw) {
  HeadPlan h = head_shape(M, K, Kw);
  const int tg = group_tiles(h.fw);
  // as many ranges as take least: whole rounds of the chip, each as long as a range and its start
  int64_t best = -1, per = 1;
  for (int64_t r = 1; r <= h.most; ++r) {
    const int64_t u = cdiv(h.units, r), t = cdiv(cdiv(h.units, u) * h.nf, h.slots) * (u * tg + 1);
    if (best < 0 || t < best) {
      best = t;
      per = u;
    }
  }
  h.per = (int)per * tg;
  h.ranges = (int)cdiv(h.units, per);
  h.stats = 0;
  h.gmax = (size_t)rup(M * h.ranges * 16, 256);
  return h;
}

bool int8_head_fits(int32_t Kw) { return cdiv(Kw, 64) <= HEAD_MAX_STEPS; }
static size_t ints_bytes(int64_t M, int32_t Kw) { return (size_t)(rup(M * Kw, 256) + rup(M * 4, 256)); }
// For every number of frames up to M: the shapes change behind 16, 32 and 64 frames, and of one shape more frames have more
// tokens and maxima; their statistics, M times ranges, are at most M times `units`, and at most those of whole tiles in
// two rounds (one round of one tile) or of one range.
size_t int8_head_bytes(int64_t M, int32_t K, int32_t Kw) {
  size_t bytes = 0;
  for (const int64_t end : {(int64_t)16, (int64_t)32, (int64_t)64, M}) {
    const int64_t m = std::min(end, M);
    const HeadPlan h = head_shape(m, K, Kw);
    const int64_t stats = h.nf == 1 ? m * h.most : std::min(m * h.units, std::max(m, 2 * h.slots * 16 * h.fn * h.fw));
    bytes = std::max(bytes, ints_bytes(m, Kw) + (size_t)rup(stats * 16, 256) + (size_t)rup(m * h.ngroup * 4, 256));
  }
  return bytes;
}

template <typename TI>
int int8_head(const TI* x, int64_t ldx, int64_t M, int32_t P, const int8_t* w, int64_t ldw, const float* ws, int32_t K,
              int32_t Kw, const float* bias, const softmax_scores& sc, char* buf, hipStream_t s) {
  const HeadPlan h = head_plan(M, K, Kw);
  HeadP p{};
  p.x = x; p.ldx = ldx; p.P = P; p.q = (int8_t*)buf; p.xs = (float*)(buf + rup(M * Kw, 256));
  p.w = w; p.ldw = ldw; p.ws = ws; p.bias = bias; p.M = M; p.K = K; p.Kw = Kw;
  p.nf = h.nf; p.ranges = h.ranges; p.per = h.per; p.ngroup = h.ngroup;
  p.it2 = LOG2E_F / sc.temperature; p.itau = 1.f / sc.temperature;
  buf += ints_bytes(M, Kw);
  p.stats = (float4*)(buf + h.stats);
  p.gmax = sc.k ? (float*)(buf + h.gmax) : nullptr;
  auto launch = [&](auto ks, auto fn, auto fw) {
    constexpr int KS = decltype(ks)::value, FN = decltype(fn)::value, FW = decltype(fw)::value;
    constexpr bool here = quantised_here(FW, KS);
    constexpr size_t bytes = head_lds(FN, FW, KS);
    auto kernel = int8_head_kernel<KS, FN, FW, typename std::conditional<here, TI, void>::type>;
    static_assert(bytes <= 160 * 1024, "LDS");
    if (!here) int8_quantize(x, ldx, M, P, p.q, Kw, Kw, p.xs, s);
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
  auto columns = [&](auto ks) {
    if (M <= 16) launch(ks, INT(1), INT(1));
    else waves(ks, INT(2));
  };
  switch (h.ks) {
    case 1: columns(INT(1)); break;
    case 2: columns(INT(2)); break;
    case 4: columns(INT(4)); break;
    case 8: columns(INT(8)); break;
    default: waves(INT(HEAD_MAX_STEPS), INT(1));
  }
#undef INT
  const int rc = blstm_check_launch("int8_head");
  if (rc) return rc;
  const HeadOut o{sc.ids, sc.logprob, sc.entropy, sc.top, sc.idx, sc.n, sc.k, h.fw};
  BLSTM_LAUNCH("int8_head_finish", int8_head_finish_kernel, dim3((unsigned)M), dim3(FT), (size_t)Kw, s, p, o);
  return blstm_check_launch("int8_head_finish");
}
template int int8_head<float>(const float*, int64_t, int64_t, int32_t, const int8_t*, int64_t, const float*, int32_t, int32_t, const float*, const softmax_scores&, char*, hipStream_t);
template int int8_head<bf16>(const bf16*, int64_t, int64_t, int32_t, const int8_t*, int64_t, const float*, int32_t, int32_t, const float*, const softmax_scores&, char*, hipStream_t);
