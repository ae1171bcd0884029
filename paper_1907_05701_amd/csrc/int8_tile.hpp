// The product of 8-bit integers in tiles, and for few tokens.
#pragma once

#include <algorithm>

#include "gemm_kc.hpp"
#include "int8.hpp"

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

// Rows of BK bytes in LDS, chunk c of row r in slot kc_slot<BK / 2>(c, r).
template <int ROWS, int BK, int NW>
__device__ __forceinline__ void stage(const int8_t* base, int64_t ld, int64_t rows, int k0, int K, char* tile, int wid,
                                      int lane) {
  const __amdgpu_buffer_rsrc_t r = dma_rsrc(base);
  constexpr int CPR = BK / 16, LOADS = ROWS * BK / 1024 / NW;
  static_assert(ROWS * BK % (1024 * NW) == 0, "rows of a tile split over the waves");
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = (i * NW + wid) * (64 / CPR) + lane / CPR;
    const int k = k0 + kc_slot<BK / 2>(lane % CPR, row) * 16;
    dma16(r, row < rows && k < K ? (uint32_t)(row * ld + k) : DMA_OFF_NONE, tile + (i * NW + wid) * 1024);
  }
}

// BM channels x BN tokens a workgroup of WM x WN waves, BK of K at a time in a ring of STAGES.
template <typename TO, int BM, int BN, int WM, int WN, int BK, int STAGES>
__global__ __launch_bounds__(WM * WN * 64, std::min(160 * 1024 / (STAGES * (BM + BN) * BK), 4) * WM * WN / 4)
void int8_tile_kernel(const Int8P p) {
  constexpr int NW = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16, STAGE = (BM + BN) * BK;
  constexpr int LOADS = (BM + BN) * BK / 1024 / NW;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wid % WM, wn = wid / WM;
  int z, tm, tn;
  kc_tile_of(p, blockIdx.x, p.gm, z, tm, tn);
  const int64_t n0 = (int64_t)tm * BM, m0 = (int64_t)tn * BN;
  const int steps = (p.K + BK - 1) / BK;
  const int8_t *wb = p.w + n0 * p.ldw, *xb = p.x + m0 * p.ldx;
  auto issue = [&](int j) {
    char* st = lds + (j % STAGES) * STAGE;
    stage<BM, BK, NW>(wb, p.ldw, p.N - n0, j * BK, p.K, st, wid, lane);
    stage<BN, BK, NW>(xb, p.ldx, p.M - m0, j * BK, p.K, st + BM * BK, wid, lane);
  };
  i32x4 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const int fr = lane & 15, fc = lane >> 4;
#pragma unroll
  for (int j = 0; j < STAGES - 1; ++j)
    if (j < steps) issue(j);
  for (int it = 0; it < steps; ++it) {
    // the oldest stage has landed, and this wave's reads of the one that is filled next are done
    if (it + STAGES - 2 < steps) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * LOADS) : "memory");
    else int8_stage_wait();
    kc_barrier();
    if (it + STAGES - 1 < steps) issue(it + STAGES - 1);
    const char* st = lds + (it % STAGES) * STAGE;
#pragma unroll
    for (int ks = 0; ks < BK / 64; ++ks) {
      i32x4 a[FM], b[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i)
        a[i] = *(const i32x4*)(st + (wm * (BM / WM) + i * 16 + fr) * BK + kc_slot<BK / 2>(ks * 4 + fc, fr) * 16);
#pragma unroll
      for (int j = 0; j < FN; ++j)
        b[j] = *(const i32x4*)(st + BM * BK + (wn * (BN / WN) + j * 16 + fr) * BK + kc_slot<BK / 2>(ks * 4 + fc, fr) * 16);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mma_i8(a[i], b[j], acc[i][j]);
    }
  }
  float xs[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) xs[j] = p.xs[min(m0 + wn * (BN / WN) + j * 16 + fr, p.M - 1)];
  if constexpr (std::is_same<TO, bf16>::value && FM % 2 == 0) {
    // two fragments' 16 channels side by side: rows of 16 lanes trade places, so that a lane stores 8 adjacent channels
    // and an instruction 64 bytes of each token (at any alignment; us, so / by four channels: 16384 x 4096 x 4096
    // 238 / 265, 3153 x 4268 x 1024 22.8 / 30.9, x 4267 28.3 / 30.3)
#pragma unroll
    for (int i = 0; i < FM; i += 2) {
      const int64_t n = n0 + wm * (BM / WM) + i * 16;
      f32x4 w[2], b[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int64_t c = min(n + u * 16 + 4 * fc + r, p.N - 1);   // channels past the last: any, dropped
          w[u][r] = p.ws[c];
          b[u][r] = p.bias ? p.bias[c] : 0.f;
        }
      const int64_t c = n + (fc & 1) * 16 + (fc >> 1) * 8;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        uint32_t o[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          bf16 v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = (bf16)int8_value(acc[i + u][j][r], scale_of(xs[j], w[u][r]), b[u][r]);
          __builtin_memcpy(o[u], v, 8);
        }
        const auto lo = __builtin_amdgcn_permlane16_swap(o[0][0], o[1][0], false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(o[0][1], o[1][1], false, false);
        const int64_t m = m0 + wn * (BN / WN) + j * 16 + fr;
        const i32x4 out{(int)lo[0], (int)hi[0], (int)lo[1], (int)hi[1]};
        bf16* y = (bf16*)p.y + m * p.ldy + c;
        if (m < p.M && c + 8 <= p.N) __builtin_memcpy(y, &out, 16);
        else if (m < p.M && c < p.N) {
          bf16 v[8];
          __builtin_memcpy(v, &out, 16);
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (c + r < p.N) y[r] = v[r];
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      put4<TO>(p, m0 + wn * (BN / WN) + j * 16 + fr, n0 + wm * (BM / WM) + i * 16 + 4 * fc, acc[i][j], xs[j]);
}

template <typename TO, int BM, int BN, int WM, int WN, int BK, int STAGES>
static void int8_tile_launch(Int8P p, hipStream_t s) {
  constexpr size_t bytes = STAGES * (BM + BN) * BK;
  static_assert(bytes <= 160 * 1024, "LDS");
  auto fn = int8_tile_kernel<TO, BM, BN, WM, WN, BK, STAGES>;
  static std::atomic<uint64_t> raised{0};
  kc_raise_lds_limit((const void*)fn, bytes, raised);
  p.ntm = (int)cdiv(p.N, BM);
  p.ntn = (int)cdiv(p.M, BN);
  p.gm = kc_group_rows;
  p.total = p.ntm * p.ntn;
  BLSTM_LAUNCH("int8_linear", fn, dim3((unsigned)p.total), dim3(WM * WN * 64), bytes, s, p);
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
  constexpr int U = 4;   // steps whose loads go out together
  for (int k = wid * 64; k < p.K; k += U * 256) {
    i32x4 a[U], b[U][FN];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = k + u * 256 + fc * 16;
      a[u] = ints16(wr, at, p.K);
#pragma unroll
      for (int j = 0; j < FN; ++j) b[u][j] = *(const i32x4*)(xr[j] + min(at, p.K - 16));   // behind K: any, times zeros
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[j] = mma_i8(a[u], b[u][j], acc[j]);
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

