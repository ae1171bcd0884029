// The selective scan's launches (ssm_scan.hip) and their kernels
// (ssm_scan_kernels.hpp, compiled for 4 and for 8 states a lane).
#pragma once

#include "ssm.hpp"

static constexpr int TS = 8;          // frames of a tile, and of a saved state's stretch
static constexpr int SCAN_CT = 64;    // channels of a tile: whole 128-byte lines of a bf16 row
#define LOG2E_F 1.4426950408889634f
#define LN2_F 0.6931471805599453f

struct ScanP {
  const void *x, *dt, *Bm, *Cm, *z, *dy;
  int64_t ldx, lddt, ldb, ldc, ldz, lddy;
  const float *A, *Dskip, *dtb, *h0, *dhl;
  const int32_t* lens;
  void *y, *dx, *ddt, *dB, *dC, *dz;
  int64_t ldy, lddx, ldddt, lddB, lddC, lddz;
  float *hlast, *saved, *dA, *par, *bc, *dh0;   // par: a workgroup's sums of dDskip, ddt_bias; bc: per-tile dB, dC
  // stretches of a sequence that workgroups walk side by side: what a stretch
  // adds to the state (or adjoint) behind it, the sum of its steps, and
  // the state (adjoint) that reaches it; starts is NULL where one workgroup walks it all
  float *ends, *sums, *starts;
  int T, B, D, N, G, Dg, tpg, softplus, nseg, segt;   // segt: frames of a stretch, whole tiles
};

// How a kernel reaches its rows.  FAR: 64-bit offsets and a branch per access
// that may lie outside.  PLAIN, GATED (without and with z): TS frames of every
// tensor lie within 2^31 bytes, so they go through a buffer resource over
// exactly the rows that exist; what lies outside reads as zeros and is not
// written.  (Branches and 64-bit offsets were 40 % of the kernels' instructions.)
enum { FAR, PLAIN, GATED };

// Which kernel: all of a pass over the stretches, or what their ends need.
enum ScanPass { SCAN_FWD, SCAN_ENDS, SCAN_ADJ, SCAN_BWD };
// lpc: lanes of a channel, 1, 2, 4 or 8.
void scan_launch_ns4(ScanPass pass, const ScanP& p, int lpc, int precision, int mode, unsigned blocks, hipStream_t s);
void scan_launch_ns8(ScanPass pass, const ScanP& p, int lpc, int precision, int mode, unsigned blocks, hipStream_t s);

// States [n0, n0 + W) of row `row` of a [rows][N] tensor; those it lacks are 0.
template <int W> struct States { float v[W]; };
template <int W>
__device__ __forceinline__ States<W> ld_states(const float* s, int64_t row, int N, int n0, bool on) {
  States<W> h;
#pragma unroll
  for (int j = 0; j < W; ++j) h.v[j] = 0.f;
  if (!s || !on) return h;
  s += row * N + n0;
  if (N % 4 == 0 && ((uintptr_t)s & 15) == 0) {
#pragma unroll
    for (int j = 0; j < W; j += 4)
      if (n0 + j < N) {
        const f32x4 f = *(const f32x4*)(s + j);
#pragma unroll
        for (int i = 0; i < 4; ++i) h.v[j + i] = f[i];
      }
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (n0 + j < N) h.v[j] = s[j];
  }
  return h;
}
template <int W>
__device__ __forceinline__ void st_states(float* s, int64_t row, int N, int n0, bool on, const States<W>& h) {
  if (!s || !on) return;
  s += row * N + n0;
  if (N % 4 == 0 && ((uintptr_t)s & 15) == 0) {
#pragma unroll
    for (int j = 0; j < W; j += 4)
      if (n0 + j < N) *(f32x4*)(s + j) = f32x4{h.v[j], h.v[j + 1], h.v[j + 2], h.v[j + 3]};
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (n0 + j < N) s[j] = h.v[j];
  }
}
