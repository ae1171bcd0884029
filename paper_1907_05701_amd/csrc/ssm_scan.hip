// Selective state space scan: forward, backward and the step of one frame.
//
//   s_t = softplus(dt_t + bias),  a_t[n] = exp(s_t A[n])
//   h_t[n] = a_t[n] h_{t-1}[n] + s_t x_t B_t[n]
//   o_t = sum_n C_t[n] h_t[n] + D x_t,  y_t = o_t silu(z_t)
// and with g = dy silu(z), dh_t = C_t g_t + a_{t+1} dh_{t+1}:
//   dx = s (dh.B) + D g        ds = x (dh.B) + sum_n A q,  q = dh a h_{t-1}
//   dA = sum s q   dB = sum_d dh s x   dC = sum_d g h   dz = dy o silu'(z)
//
// A workgroup owns a tile of CT adjacent channels of one group of one sequence
// and walks its frames in tiles of TS.  LPC adjacent lanes share a
// channel, each with NS = 4 of its states in registers, so N <= 4 LPC.  What
// is per channel and frame (the step, x times the step, the gate) is computed once by a thread
// that owns four adjacent channels of a frame, with 4-wide loads and stores, and goes
// through LDS to the lanes that scan.
#include <math.h>

#include <cmath>

#include "ssm.hpp"

static constexpr int TS = 16;   // frames of a tile, and of a saved state's stretch
static constexpr int NS = 4;    // states of a lane
#define LOG2E_F 1.4426950408889634f
#define LN2_F 0.6931471805599453f

template <int LPC> struct Tile {
  static constexpr int CT = LPC == 16 ? 32 : 64;   // channels
  static constexpr int NT = CT * LPC;              // threads
  static constexpr int NP = NS * LPC;              // states, padded
  static constexpr int ROW = CT / 4;               // threads of a frame's row in the 4-wide passes
  static constexpr int IT = (TS * ROW + NT - 1) / NT;
  static constexpr int BCI = (TS * NP + NT - 1) / NT;
  static constexpr int WAVES = (NT + 63) / 64;
};

struct ScanP {
  const void *x, *dt, *Bm, *Cm, *z, *dy;
  int64_t ldx, lddt, ldb, ldc, ldz, lddy;
  const float *A, *Dskip, *dtb, *h0, *dhl;
  const int32_t* lens;
  void *y, *dx, *ddt, *dB, *dC, *dz;
  int64_t ldy, lddx, ldddt, lddB, lddC, lddz;
  float *hlast, *saved, *dA, *par, *bc, *dh0;   // par: per-(sequence) sums of dDskip, ddt_bias; bc: per-tile dB, dC
  int T, B, D, N, G, Dg, tpg, softplus;
  bool vx, vdt, vz, vy, vdy, vdx, vddt, vdz;    // 4-wide accesses possible
};

struct Place {
  int g, c0, nc, b, tile;   // group, first channel, channels, sequence, tile within the group
};
template <int LPC>
__device__ __forceinline__ Place place(const ScanP& p) {
  Place q;
  const int tiles = p.G * p.tpg;
  const int t = (int)(blockIdx.x % (unsigned)tiles);
  q.b = (int)(blockIdx.x / (unsigned)tiles);
  q.g = t / p.tpg;
  q.tile = t % p.tpg;
  q.c0 = q.g * p.Dg + q.tile * Tile<LPC>::CT;
  q.nc = min(Tile<LPC>::CT, p.Dg - q.tile * Tile<LPC>::CT);
  return q;
}
__device__ __forceinline__ int length(const ScanP& p, int b) {
  return p.lens ? max(0, min(p.T, p.lens[b])) : p.T;
}

// The four states of lane `part` of channel d from a [B][D][N] tensor.
__device__ __forceinline__ f32x4 ld_state(const float* s, int64_t row, int N, int part, bool on) {
  f32x4 h{0.f, 0.f, 0.f, 0.f};
  if (s && on) {
#pragma unroll
    for (int j = 0; j < NS; ++j)
      if (part * NS + j < N) h[j] = s[row * N + part * NS + j];
  }
  return h;
}
__device__ __forceinline__ void st_state(float* s, int64_t row, int N, int part, bool on, f32x4 h) {
  if (s && on) {
#pragma unroll
    for (int j = 0; j < NS; ++j)
      if (part * NS + j < N) s[row * N + part * NS + j] = h[j];
  }
}

// B or C of a tile's frames to LDS as floats, states behind N and frames
// behind the sequence as zeros.
template <typename T, int LPC>
__device__ __forceinline__ void stage_bc(float (*dst)[Tile<LPC>::NP], const T* src, int64_t ld, const ScanP& p,
                                         const Place& q, int t0, int ns) {
  constexpr int NP = Tile<LPC>::NP;
#pragma unroll
  for (int i = 0; i < Tile<LPC>::BCI; ++i) {
    const int e = i * Tile<LPC>::NT + (int)threadIdx.x;
    const int r = e / NP, n = e % NP;
    if (r < TS) {
      float v = 0.f;
      if (r < ns && n < p.N) v = to_f32(src[((int64_t)(t0 + r) * p.B + q.b) * ld + q.g * p.N + n]);
      dst[r][n] = v;
    }
  }
}

template <typename T, int LPC>
__global__ __launch_bounds__(Tile<LPC>::NT) void ssm_scan_fwd_kernel(const ScanP p) {
  using K = Tile<LPC>;
  constexpr int CT = K::CT;
  __shared__ float sS[TS][CT], sX[TS][CT];   // the step; step times x, then y
  __shared__ float sB[TS][K::NP], sC[TS][K::NP];
  const Place q = place<LPC>(p);
  const int len = length(p, q.b);
  const int tid = threadIdx.x, part = tid % LPC, ch = tid / LPC;
  const bool on = ch < q.nc;
  const int64_t srow = (int64_t)q.b * p.D + q.c0 + ch;
  f32x4 h = ld_state(p.h0, srow, p.N, part, on);
  f32x4 A2 = ld_state(p.A, q.c0 + ch, p.N, part, on) * LOG2E_F;
  const int col = (tid % K::ROW) * 4, row0 = tid / K::ROW, nv = min(4, q.nc - col);
  f32x4 bias{0.f, 0.f, 0.f, 0.f}, skip = bias;
  for (int i = 0; i < nv; ++i) {
    if (p.dtb) bias[i] = p.dtb[q.c0 + col + i];
    if (p.Dskip) skip[i] = p.Dskip[q.c0 + col + i];
  }
  const T *x = (const T*)p.x, *dt = (const T*)p.dt, *z = (const T*)p.z;
  T* y = (T*)p.y;
  for (int t0 = 0; t0 < p.T; t0 += TS) {
    const int ns = max(0, min(TS, len - t0));
    f32x4 xs[K::IT], zs[K::IT];
#pragma unroll
    for (int i = 0; i < K::IT; ++i) {
      const int r = row0 + i * (K::NT / K::ROW);
      if (r >= TS) continue;
      f32x4 s{0.f, 0.f, 0.f, 0.f}, u = s;
      xs[i] = zs[i] = s;
      if (r < ns && nv > 0) {
        const int64_t m = (int64_t)(t0 + r) * p.B + q.b;
        xs[i] = widen(ld4_raw(x + m * p.ldx + q.c0 + col, nv, p.vx));
        s = widen(ld4_raw(dt + m * p.lddt + q.c0 + col, nv, p.vdt)) + bias;
        if (p.z) zs[i] = widen(ld4_raw(z + m * p.ldz + q.c0 + col, nv, p.vz));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (p.softplus) s[j] = softplusf_(s[j]);
          u[j] = s[j] * xs[i][j];
        }
      }
      *(f32x4*)&sS[r][col] = s;
      *(f32x4*)&sX[r][col] = u;
    }
    stage_bc<T, LPC>(sB, (const T*)p.Bm, p.ldb, p, q, t0, ns);
    stage_bc<T, LPC>(sC, (const T*)p.Cm, p.ldc, p, q, t0, ns);
    __syncthreads();
    if (p.saved && on)
      *(f32x4*)(p.saved + (((int64_t)(t0 / TS) * p.B + q.b) * p.D + q.c0 + ch) * K::NP + part * NS) = h;
    for (int r = 0; r < ns; ++r) {
      const float s = sS[r][ch], u = sX[r][ch];
      const f32x4 Bv = *(const f32x4*)&sB[r][part * NS], Cv = *(const f32x4*)&sC[r][part * NS];
      float o = 0.f;
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        h[j] = __builtin_amdgcn_exp2f(s * A2[j]) * h[j] + u * Bv[j];
        o += Cv[j] * h[j];
      }
      o = group_sum<LPC>(o);
      if (part == 0) sX[r][ch] = o;   // read by this group only, above
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K::IT; ++i) {
      const int r = row0 + i * (K::NT / K::ROW);
      if (r >= TS || t0 + r >= p.T || nv <= 0) continue;
      f32x4 o{0.f, 0.f, 0.f, 0.f};
      if (r < ns) {
        o = *(const f32x4*)&sX[r][col] + skip * xs[i];
        if (p.z) {
#pragma unroll
          for (int j = 0; j < 4; ++j) o[j] *= siluf_(zs[i][j]);
        }
      }
      st4(y + ((int64_t)(t0 + r) * p.B + q.b) * p.ldy + q.c0 + col, o, nv, p.vy);
    }
  }
  st_state(p.hlast, srow, p.N, part, on, h);
}

// Backward.  Tiles in reverse; each tile recomputes its states from the
// saved one into registers (TS + 1 of them, 4 states each) and then runs the
// adjoint from its last frame to its first.  dB and dC are sums over
// channels: a wave adds its channels by swaps between rows of lanes, the waves
// meet in LDS, the tiles of a group in a second launch.
template <typename T, int LPC>
__global__ __launch_bounds__(Tile<LPC>::NT) void ssm_scan_bwd_kernel(const ScanP p) {
  using K = Tile<LPC>;
  constexpr int CT = K::CT, NP = K::NP;
  __shared__ float sS[TS][CT], sX[TS][CT], sG[TS][CT], sY[TS][CT];
  __shared__ float sB[TS][NP], sC[TS][NP];
  __shared__ float red[K::WAVES][TS][2 * NP];
  const Place q = place<LPC>(p);
  const int len = length(p, q.b);
  const int tid = threadIdx.x, part = tid % LPC, ch = tid / LPC, lane = tid & 63, wave = tid >> 6;
  const bool on = ch < q.nc;
  const int64_t srow = (int64_t)q.b * p.D + q.c0 + ch;
  const f32x4 A2 = ld_state(p.A, q.c0 + ch, p.N, part, on) * LOG2E_F;
  f32x4 dh = ld_state(p.dhl, srow, p.N, part, on);   // the adjoint that reaches the frames before
  f32x4 dA{0.f, 0.f, 0.f, 0.f};
  const int col = (tid % K::ROW) * 4, row0 = tid / K::ROW, nv = min(4, q.nc - col);
  f32x4 bias{0.f, 0.f, 0.f, 0.f}, skip = bias, dD = bias, db = bias;
  for (int i = 0; i < nv; ++i) {
    if (p.dtb) bias[i] = p.dtb[q.c0 + col + i];
    if (p.Dskip) skip[i] = p.Dskip[q.c0 + col + i];
  }
  const T *x = (const T*)p.x, *dt = (const T*)p.dt, *z = (const T*)p.z, *dy = (const T*)p.dy;
  for (int t0 = (p.T - 1) / TS * TS; t0 >= 0; t0 -= TS) {
    const int ns = max(0, min(TS, len - t0));
    f32x4 xs[K::IT], vs[K::IT], zs[K::IT], ys[K::IT];
#pragma unroll
    for (int i = 0; i < K::IT; ++i) {
      const int r = row0 + i * (K::NT / K::ROW);
      if (r >= TS) continue;
      f32x4 s{0.f, 0.f, 0.f, 0.f}, u = s, g = s;
      xs[i] = vs[i] = zs[i] = ys[i] = s;
      if (r < ns && nv > 0) {
        const int64_t m = (int64_t)(t0 + r) * p.B + q.b;
        xs[i] = widen(ld4_raw(x + m * p.ldx + q.c0 + col, nv, p.vx));
        vs[i] = widen(ld4_raw(dt + m * p.lddt + q.c0 + col, nv, p.vdt)) + bias;
        ys[i] = widen(ld4_raw(dy + m * p.lddy + q.c0 + col, nv, p.vdy));
        if (p.z) zs[i] = widen(ld4_raw(z + m * p.ldz + q.c0 + col, nv, p.vz));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[j] = p.softplus ? softplusf_(vs[i][j]) : vs[i][j];
          u[j] = s[j] * xs[i][j];
          g[j] = p.z ? ys[i][j] * siluf_(zs[i][j]) : ys[i][j];
        }
      }
      *(f32x4*)&sS[r][col] = s;
      *(f32x4*)&sX[r][col] = u;
      *(f32x4*)&sG[r][col] = g;
    }
    stage_bc<T, LPC>(sB, (const T*)p.Bm, p.ldb, p, q, t0, ns);
    stage_bc<T, LPC>(sC, (const T*)p.Cm, p.ldc, p, q, t0, ns);
    __syncthreads();
    f32x4 hist[TS + 1];
    hist[0] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (on) hist[0] = *(const f32x4*)(p.saved + (((int64_t)(t0 / TS) * p.B + q.b) * p.D + q.c0 + ch) * NP + part * NS);
#pragma unroll
    for (int r = 0; r < TS; ++r) {
      hist[r + 1] = hist[r];
      if (r < ns) {
        const float s = sS[r][ch], u = sX[r][ch];
        const f32x4 Bv = *(const f32x4*)&sB[r][part * NS];
#pragma unroll
        for (int j = 0; j < NS; ++j) hist[r + 1][j] = __builtin_amdgcn_exp2f(s * A2[j]) * hist[r][j] + u * Bv[j];
        if (p.z) {
          const f32x4 Cv = *(const f32x4*)&sC[r][part * NS];
          float o = 0.f;
#pragma unroll
          for (int j = 0; j < NS; ++j) o += Cv[j] * hist[r + 1][j];
          o = group_sum<LPC>(o);
          if (part == 0) sY[r][ch] = o;
        }
      }
    }
#pragma unroll
    for (int r = TS - 1; r >= 0; --r) {
      if (r < ns) {
        const float s = sS[r][ch], u = sX[r][ch], g = sG[r][ch];
        const f32x4 Bv = *(const f32x4*)&sB[r][part * NS], Cv = *(const f32x4*)&sC[r][part * NS];
        float v[2 * NS], into = 0.f, da = 0.f;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          const float d = dh[j] + Cv[j] * g;
          v[j] = d * u;                       // dB
          v[NS + j] = hist[r + 1][j] * g;     // dC
          into += d * Bv[j];
          dh[j] = d * __builtin_amdgcn_exp2f(s * A2[j]);
          const float qa = dh[j] * hist[r][j];
          da += qa * A2[j];
          dA[j] += qa * s;
        }
        into = group_sum<LPC>(into);
        da = group_sum<LPC>(da);
        if (part == 0) {
          sX[r][ch] = into;
          sS[r][ch] = da * LN2_F;
        }
        // over the wave's channels: rows of lanes first (each swap halves the
        // values a lane holds), then the channels within a row.  Lanes of rows
        // 0, 1 end with dB, of 2, 3 with dC; even rows with states 0, 1 of
        // their lane's four and odd ones with 2, 3.  Fewer than 64 lanes: one channel group
        float w[NS], o2[2];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
          const auto e = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[j]), __float_as_uint(v[NS + j]), false, false);
          w[j] = __uint_as_float(e[0]) + __uint_as_float(e[1]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const auto e = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[j]), __float_as_uint(w[2 + j]), false, false);
          o2[j] = stride_sum<LPC>(__uint_as_float(e[0]) + __uint_as_float(e[1]));
        }
        if ((lane & 15) < LPC) {
          float* o = &red[wave][r][(lane >> 5) * NP + part * NS + ((lane >> 4) & 1) * 2];
          o[0] = o2[0];
          o[1] = o2[1];
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K::IT; ++i) {
      const int r = row0 + i * (K::NT / K::ROW);
      if (r >= TS || t0 + r >= p.T || nv <= 0) continue;
      const int64_t m = (int64_t)(t0 + r) * p.B + q.b;
      f32x4 gx{0.f, 0.f, 0.f, 0.f}, gt = gx, gz = gx;
      if (r < ns) {
        const f32x4 into = *(const f32x4*)&sX[r][col], da = *(const f32x4*)&sS[r][col];
        const f32x4 g = *(const f32x4*)&sG[r][col];
        const f32x4 o = p.z ? *(const f32x4*)&sY[r][col] : gx;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float s = p.softplus ? softplusf_(vs[i][j]) : vs[i][j];
          gx[j] = s * into[j] + skip[j] * g[j];
          const float ds = xs[i][j] * into[j] + da[j];
          gt[j] = p.softplus ? ds * sigmoidf_(vs[i][j]) : ds;
          if (p.z) gz[j] = ys[i][j] * (o[j] + skip[j] * xs[i][j]) * dsiluf_(zs[i][j]);
          dD[j] += g[j] * xs[i][j];
          db[j] += gt[j];
        }
      }
      st4((T*)p.dx + m * p.lddx + q.c0 + col, gx, nv, p.vdx);
      st4((T*)p.ddt + m * p.ldddt + q.c0 + col, gt, nv, p.vddt);
      if (p.z) st4((T*)p.dz + m * p.lddz + q.c0 + col, gz, nv, p.vdz);
    }
    // the waves' dB and dC, in wave order
    for (int e = tid; e < TS * 2 * NP; e += K::NT) {
      const int r = e / (2 * NP), c = e % (2 * NP), n = c % NP;
      if (t0 + r >= p.T || n >= p.N) continue;
      float v = 0.f;
      if (r < ns) {
#pragma unroll
        for (int w = 0; w < K::WAVES; ++w) v += red[w][r][c];
      }
      const int64_t m = (int64_t)(t0 + r) * p.B + q.b;
      if (p.bc) {
        p.bc[(((int64_t)q.tile * p.T * p.B + m) * p.G + q.g) * 2 * p.N + (c / NP) * p.N + n] = v;
      } else if (c < NP) {
        ((T*)p.dB)[m * p.lddB + q.g * p.N + n] = from_f32<T>(v);
      } else {
        ((T*)p.dC)[m * p.lddC + q.g * p.N + n] = from_f32<T>(v);
      }
    }
    __syncthreads();
  }
  st_state(p.dA, srow, p.N, part, on, dA);
  st_state(p.dh0, srow, p.N, part, on, dh);
  // dDskip and ddt_bias: the rows of threads that share a column, in row order
  constexpr int ROWS = K::NT / K::ROW;
  f32x4* r4 = (f32x4*)&sS[0][0];   // TS * CT floats hold TS rows of columns
  for (int k = 0; k < 2; ++k) {
    if (row0 < TS) r4[row0 * K::ROW + tid % K::ROW] = k ? db : dD;
    __syncthreads();
    if (row0 == 0) {
      f32x4 v{0.f, 0.f, 0.f, 0.f};
      for (int r = 0; r < (ROWS < TS ? ROWS : TS); ++r) v += r4[r * K::ROW + tid];
      for (int j = 0; j < nv; ++j) p.par[((int64_t)q.b * 2 + k) * p.D + q.c0 + col + j] = v[j];
    }
    __syncthreads();
  }
}

// Sums of the backward's partials: dB and dC over the tiles of a group; dA,
// dDskip and ddt_bias over the sequences.
struct ScanSum {
  const float *bc, *dA, *par;
  void *dB, *dC;
  int64_t lddB, lddC;
  float *oA, *oD, *ob;
  int tpg, G, N, D, rows;
  int64_t M, nbc;   // rows of dB; elements of dB and dC together (0: written already)
  int64_t blocks_bc;
};
template <typename T>
__global__ __launch_bounds__(256) void ssm_scan_sum_kernel(const ScanSum p) {
  if ((int64_t)blockIdx.x < p.blocks_bc) {
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= p.nbc) return;
    float v = 0.f;
    for (int t = 0; t < p.tpg; ++t) v += p.bc[t * p.nbc + e];
    const int c = (int)(e % (2 * p.N)), n = c % p.N;
    const int64_t mg = e / (2 * p.N), m = mg / p.G;
    const int g = (int)(mg % p.G);
    if (c < p.N) ((T*)p.dB)[m * p.lddB + g * p.N + n] = from_f32<T>(v);
    else ((T*)p.dC)[m * p.lddC + g * p.N + n] = from_f32<T>(v);
    return;
  }
  // 16 columns a workgroup, 16 row ranges summed in order and then in range order
  __shared__ float sh[16][17];
  const int64_t nA = (int64_t)p.D * p.N, cols = nA + 2 * p.D;
  const int cl = threadIdx.x & 15, rg = threadIdx.x >> 4;
  const int64_t c = ((int64_t)blockIdx.x - p.blocks_bc) * 16 + cl;
  const int per = (p.rows + 15) / 16, r0 = rg * per, r1 = min(p.rows, r0 + per);
  float v = 0.f;
  if (c < cols) {
    const float* src = c < nA ? p.dA + c : p.par + (c - nA);
    const int64_t st = c < nA ? nA : 2 * p.D;
#pragma unroll 8
    for (int r = r0; r < r1; ++r) v += src[r * st];
  }
  sh[rg][cl] = v;
  __syncthreads();
  if (rg == 0 && c < cols) {
    float t = 0.f;
    for (int i = 0; i < 16; ++i) t += sh[i][cl];
    if (c < nA) p.oA[c] = t;
    else if (c < nA + p.D) { if (p.oD) p.oD[c - nA] = t; }
    else if (p.ob) p.ob[c - nA - p.D] = t;
  }
}

// One frame of B streams: LPC lanes a channel as above, the state read and
// written once.
template <typename T, int LPC>
__global__ __launch_bounds__(256) void ssm_scan_step_kernel(const ScanP p, const int32_t* __restrict__ slots,
                                                            int n_slots, float* state) {
  constexpr int CH = 256 / LPC;   // channels of a workgroup
  const int tiles = (p.D + CH - 1) / CH;
  const int b = (int)(blockIdx.x / (unsigned)tiles), d = (int)(blockIdx.x % (unsigned)tiles) * CH + threadIdx.x / LPC;
  const int part = threadIdx.x % LPC;
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
  if (d >= p.D) return;
  float o = 0.f, xv = 0.f;
  if (slot >= 0) {
    const int g = d / p.Dg;
    xv = to_f32(((const T*)p.x)[(int64_t)b * p.ldx + d]);
    float s = to_f32(((const T*)p.dt)[(int64_t)b * p.lddt + d]) + (p.dtb ? p.dtb[d] : 0.f);
    if (p.softplus) s = softplusf_(s);
    const float u = s * xv;
    const int64_t row = (int64_t)slot * p.D + d;
    f32x4 h = ld_state(state, row, p.N, part, true);
    const f32x4 A = ld_state(p.A, d, p.N, part, true);
    const T* Bm = (const T*)p.Bm + (int64_t)b * p.ldb + g * p.N;
    const T* Cm = (const T*)p.Cm + (int64_t)b * p.ldc + g * p.N;
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      const int n = part * NS + j;
      const float Bv = n < p.N ? to_f32(Bm[n]) : 0.f, Cv = n < p.N ? to_f32(Cm[n]) : 0.f;
      h[j] = __builtin_amdgcn_exp2f(s * LOG2E_F * A[j]) * h[j] + u * Bv;
      o += Cv * h[j];
    }
    st_state(state, row, p.N, part, true, h);
  }
  o = group_sum<LPC>(o);
  if (part == 0) {
    if (slot >= 0) {
      if (p.Dskip) o += p.Dskip[d] * xv;
      if (p.z) o *= siluf_(to_f32(((const T*)p.z)[(int64_t)b * p.ldz + d]));
    }
    ((T*)p.y)[(int64_t)b * p.ldy + d] = from_f32<T>(o);
  }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
int ssm_check_dims(const ssm_dims* d, const char* fn) {
  if (!d) return blstm_fail(BLSTM_EINVAL, "%s: null dims", fn);
  if (d->T < 1 || d->B < 1 || d->D < 1 || d->N < 1 || d->G < 1 || d->W < 1)
    return blstm_fail(BLSTM_EINVAL, "%s: all dims must be positive (T=%d B=%d D=%d N=%d G=%d W=%d)", fn, d->T, d->B,
                      d->D, d->N, d->G, d->W);
  if (d->precision != BLSTM_FP32 && d->precision != BLSTM_BF16)
    return blstm_fail(BLSTM_EINVAL, "%s: precision must be BLSTM_FP32 or BLSTM_BF16", fn);
  if (d->D % d->G) return blstm_fail(BLSTM_EINVAL, "%s: G=%d does not divide D=%d", fn, d->G, d->D);
  if (d->N > 64) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: N > 64", fn);
  if (d->W > 8) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: W > 8", fn);
  if (d->D > (1 << 20)) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: D > 2^20", fn);
  if ((int64_t)d->T * d->B > (1 << 24)) return blstm_fail(BLSTM_EUNSUPPORTED, "%s: T*B too large", fn);
  return BLSTM_OK;
}

static int lanes_of(int N) { return N <= 4 ? 1 : N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }
static size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

struct ScanPlan {
  int lpc, ct, np, tpg;
  int64_t blocks;
  size_t saved, bc, dA, par, bwd;   // bytes; bc, dA, par in this order in the backward's scratch
};
static int scan_plan(const ssm_dims* d, ScanPlan* o) {
  o->lpc = lanes_of(d->N);
  o->ct = o->lpc == 16 ? 32 : 64;
  o->np = NS * o->lpc;
  o->tpg = (int)cdiv(d->D / d->G, o->ct);
  o->blocks = (int64_t)d->B * d->G * o->tpg;
  if (o->blocks > 0x7fffffff) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan: B*D too large");
  o->saved = (size_t)cdiv(d->T, TS) * d->B * d->D * o->np * 4;
  o->bc = o->tpg > 1 ? up256((size_t)o->tpg * d->T * d->B * d->G * 2 * d->N * 4) : 0;
  o->dA = up256((size_t)d->B * d->D * d->N * 4);
  o->par = up256((size_t)d->B * 2 * d->D * 4);
  o->bwd = o->bc + o->dA + o->par;
  return BLSTM_OK;
}

size_t ssm_conv_bwd_bytes(const ssm_dims* d);

extern "C" int ssm_workspace_bytes(const ssm_dims* dims, size_t* saved, size_t* fwd, size_t* bwd, size_t* conv_bwd) {
  ScanPlan pl;
  int rc = ssm_check_dims(dims, "ssm_workspace_bytes");
  if (!rc) rc = scan_plan(dims, &pl);
  if (rc) return rc;
  if (saved) *saved = pl.saved;
  if (fwd) *fwd = 0;
  if (bwd) *bwd = pl.bwd;
  if (conv_bwd) *conv_bwd = ssm_conv_bwd_bytes(dims);
  return BLSTM_OK;
}

// Whether rows of this tensor can be read four elements at a time: base and
// pitch, and the groups' first channels, are multiples of four.
static bool four(const ssm_dims* d, const void* p, int64_t ld, size_t es) {
  return ((uintptr_t)p % (4 * es)) == 0 && ld % 4 == 0 && (d->G == 1 || (d->D / d->G) % 4 == 0);
}

static int scan_in(const ssm_dims* d, const ssm_scan_in* in, const char* fn, ScanP* p) {
  if (!in || !in->x || !in->dt || !in->Bm || !in->Cm || !in->A) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (in->flags & ~(uint32_t)SSM_SOFTPLUS) return blstm_fail(BLSTM_EINVAL, "%s: unknown flags", fn);
  const int64_t bcw = (int64_t)d->G * d->N;
  if (in->ldx < d->D || in->lddt < d->D || in->ldb < bcw || in->ldc < bcw || (in->z && in->ldz < d->D))
    return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  const size_t es = d->precision == BLSTM_BF16 ? 2 : 4;
  *p = ScanP{};
  p->x = in->x; p->dt = in->dt; p->Bm = in->Bm; p->Cm = in->Cm; p->z = in->z;
  p->ldx = in->ldx; p->lddt = in->lddt; p->ldb = in->ldb; p->ldc = in->ldc; p->ldz = in->ldz;
  p->A = in->A; p->Dskip = in->Dskip; p->dtb = in->dt_bias; p->h0 = in->h0; p->lens = in->lens;
  p->T = d->T; p->B = d->B; p->D = d->D; p->N = d->N; p->G = d->G; p->Dg = d->D / d->G;
  p->softplus = in->flags & SSM_SOFTPLUS;
  p->vx = four(d, in->x, in->ldx, es);
  p->vdt = four(d, in->dt, in->lddt, es);
  p->vz = in->z && four(d, in->z, in->ldz, es);
  return BLSTM_OK;
}

#define SCAN_BY_LANES(T, LAUNCH)                                     \
  switch (pl.lpc) {                                                  \
    case 1: LAUNCH(T, 1); break;                                     \
    case 2: LAUNCH(T, 2); break;                                     \
    case 4: LAUNCH(T, 4); break;                                     \
    case 8: LAUNCH(T, 8); break;                                     \
    default: LAUNCH(T, 16); break;                                   \
  }
#define SCAN_DISPATCH(LAUNCH)                                        \
  if (dims->precision == BLSTM_BF16) { SCAN_BY_LANES(bf16, LAUNCH) } \
  else { SCAN_BY_LANES(float, LAUNCH) }

extern "C" int ssm_scan_fwd(const ssm_dims* dims, const ssm_scan_in* in, void* y, int64_t ldy, float* h_last,
                            void* saved, void* ws, hipStream_t stream) {
  ScanPlan pl;
  ScanP p;
  int rc = ssm_check_dims(dims, "ssm_scan_fwd");
  if (!rc) rc = scan_plan(dims, &pl);
  if (!rc) rc = scan_in(dims, in, "ssm_scan_fwd", &p);
  if (rc) return rc;
  if (!y) return blstm_fail(BLSTM_EINVAL, "ssm_scan_fwd: NULL pointer");
  if (ldy < dims->D) return blstm_fail(BLSTM_EINVAL, "ssm_scan_fwd: a row pitch is below its row");
  p.y = y; p.ldy = ldy; p.hlast = h_last; p.saved = (float*)saved; p.tpg = pl.tpg;
  p.vy = four(dims, y, ldy, dims->precision == BLSTM_BF16 ? 2 : 4);
  (void)ws;
#define FWD(T, L) \
  BLSTM_LAUNCH("ssm_scan_fwd", (ssm_scan_fwd_kernel<T, L>), dim3((unsigned)pl.blocks), dim3(Tile<L>::NT), 0, stream, p)
  SCAN_DISPATCH(FWD)
  return blstm_check_launch("ssm_scan_fwd");
}

extern "C" int ssm_scan_bwd(const ssm_dims* dims, const ssm_scan_in* in, const void* dy, int64_t lddy,
                            const float* dh_last, const void* saved, const ssm_scan_grads* out, void* ws,
                            hipStream_t stream) {
  ScanPlan pl;
  ScanP p;
  int rc = ssm_check_dims(dims, "ssm_scan_bwd");
  if (!rc) rc = scan_plan(dims, &pl);
  if (!rc) rc = scan_in(dims, in, "ssm_scan_bwd", &p);
  if (rc) return rc;
  if (!dy || !saved || !ws || !out || !out->dx || !out->ddt || !out->dBm || !out->dCm || !out->dA || (in->z && !out->dz))
    return blstm_fail(BLSTM_EINVAL, "ssm_scan_bwd: NULL pointer");
  const int64_t bcw = (int64_t)dims->G * dims->N;
  if (lddy < dims->D || out->lddx < dims->D || out->ldddt < dims->D || out->lddb < bcw || out->lddc < bcw ||
      (in->z && out->lddz < dims->D))
    return blstm_fail(BLSTM_EINVAL, "ssm_scan_bwd: a row pitch is below its row");
  const size_t es = dims->precision == BLSTM_BF16 ? 2 : 4;
  char* w = (char*)ws;
  p.dy = dy; p.lddy = lddy; p.dhl = dh_last; p.saved = (float*)saved;
  p.dx = out->dx; p.ddt = out->ddt; p.dB = out->dBm; p.dC = out->dCm; p.dz = out->dz;
  p.lddx = out->lddx; p.ldddt = out->ldddt; p.lddB = out->lddb; p.lddC = out->lddc; p.lddz = out->lddz;
  p.dh0 = out->dh0;
  p.bc = pl.bc ? (float*)w : nullptr;
  p.dA = (float*)(w + pl.bc);
  p.par = (float*)(w + pl.bc + pl.dA);
  p.tpg = pl.tpg;
  p.vdy = four(dims, dy, lddy, es);
  p.vdx = four(dims, out->dx, out->lddx, es);
  p.vddt = four(dims, out->ddt, out->ldddt, es);
  p.vdz = in->z && four(dims, out->dz, out->lddz, es);
#define BWD(T, L) \
  BLSTM_LAUNCH("ssm_scan_bwd", (ssm_scan_bwd_kernel<T, L>), dim3((unsigned)pl.blocks), dim3(Tile<L>::NT), 0, stream, p)
  SCAN_DISPATCH(BWD)
  ScanSum s{};
  s.bc = p.bc; s.dA = p.dA; s.par = p.par;
  s.dB = p.dB; s.dC = p.dC; s.lddB = p.lddB; s.lddC = p.lddC;
  s.oA = out->dA; s.oD = out->dDskip; s.ob = out->ddt_bias;
  s.tpg = pl.tpg; s.G = dims->G; s.N = dims->N; s.D = dims->D; s.rows = dims->B;
  s.M = (int64_t)dims->T * dims->B;
  s.nbc = pl.bc ? s.M * dims->G * 2 * dims->N : 0;
  s.blocks_bc = cdiv(s.nbc, 256);
  const int64_t nb = s.blocks_bc + cdiv((int64_t)dims->D * (dims->N + 2), 16);
  if (nb > 0x7fffffff) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan_bwd: T*B*G*N too large");
  if (es == 2) BLSTM_LAUNCH("ssm_scan_sum", ssm_scan_sum_kernel<bf16>, dim3((unsigned)nb), dim3(256), 0, stream, s);
  else BLSTM_LAUNCH("ssm_scan_sum", ssm_scan_sum_kernel<float>, dim3((unsigned)nb), dim3(256), 0, stream, s);
  return blstm_check_launch("ssm_scan_bwd");
}

extern "C" int ssm_scan_step(const ssm_dims* dims, const ssm_scan_in* in, const int32_t* slots, int32_t n_slots,
                             float* state, void* y, int64_t ldy, hipStream_t stream) {
  ScanPlan pl;
  ScanP p;
  int rc = ssm_check_dims(dims, "ssm_scan_step");
  if (!rc) rc = scan_plan(dims, &pl);
  if (!rc) rc = scan_in(dims, in, "ssm_scan_step", &p);
  if (rc) return rc;
  if (!state || !y) return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: NULL pointer");
  if (dims->T != 1) return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: T must be 1");
  if (n_slots < 1 || (!slots && n_slots < dims->B))
    return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: %d slots for %d streams", n_slots, dims->B);
  if (ldy < dims->D) return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: a row pitch is below its row");
  p.y = y; p.ldy = ldy;
  const int64_t blocks = (int64_t)dims->B * cdiv(dims->D, 256 / pl.lpc);
  if (blocks > 0x7fffffff) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan_step: B*D too large");
#define STEP(T, L) \
  BLSTM_LAUNCH("ssm_scan_step", (ssm_scan_step_kernel<T, L>), dim3((unsigned)blocks), dim3(256), 0, stream, p, slots, n_slots, state)
  SCAN_DISPATCH(STEP)
  return blstm_check_launch("ssm_scan_step");
}
