// Selective state space scan: forward, backward and the step of one frame.
//
//   s_t = softplus(dt_t + bias),  a_t[n] = exp(s_t A[n])
//   h_t[n] = a_t[n] h_{t-1}[n] + s_t x_t B_t[n]
//   o_t = sum_n C_t[n] h_t[n] + D x_t,  y_t = o_t silu(z_t)
// and with g = dy silu(z), dh_t = C_t g_t + a_{t+1} dh_{t+1}:
//   dx = s (dh.B) + D g        ds = x (dh.B) + sum_n A q,  q = dh a h_{t-1}
//   dA = sum s q   dB = sum_d dh s x   dC = sum_d g h   dz = dy o silu'(z)
//
// A workgroup owns a tile of CT adjacent channels of one group of one
// sequence and walks its frames in tiles of TS.  LPC adjacent lanes share a
// channel, each with NS = 8 of its states in registers, so N <= 8 LPC.  What is per channel and
// frame (the step, the gate, the outputs) is computed once, by the lane whose
// turn the frame is (frame r of a tile: lane r % LPC), and reaches the others as
// a DPP operand: no activation goes through LDS.  B and C, which every channel of the
// group shares, do, staged a tile ahead.
//
// The vector unit bounds these kernels (N = 16: an exponential, three
// multiply-adds and a product a state and frame forward, three times that
// backward), so what is beside the states is kept small.
#include <math.h>

#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "dma.hpp"
#include "ssm.hpp"

static constexpr int TS = 8;    // frames of a tile, and of a saved state's stretch
static constexpr int NS = 8;    // states of a lane
#define LOG2E_F 1.4426950408889634f
#define LN2_F 0.6931471805599453f

template <int LPC> struct Tile {
  static constexpr int CT = 64;                       // channels: whole 128-byte lines of a bf16 row
  static constexpr int NT = CT * LPC;                 // threads
  static constexpr int NP = NS * LPC;                 // states, padded
  static constexpr int FL = (TS + LPC - 1) / LPC;     // frames of a tile that are a lane's
  static constexpr int BCI = (TS * NP + NT - 1) / NT; // elements of B of a tile that a thread stages
};
static_assert(TS % 8 == 0, "frames of a tile in whole turns of up to 8 lanes");

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

struct Place {
  int g, c0, nc, b, tile;   // group, first channel, channels, sequence, tile within the group
  int seg, t0, t1;          // stretch and its frames
};
template <int LPC>
__device__ __forceinline__ Place place(const ScanP& p, int first) {
  Place q;
  const int tiles = p.G * p.tpg;
  const int t = (int)(blockIdx.x % (unsigned)tiles);
  const unsigned r = blockIdx.x / (unsigned)tiles;
  q.b = (int)(r % (unsigned)p.B);
  q.seg = (int)(r / (unsigned)p.B) + first;
  q.t0 = q.seg * p.segt;
  q.t1 = min(p.T, q.t0 + p.segt);
  q.g = t / p.tpg;
  q.tile = t % p.tpg;
  q.c0 = q.g * p.Dg + q.tile * Tile<LPC>::CT;
  q.nc = min(Tile<LPC>::CT, p.Dg - q.tile * Tile<LPC>::CT);
  return q;
}
__device__ __forceinline__ int length(const ScanP& p, int b) {
  return p.lens ? max(0, min(p.T, p.lens[b])) : p.T;
}

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
// The same in a [stretch][B][D][NP] scratch tensor, where a workgroup's are adjacent.
template <int LPC>
__device__ __forceinline__ float* lane_states(float* s, const ScanP& p, int seg, const Place& q) {
  return s + (((int64_t)seg * p.B + q.b) * p.D + q.c0) * Tile<LPC>::NP + threadIdx.x * NS;
}
__device__ __forceinline__ States<NS> ld_scratch(const float* s) {
  States<NS> h;
#pragma unroll
  for (int j = 0; j < NS; j += 4) {
    const f32x4 f = *(const f32x4*)(s + j);
#pragma unroll
    for (int i = 0; i < 4; ++i) h.v[j + i] = f[i];
  }
  return h;
}
__device__ __forceinline__ void st_scratch(float* s, const States<NS>& h) {
#pragma unroll
  for (int j = 0; j < NS; j += 4) *(f32x4*)(s + j) = f32x4{h.v[j], h.v[j + 1], h.v[j + 2], h.v[j + 3]};
}

// How a kernel reaches its rows.  FAR: 64-bit offsets and a branch per access
// that may lie outside.  PLAIN, GATED (without and with z): TS frames of every
// tensor lie within 2^31 bytes, so they go through a buffer resource over
// exactly the rows that exist; what lies outside reads as zeros and is not
// written.  (Branches and 64-bit offsets were 40 % of the kernels' instructions.)
enum { FAR, PLAIN, GATED };

// Rows of a frame-major tensor for one sequence: from frame t on, from column j0.
template <typename T>
__device__ __forceinline__ T* frame_row(const void* base, int64_t ld, const ScanP& p, const Place& q, int t, int j0) {
  return (T*)base + ((int64_t)t * p.B + q.b) * ld + j0;
}
// Byte offset of column j of row r (j < w, else outside).
__device__ __forceinline__ uint32_t row_off(int row_bytes, int r, int j, int w, int es) {
  return j < w ? (uint32_t)(r * row_bytes + j * es) : DMA_OFF_NONE;
}
// A resource over `rows` rows, w elements of the last one.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const T* row, int row_bytes, int rows, int w) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)row, (short)0, rows > 0 ? (rows - 1) * row_bytes + w * (int)sizeof(T) : 0,
                                           0x00020000);
}
__device__ __forceinline__ void buf_load(bf16& v, __amdgpu_buffer_rsrc_t r, uint32_t off) {
  v = __builtin_bit_cast(bf16, (short)__builtin_amdgcn_raw_buffer_load_b16(r, (int)off, 0, 0));
}
__device__ __forceinline__ void buf_load(float& v, __amdgpu_buffer_rsrc_t r, uint32_t off) {
  v = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, (int)off, 0, 0));
}
__device__ __forceinline__ void buf_store(bf16 v, __amdgpu_buffer_rsrc_t r, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(short, v), r, (int)off, 0, 0);
}
__device__ __forceinline__ void buf_store(float v, __amdgpu_buffer_rsrc_t r, uint32_t off) {
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, (int)off, 0, 0);
}

// B or C of a tile's frames: the thread's elements, states behind N and frames
// behind the sequence as zeros; then to LDS as floats.
template <typename T, int LPC> struct BcRegs { T v[Tile<LPC>::BCI]; };
template <int MODE, typename T, int LPC>
__device__ __forceinline__ void load_bc(BcRegs<T, LPC>& o, const void* src, int64_t ld, const ScanP& p, const Place& q,
                                        int t0, int ns) {
  const T* row = frame_row<const T>(src, ld, p, q, t0, q.g * p.N);
  const int rb = p.B * (int)ld * (int)sizeof(T);
  const __amdgpu_buffer_rsrc_t rs = rows_rsrc(row, rb, ns, p.N);
#pragma unroll
  for (int i = 0; i < Tile<LPC>::BCI; ++i) {
    const int e = i * Tile<LPC>::NT + (int)threadIdx.x;
    const int r = e / Tile<LPC>::NP, n = e % Tile<LPC>::NP;
    if constexpr (MODE == FAR) {
      o.v[i] = (T)0.f;
      if (r < ns && n < p.N) o.v[i] = row[(int64_t)r * p.B * ld + n];
    } else {
      buf_load(o.v[i], rs, row_off(rb, r, n, p.N, sizeof(T)));
    }
  }
}
template <typename T, int LPC>
__device__ __forceinline__ void store_bc(float (*dst)[Tile<LPC>::NP], const BcRegs<T, LPC>& o) {
#pragma unroll
  for (int i = 0; i < Tile<LPC>::BCI; ++i) {
    const int e = i * Tile<LPC>::NT + (int)threadIdx.x;
    if (e < TS * Tile<LPC>::NP) dst[e / Tile<LPC>::NP][e % Tile<LPC>::NP] = to_f32(o.v[i]);
  }
}
// A lane's eight states' values of a staged row.
__device__ __forceinline__ States<NS> row_states(const float* r) { return ld_scratch(r); }

// The lane's channel at its frames of a tile (frame i * LPC + part), as it
// lies in memory; zeros behind the end and beside the channels.
template <typename T, int LPC> struct Own { T v[Tile<LPC>::FL]; };
template <int MODE, typename T, int LPC>
__device__ __forceinline__ void load_own(Own<T, LPC>& o, const void* src, int64_t ld, const ScanP& p, const Place& q,
                                         int t0, int ns, int part, int ch) {
  const T* row = frame_row<const T>(src, ld, p, q, t0, q.c0);
  const int rb = p.B * (int)ld * (int)sizeof(T);
  const __amdgpu_buffer_rsrc_t rs = rows_rsrc(row, rb, ns, q.nc);
  const uint32_t off = row_off(rb, part, ch, q.nc, sizeof(T));
#pragma unroll
  for (int i = 0; i < Tile<LPC>::FL; ++i) {
    if constexpr (MODE == FAR) {
      o.v[i] = (T)0.f;
      if (i * LPC + part < ns && ch < q.nc) o.v[i] = row[(int64_t)(i * LPC + part) * p.B * ld + ch];
    } else {
      buf_load(o.v[i], rs, off + i * LPC * rb);
    }
  }
}
// The same to memory: every frame of the stretch.
template <int MODE, typename T, int LPC>
__device__ __forceinline__ void store_own(void* dst, int64_t ld, const ScanP& p, const Place& q, int t0, int part, int ch,
                                          const float (&v)[Tile<LPC>::FL]) {
  T* row = frame_row<T>(dst, ld, p, q, t0, q.c0);
  const int rb = p.B * (int)ld * (int)sizeof(T);
  const __amdgpu_buffer_rsrc_t rs = rows_rsrc(row, rb, min(TS, q.t1 - t0), q.nc);
  const uint32_t off = row_off(rb, part, ch, q.nc, sizeof(T));
#pragma unroll
  for (int i = 0; i < Tile<LPC>::FL; ++i) {
    if constexpr (MODE == FAR) {
      if (t0 + i * LPC + part < q.t1 && ch < q.nc) row[(int64_t)(i * LPC + part) * p.B * ld + ch] = from_f32<T>(v[i]);
    } else {
      buf_store(from_f32<T>(v[i]), rs, off + i * LPC * rb);
    }
  }
}

// Frame R's value from the lane of the channel whose turn it is, to all of them.
template <int LPC, int R>
__device__ __forceinline__ float turn(const float (&v)[Tile<LPC>::FL]) {
  constexpr int P = R % LPC;
  const int x = __float_as_int(v[R / LPC]);
  if constexpr (LPC == 1) return v[R];
  else if constexpr (LPC == 2)
    return __int_as_float(__builtin_amdgcn_update_dpp(0, x, P | P << 2 | (2 + P) << 4 | (2 + P) << 6, 0xf, 0xf, true));
  else if constexpr (LPC == 4) return __int_as_float(__builtin_amdgcn_update_dpp(0, x, P * 0x55, 0xf, 0xf, true));
  else return __int_as_float(__builtin_amdgcn_ds_swizzle(x, 0x18 | P << 5));   // lane (l & 24) | P
}
// A result of frame R, which every lane of the channel has, kept by the lane whose turn it is.
template <int LPC, int R>
__device__ __forceinline__ void keep(float (&v)[Tile<LPC>::FL], float x, int part) {
  if constexpr (LPC == 1) v[R] = x;
  else v[R / LPC] = part == R % LPC ? x : v[R / LPC];
}
template <int I, int E, typename F> __device__ __forceinline__ void unrolled(F f) {
  if constexpr (I < E) {
    f(std::integral_constant<int, I>{});
    unrolled<I + 1, E>(f);
  }
}
// f(frame) for the ns first frames of a tile (and, where ns is odd, the one
// behind them, whose step is zero), in order or in reverse: all of them
// in one stretch of code, or pair by pair in a short tile.
template <bool REV, typename F> __device__ __forceinline__ void by_pairs(int ns, F f) {
  if (ns == TS) {
    unrolled<0, TS>([&](auto i) { f(std::integral_constant<int, REV ? TS - 1 - decltype(i)::value : decltype(i)::value>{}); });
  } else {
    unrolled<0, TS / 2>([&](auto i) {
      constexpr int R = REV ? TS - 2 - 2 * decltype(i)::value : 2 * decltype(i)::value;
      if (R >= ns) return;
      f(std::integral_constant<int, REV ? R + 1 : R>{});
      f(std::integral_constant<int, REV ? R : R + 1>{});
    });
  }
}
#define LANES                                                                                             \
  using K = Tile<LPC>;                                                                                    \
  constexpr int NP = K::NP, FL = K::FL;                                                                   \
  const bool gate = MODE == FAR ? p.z != nullptr : MODE == GATED;                                         \
  const int tid = threadIdx.x, part = tid % LPC, ch = tid / LPC;                                          \
  const int len = length(p, q.b);                                                                         \
  const bool on = ch < q.nc;                                                                              \
  States<NS> A2 = ld_states<NS>(p.A, q.c0 + ch, p.N, part * NS, on);                                      \
  for (int j = 0; j < NS; ++j) A2.v[j] *= LOG2E_F;                                                        \
  const float bias = p.dtb && on ? p.dtb[q.c0 + ch] : 0.f

// ENDS: only what the stretch, from a state of zeros, leaves behind it, and
// the sum of its steps (the product of its decays is the exponential of that
// times A).
template <typename T, int LPC, int MODE, bool ENDS>
__global__ __launch_bounds__(Tile<LPC>::NT) void ssm_scan_fwd_kernel(const ScanP p) {
  __shared__ __attribute__((aligned(16))) float sB[2][TS][Tile<LPC>::NP], sC[ENDS ? 1 : 2][TS][Tile<LPC>::NP];
  const Place q = place<LPC>(p, 0);
  LANES;
  Own<T, LPC> rx, rt, rz;
  BcRegs<T, LPC> rb, rc;
  auto load = [&](int t0) {
    const int ns = max(0, min(TS, len - t0));
    load_own<MODE, T, LPC>(rx, p.x, p.ldx, p, q, t0, ns, part, ch);
    load_own<MODE, T, LPC>(rt, p.dt, p.lddt, p, q, t0, ns, part, ch);
    if (!ENDS && gate) load_own<MODE, T, LPC>(rz, p.z, p.ldz, p, q, t0, ns, part, ch);
    load_bc<MODE, T, LPC>(rb, p.Bm, p.ldb, p, q, t0, ns);
    if constexpr (!ENDS) load_bc<MODE, T, LPC>(rc, p.Cm, p.ldc, p, q, t0, ns);
  };
  load(q.t0);
  const int64_t srow = (int64_t)q.b * p.D + q.c0 + ch;
  States<NS> h = ld_states<NS>(nullptr, 0, 0, 0, false);
  float skip = 0.f, steps = 0.f;
  if constexpr (!ENDS) {
    if (!p.starts) h = ld_states<NS>(p.h0, srow, p.N, part * NS, on);
    else if (on) h = ld_scratch(lane_states<LPC>(p.starts, p, q.seg, q));
    if (p.Dskip && on) skip = p.Dskip[q.c0 + ch];
  }
  int buf = 0;
  for (int t0 = q.t0; t0 < q.t1; t0 += TS, buf ^= 1) {
    const int ns = max(0, min(TS, len - t0));
    if (ENDS && ns == 0) break;
    store_bc<T, LPC>(sB[buf], rb);
    if constexpr (!ENDS) store_bc<T, LPC>(sC[buf], rc);
    // frames behind the end: a step of zero, which leaves the state as it is
    float x[FL], z[FL], s[FL], u[FL], o[FL];
#pragma unroll
    for (int i = 0; i < FL; ++i) {
      x[i] = to_f32(rx.v[i]);
      if (!ENDS && gate) z[i] = to_f32(rz.v[i]);
      s[i] = to_f32(rt.v[i]) + bias;
      if (p.softplus) s[i] = softplusf_(s[i]);
      s[i] = i * LPC + part < ns ? s[i] : 0.f;
      u[i] = s[i] * x[i];
      if constexpr (ENDS) steps += s[i];
    }
    // the only barrier of a tile: a buffer is written again two tiles later
    __syncthreads();
    if (t0 + TS < q.t1) load(t0 + TS);   // in flight while this tile's frames run
    if (!ENDS && p.saved && on) st_scratch(lane_states<LPC>(p.saved, p, t0 / TS, q), h);
    auto frame = [&](auto r) {
      constexpr int R = decltype(r)::value;
      const float sr = turn<LPC, R>(s), ur = turn<LPC, R>(u);
      const States<NS> Bv = row_states(&sB[buf][R][part * NS]);
#pragma unroll
      for (int j = 0; j < NS; ++j) h.v[j] = __builtin_amdgcn_exp2f(sr * A2.v[j]) * h.v[j] + ur * Bv.v[j];
      if constexpr (!ENDS) {
        const States<NS> Cv = row_states(&sC[buf][R][part * NS]);
        float a = 0.f;
#pragma unroll
        for (int j = 0; j < NS; ++j) a += Cv.v[j] * h.v[j];
        keep<LPC, R>(o, group_sum<LPC>(a), part);
      }
    };
    by_pairs<false>(ns, frame);
    if constexpr (!ENDS) {
#pragma unroll
      for (int i = 0; i < FL; ++i) {
        o[i] += skip * x[i];
        if (gate) o[i] *= siluf_(z[i]);
        o[i] = i * LPC + part < ns ? o[i] : 0.f;
      }
      store_own<MODE, T, LPC>(p.y, p.ldy, p, q, t0, part, ch, o);
    }
  }
  if constexpr (ENDS) {
    steps = group_sum<LPC>(steps);
    if (on) {
      st_scratch(lane_states<LPC>(p.ends, p, q.seg, q), h);
      if (part == 0) p.sums[((int64_t)q.seg * p.B + q.b) * p.D + q.c0 + ch] = steps;
    }
  } else if (q.seg == p.nseg - 1) {
    st_states<NS>(p.hlast, srow, p.N, part * NS, on, h);
  }
}

// What a stretch, with nothing behind it, passes to the adjoint before it:
// the backward's counterpart of the ends above, frames in reverse.  The first
// stretch has none before it.
template <typename T, int LPC, int MODE>
__global__ __launch_bounds__(Tile<LPC>::NT) void ssm_scan_adj_kernel(const ScanP p) {
  __shared__ __attribute__((aligned(16))) float sC[2][TS][Tile<LPC>::NP];
  const Place q = place<LPC>(p, 1);
  LANES;
  Own<T, LPC> rt, rz, ry;
  BcRegs<T, LPC> rc;
  auto load = [&](int t0) {
    const int ns = max(0, min(TS, len - t0));
    load_own<MODE, T, LPC>(rt, p.dt, p.lddt, p, q, t0, ns, part, ch);
    load_own<MODE, T, LPC>(ry, p.dy, p.lddy, p, q, t0, ns, part, ch);
    if (gate) load_own<MODE, T, LPC>(rz, p.z, p.ldz, p, q, t0, ns, part, ch);
    load_bc<MODE, T, LPC>(rc, p.Cm, p.ldc, p, q, t0, ns);
  };
  const int last = q.t0 + (min(q.t1, max(len, q.t0 + 1)) - q.t0 - 1) / TS * TS;   // the tile of the last frame
  load(last);
  States<NS> dh = ld_states<NS>(nullptr, 0, 0, 0, false);
  float steps = 0.f;
  int buf = 0;
  for (int t0 = last; t0 >= q.t0; t0 -= TS, buf ^= 1) {
    const int ns = max(0, min(TS, len - t0));
    store_bc<T, LPC>(sC[buf], rc);
    float s[FL], g[FL];
#pragma unroll
    for (int i = 0; i < FL; ++i) {
      s[i] = to_f32(rt.v[i]) + bias;
      if (p.softplus) s[i] = softplusf_(s[i]);
      s[i] = i * LPC + part < ns ? s[i] : 0.f;
      g[i] = to_f32(ry.v[i]);
      if (gate) g[i] *= siluf_(to_f32(rz.v[i]));
      steps += s[i];
    }
    __syncthreads();
    if (t0 > q.t0) load(t0 - TS);
    by_pairs<true>(ns, [&](auto r) {
      constexpr int R = decltype(r)::value;
      const float sr = turn<LPC, R>(s), gr = turn<LPC, R>(g);
      const States<NS> Cv = row_states(&sC[buf][R][part * NS]);
#pragma unroll
      for (int j = 0; j < NS; ++j) dh.v[j] = (dh.v[j] + Cv.v[j] * gr) * __builtin_amdgcn_exp2f(sr * A2.v[j]);
    });
  }
  steps = group_sum<LPC>(steps);
  if (on) {
    st_scratch(lane_states<LPC>(p.ends, p, q.seg, q), dh);
    if (part == 0) p.sums[((int64_t)q.seg * p.B + q.b) * p.D + q.c0 + ch] = steps;
  }
}

// The states (REV: adjoints) that reach each stretch, from those that the
// stretches add.  A thread has four states of a channel and one of 16 runs of
// adjacent stretches: it joins its run, the runs meet in LDS, and it goes
// through its run again from what reaches it.  The loads of eight stretches
// are in flight at a time, and up to 128 stretches they are read once.  (One
// thread over all of 64 stretches waited for memory 26 us, eight runs that
// read twice took 15 us at 128.)
template <bool REV>
__global__ __launch_bounds__(512) void ssm_scan_join_kernel(const float* __restrict__ ends, const float* __restrict__ sums,
                                                            float* __restrict__ starts, const float* __restrict__ A,
                                                            const float* first, int64_t BD, int D, int N, int NP,
                                                            int nseg) {
  constexpr int RUNS = 16;
  __shared__ f32x4 sh[RUNS][32];
  __shared__ float ss[RUNS][32];
  const int el = threadIdx.x & 31, run = threadIdx.x >> 5;
  const int64_t e = (int64_t)blockIdx.x * 32 + el;   // four states
  const int per = NP / 4;
  const int64_t row = e / per;
  const int part = (int)(e % per);
  const bool on = row < BD;
  States<4> A2 = ld_states<4>(A, row % D, N, part * 4, on);
  for (int j = 0; j < 4; ++j) A2.v[j] *= LOG2E_F;
  const int64_t n4 = BD * per;
  const f32x4* in = (const f32x4*)ends + e;
  const int len = (nseg - 1 + RUNS - 1) / RUNS, k0 = run * len, k1 = on ? min(nseg - 1, k0 + len) : 0;
  f32x4 v[8];
  float s[8];
  auto load = [&](int k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = min(k + i, k1 - 1), g = REV ? nseg - 1 - c : c;
      v[i] = in[g * n4];
      s[i] = sums[g * BD + row];
    }
  };
  auto walk = [&](f32x4& h, float& sum, int k, bool write) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (k + i >= k1) break;
      const int g = REV ? nseg - 1 - (k + i) : k + i;
      sum += s[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = __builtin_amdgcn_exp2f(s[i] * A2.v[j]) * h[j] + v[i][j];
      // a stretch's end, from its start, reaches the next one
      if (write) ((f32x4*)starts)[(REV ? g - 1 : g + 1) * n4 + e] = h;
    }
  };
  f32x4 h{0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  for (int k = k0; k < k1; k += 8) {
    load(k);
    walk(h, sum, k, false);
  }
  sh[run][el] = h;
  ss[run][el] = sum;
  __syncthreads();
  if (!on) return;
  const States<4> f = ld_states<4>(first, row, N, part * 4, true);
  for (int j = 0; j < 4; ++j) h[j] = f.v[j];
  if (run == 0) ((f32x4*)starts)[(REV ? nseg - 1 : 0) * n4 + e] = h;
  for (int r = 0; r < run; ++r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = __builtin_amdgcn_exp2f(ss[r][el] * A2.v[j]) * h[j] + sh[r][el][j];
  }
  for (int k = k0; k < k1; k += 8) {
    if (len > 8) load(k);
    walk(h, sum, k, true);
  }
}

// Two words of each lane joined across lanes 2^BIT apart: lanes with that
// bit clear get the sum of `a` over the two, the others that of `b`.
template <int BIT>
__device__ __forceinline__ float join2(float a, float b) {
  if constexpr (BIT == 5) {
    const auto e = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(e[0]) + __uint_as_float(e[1]);
  } else {
    const auto e = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(e[0]) + __uint_as_float(e[1]);
  }
}

// Backward.  Tiles in reverse; each tile recomputes its states from the
// saved one into registers (TS + 1 of them) and then runs the adjoint from
// its last frame to its first.  dB and dC are sums over channels: a wave adds
// its channels by swaps between rows of lanes, the workgroup's waves meet in
// LDS, the tiles of a group in a second launch.
template <typename T, int LPC, int MODE>
__global__ __launch_bounds__(Tile<LPC>::NT, LPC == 2 || LPC == 4 ? 2 : 1) void ssm_scan_bwd_kernel(const ScanP p) {
  __shared__ __attribute__((aligned(16))) float sB[2][TS][Tile<LPC>::NP], sC[2][TS][Tile<LPC>::NP];
  __shared__ __attribute__((aligned(16))) float red[2][LPC][TS][2 * Tile<LPC>::NP];
  const Place q = place<LPC>(p, 0);
  LANES;
  const int lane = tid & 63, wave = tid >> 6;
  const int64_t srow = (int64_t)q.b * p.D + q.c0 + ch;
  Own<T, LPC> rx, rt, rz, ry;
  BcRegs<T, LPC> rb, rc;
  States<NS> rh;
  auto load = [&](int t0) {
    const int ns = max(0, min(TS, len - t0));
    load_own<MODE, T, LPC>(rx, p.x, p.ldx, p, q, t0, ns, part, ch);
    load_own<MODE, T, LPC>(rt, p.dt, p.lddt, p, q, t0, ns, part, ch);
    load_own<MODE, T, LPC>(ry, p.dy, p.lddy, p, q, t0, ns, part, ch);
    if (gate) load_own<MODE, T, LPC>(rz, p.z, p.ldz, p, q, t0, ns, part, ch);
    load_bc<MODE, T, LPC>(rb, p.Bm, p.ldb, p, q, t0, ns);
    load_bc<MODE, T, LPC>(rc, p.Cm, p.ldc, p, q, t0, ns);
  };
  const int last = q.t0 + (q.t1 - q.t0 - 1) / TS * TS;
  load(last);
  // the adjoint that reaches the frames before
  States<NS> dh = ld_states<NS>(nullptr, 0, 0, 0, false), dA = dh;
  if (!p.starts) dh = ld_states<NS>(p.dhl, srow, p.N, part * NS, on);
  else if (on) dh = ld_scratch(lane_states<LPC>(p.starts, p, q.seg, q));
  const float skip = p.Dskip && on ? p.Dskip[q.c0 + ch] : 0.f;
  float dD = 0.f, db = 0.f;
  int buf = 0;
  for (int t0 = last; t0 >= q.t0; t0 -= TS, buf ^= 1) {
    const int ns = max(0, min(TS, len - t0));
    store_bc<T, LPC>(sB[buf], rb);
    store_bc<T, LPC>(sC[buf], rc);
    const Own<T, LPC> cx = rx, ct = rt, cz = rz, cy = ry;
    // frames behind the end: zeros, which pass the state and its adjoint on
    float s[FL], u[FL], g[FL], o[FL], into[FL], da[FL];
#pragma unroll
    for (int i = 0; i < FL; ++i) {
      s[i] = to_f32(ct.v[i]) + bias;
      if (p.softplus) s[i] = softplusf_(s[i]);
      s[i] = i * LPC + part < ns ? s[i] : 0.f;
      u[i] = s[i] * to_f32(cx.v[i]);
      g[i] = to_f32(cy.v[i]);
      if (gate) g[i] *= siluf_(to_f32(cz.v[i]));
    }
    States<NS> first = ld_states<NS>(nullptr, 0, 0, 0, false);
    if (on) first = ld_scratch(lane_states<LPC>(p.saved, p, t0 / TS, q));
    __syncthreads();
    if (t0 > q.t0) load(t0 - TS);
    // frame R forward, the later ones, frame R back: nested, so that the
    // states of frames that a short tile lacks are never live
    auto frames = [&](auto self, auto r, const States<NS>& before) -> void {
      constexpr int R = decltype(r)::value;
      if constexpr (R % 2 == 0) {
        if (R >= ns) return;
      }
      States<NS> h;
      {
        const float sr = turn<LPC, R>(s), ur = turn<LPC, R>(u);
        const States<NS> Bv = row_states(&sB[buf][R][part * NS]);
#pragma unroll
        for (int j = 0; j < NS; ++j) h.v[j] = __builtin_amdgcn_exp2f(sr * A2.v[j]) * before.v[j] + ur * Bv.v[j];
        if (gate) {
          const States<NS> Cv = row_states(&sC[buf][R][part * NS]);
          float a = 0.f;
#pragma unroll
          for (int j = 0; j < NS; ++j) a += Cv.v[j] * h.v[j];
          keep<LPC, R>(o, group_sum<LPC>(a), part);
        }
      }
      if constexpr (R + 1 < TS) self(self, std::integral_constant<int, R + 1>{}, h);
      // B, C and the decays are read and computed again, which the compiler
      // can't see through this: carried over from above they would be 24 registers a frame
      int pt = part;
      asm volatile("" : "+v"(pt));
      float sr = turn<LPC, R>(s);
      asm volatile("" : "+v"(sr));
      const float ur = turn<LPC, R>(u), gr = turn<LPC, R>(g);
      const States<NS> Bv = row_states(&sB[buf][R][pt * NS]), Cv = row_states(&sC[buf][R][pt * NS]);
      float v[2 * NS], in = 0.f, ad = 0.f;
#pragma unroll
      for (int j = 0; j < NS; ++j) {
        const float d = dh.v[j] + Cv.v[j] * gr;
        v[j] = d * ur;              // dB
        v[NS + j] = h.v[j] * gr;    // dC
        in += d * Bv.v[j];
        dh.v[j] = d * __builtin_amdgcn_exp2f(sr * A2.v[j]);
        const float qa = dh.v[j] * before.v[j];
        ad += qa * A2.v[j];
        dA.v[j] += qa * sr;
      }
      keep<LPC, R>(into, group_sum<LPC>(in), part);
      keep<LPC, R>(da, group_sum<LPC>(ad), part);
      // over the wave's channels: rows of lanes first (each swap halves the
      // values a lane holds), then the channels within a row.  Lanes of rows
      // 0, 1 end with dB, of 2, 3 with dC; even rows with the first four of
      // their lane's states and odd ones with the others
      f32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = stride_sum<LPC>(join2<4>(join2<5>(v[j], v[NS + j]), join2<5>(v[4 + j], v[NS + 4 + j])));
      if ((lane & 15) < LPC) *(f32x4*)&red[buf][wave][R][(lane >> 5) * NP + part * NS + ((lane >> 4) & 1) * 4] = w;
    };
    frames(frames, std::integral_constant<int, 0>{}, first);
    float gx[FL], gt[FL], gz[FL];
#pragma unroll
    for (int i = 0; i < FL; ++i) {
      const bool live = i * LPC + part < ns;
      const float x = to_f32(cx.v[i]), vt = to_f32(ct.v[i]) + bias;
      gx[i] = s[i] * into[i] + skip * g[i];
      gt[i] = x * into[i] + da[i] * LN2_F;
      if (p.softplus) gt[i] *= sigmoidf_(vt);
      if (gate) {
        gz[i] = to_f32(cy.v[i]) * (o[i] + skip * x) * dsiluf_(to_f32(cz.v[i]));
        gz[i] = live ? gz[i] : 0.f;
      }
      gx[i] = live ? gx[i] : 0.f;
      gt[i] = live ? gt[i] : 0.f;
      dD += g[i] * x;   // g is zero behind the end
      db += gt[i];
    }
    store_own<MODE, T, LPC>(p.dx, p.lddx, p, q, t0, part, ch, gx);
    store_own<MODE, T, LPC>(p.ddt, p.ldddt, p, q, t0, part, ch, gt);
    if (gate) store_own<MODE, T, LPC>(p.dz, p.lddz, p, q, t0, part, ch, gz);
    // the waves' dB and dC, in wave order (red is written again two tiles
    // later, behind the next tile's barrier)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < (TS * 2 * NP + K::NT - 1) / K::NT; ++i) {
      const int e = i * K::NT + tid, r = e / (2 * NP), c = e % (2 * NP), n = c % NP;
      if (r >= TS || t0 + r >= q.t1 || n >= p.N) continue;
      float v = 0.f;
      if (r < ns) {
#pragma unroll
        for (int w = 0; w < LPC; ++w) v += red[buf][w][r][c];
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
  }
  const int64_t prow = (int64_t)q.seg * p.B + q.b;   // the workgroup's row of the partial sums
  st_states<NS>(p.dA, prow * p.D + q.c0 + ch, p.N, part * NS, on, dA);
  if (q.seg == 0) st_states<NS>(p.dh0, srow, p.N, part * NS, on, dh);
  dD = group_sum<LPC>(dD);
  db = group_sum<LPC>(db);
  if (on && part == 0) {
    p.par[prow * 2 * p.D + q.c0 + ch] = dD;
    p.par[(prow * 2 + 1) * p.D + q.c0 + ch] = db;
  }
}

// Sums of the backward's partials: dB and dC over the tiles of a group; dA,
// dDskip and ddt_bias over the sequences and their stretches.
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
#pragma unroll 8
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

// One frame of B streams: LPC lanes a channel, four states each; the state is
// read and written once, which bounds the kernel.  A thread has CPT channels,
// whose states it loads before it computes, and reads B and C once for them.
// (512 streams of 1024 channels and 16 states, bf16: 1 channel 23.3, 2 19.5, 4 21.1, 8 28.7 us.)
static constexpr int CPT = 2;
template <typename T, int LPC>
__global__ __launch_bounds__(256) void ssm_scan_step_kernel(const ScanP p, const int32_t* __restrict__ slots,
                                                            int n_slots, float* state) {
  constexpr int CH = 256 / LPC;   // channels that a workgroup has at a time
  // workgroups do not cross groups: B and C are one row for all of its channels
  const int per = p.tpg, tiles = p.G * per;
  const int b = (int)(blockIdx.x / (unsigned)tiles), tile = (int)(blockIdx.x % (unsigned)tiles);
  const int g = tile / per, c0 = tile % per * CH * CPT + threadIdx.x / LPC;   // within the group
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
  T* y = (T*)p.y + (int64_t)b * p.ldy + g * p.Dg;
  if (slot < 0) {
    for (int i = 0; i < CPT; ++i)
      if (part == 0 && c0 + i * CH < p.Dg) y[c0 + i * CH] = from_f32<T>(0.f);
    return;
  }
  States<4> h[CPT], A[CPT];
  float x[CPT], dt[CPT], z[CPT], skip[CPT];
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    const int c = c0 + i * CH, d = g * p.Dg + c;
    const bool on = c < p.Dg;
    h[i] = ld_states<4>(state, (int64_t)slot * p.D + d, p.N, part * 4, on);
    A[i] = ld_states<4>(p.A, d, p.N, part * 4, on);
    x[i] = dt[i] = z[i] = skip[i] = 0.f;
    if (on) {
      x[i] = to_f32(((const T*)p.x)[(int64_t)b * p.ldx + d]);
      dt[i] = to_f32(((const T*)p.dt)[(int64_t)b * p.lddt + d]) + (p.dtb ? p.dtb[d] : 0.f);
      if (p.z) z[i] = to_f32(((const T*)p.z)[(int64_t)b * p.ldz + d]);
      if (p.Dskip) skip[i] = p.Dskip[d];
    }
  }
  const T* Bm = (const T*)p.Bm + (int64_t)b * p.ldb + g * p.N;
  const T* Cm = (const T*)p.Cm + (int64_t)b * p.ldc + g * p.N;
  float Bv[4], Cv[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int n = part * 4 + j;
    Bv[j] = n < p.N ? to_f32(Bm[n]) : 0.f;
    Cv[j] = n < p.N ? to_f32(Cm[n]) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < CPT; ++i) {
    const int c = c0 + i * CH;
    const float s = p.softplus ? softplusf_(dt[i]) : dt[i], u = s * x[i], s2 = s * LOG2E_F;
    float o = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      h[i].v[j] = __builtin_amdgcn_exp2f(s2 * A[i].v[j]) * h[i].v[j] + u * Bv[j];
      o += Cv[j] * h[i].v[j];
    }
    st_states<4>(state, (int64_t)slot * p.D + g * p.Dg + c, p.N, part * 4, c < p.Dg, h[i]);
    o = group_sum<LPC>(o) + skip[i] * x[i];
    if (p.z) o *= siluf_(z[i]);
    if (part == 0 && c < p.Dg) y[c] = from_f32<T>(o);
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

// Lanes of a channel with `ns` states each.
static int lanes_of(int N, int ns) {
  int l = 1;
  while (l * ns < N) l *= 2;
  return l;
}
static size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

struct ScanPlan {
  int lpc, np, tpg, nseg, segt;
  int64_t blocks;   // of one stretch
  // bytes; the stretches' ends, starts and sums lie first in either scratch,
  // then the backward's bc, dA, par
  size_t saved, ends, sums, fwd, bc, dA, par, bwd;
};
static int scan_plan(const ssm_dims* d, ScanPlan* o) {
  o->lpc = lanes_of(d->N, NS);
  o->np = NS * o->lpc;
  o->tpg = (int)cdiv(d->D / d->G, Tile<1>::CT);
  o->blocks = (int64_t)d->B * d->G * o->tpg;
  if (o->blocks > 0x7fffffff) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan: B*D too large");
  o->saved = (size_t)cdiv(d->T, TS) * d->B * d->D * o->np * 4;
  // Stretches: a sequence is split where its waves are few, so that 6144 run
  // (one row of 6000 frames / four padded ones of up to 1500 with their
  // backward, us: unsplit 1127 / 1104, 2048 waves 79 / 229, 4096 68 / 209, 6144 69 / 196,
  // 8192 70 / 191).  A stretch's ends cost the exponentials again, 0.75 of the
  // forward, and two more launches, about 64 frames' time: shorter sequences stay whole.
  const int64_t waves = o->blocks * o->lpc, tiles = cdiv(d->T, TS);
  int64_t want = std::min(tiles, 6144 / waves);
  if (want < 2 || d->T * (1 - 1.75 / want) < 64) want = 1;
  o->segt = (int)(cdiv(tiles, want) * TS);
  o->nseg = (int)cdiv(d->T, o->segt);
  o->ends = o->nseg > 1 ? up256((size_t)o->nseg * d->B * d->D * o->np * 4) : 0;
  o->sums = o->nseg > 1 ? up256((size_t)o->nseg * d->B * d->D * 4) : 0;
  o->fwd = 2 * o->ends + o->sums;
  o->bc = o->tpg > 1 ? up256((size_t)o->tpg * d->T * d->B * d->G * 2 * d->N * 4) : 0;
  o->dA = up256((size_t)o->nseg * d->B * d->D * d->N * 4);
  o->par = up256((size_t)o->nseg * d->B * 2 * d->D * 4);
  o->bwd = o->fwd + o->bc + o->dA + o->par;
  if (o->blocks * o->nseg > 0x7fffffff) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan: B*D too large");
  if ((int64_t)d->T * d->B * d->G * d->N > ((int64_t)1 << 36)) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan: T*B*G*N too large");
  return BLSTM_OK;
}

size_t ssm_conv_bwd_bytes(const ssm_dims* d);

extern "C" int ssm_workspace_bytes(const ssm_dims* dims, size_t* saved, size_t* fwd, size_t* bwd, size_t* conv_bwd) {
  ScanPlan pl;
  int rc = ssm_check_dims(dims, "ssm_workspace_bytes");
  if (!rc) rc = scan_plan(dims, &pl);
  if (rc) return rc;
  if (saved) *saved = pl.saved;
  if (fwd) *fwd = pl.fwd;
  if (bwd) *bwd = pl.bwd;
  if (conv_bwd) *conv_bwd = ssm_conv_bwd_bytes(dims);
  return BLSTM_OK;
}

static int scan_in(const ssm_dims* d, const ssm_scan_in* in, const char* fn, ScanP* p) {
  if (!in || !in->x || !in->dt || !in->Bm || !in->Cm || !in->A) return blstm_fail(BLSTM_EINVAL, "%s: NULL pointer", fn);
  if (in->flags & ~(uint32_t)SSM_SOFTPLUS) return blstm_fail(BLSTM_EINVAL, "%s: unknown flags", fn);
  const int64_t bcw = (int64_t)d->G * d->N;
  if (in->ldx < d->D || in->lddt < d->D || in->ldb < bcw || in->ldc < bcw || (in->z && in->ldz < d->D))
    return blstm_fail(BLSTM_EINVAL, "%s: a row pitch is below its row", fn);
  *p = ScanP{};
  p->x = in->x; p->dt = in->dt; p->Bm = in->Bm; p->Cm = in->Cm; p->z = in->z;
  p->ldx = in->ldx; p->lddt = in->lddt; p->ldb = in->ldb; p->ldc = in->ldc; p->ldz = in->ldz;
  p->A = in->A; p->Dskip = in->Dskip; p->dtb = in->dt_bias; p->h0 = in->h0; p->lens = in->lens;
  p->T = d->T; p->B = d->B; p->D = d->D; p->N = d->N; p->G = d->G; p->Dg = d->D / d->G;
  p->softplus = in->flags & SSM_SOFTPLUS;
  p->nseg = 1;
  p->segt = (int)rup(d->T, TS);
  return BLSTM_OK;
}

// LAUNCH(type, lanes, mode)
#define SCAN_BY_LANES(T, M, LAUNCH)   \
  switch (pl.lpc) {                   \
    case 1: LAUNCH(T, 1, M); break;   \
    case 2: LAUNCH(T, 2, M); break;   \
    case 4: LAUNCH(T, 4, M); break;   \
    default: LAUNCH(T, 8, M); break;  \
  }
#define SCAN_BY_MODE(T, LAUNCH)                        \
  if (mode == FAR) { SCAN_BY_LANES(T, FAR, LAUNCH) }   \
  else if (mode == PLAIN) { SCAN_BY_LANES(T, PLAIN, LAUNCH) } \
  else { SCAN_BY_LANES(T, GATED, LAUNCH) }
#define SCAN_DISPATCH(LAUNCH)                                 \
  if (dims->precision == BLSTM_BF16) { SCAN_BY_MODE(bf16, LAUNCH) } \
  else { SCAN_BY_MODE(float, LAUNCH) }

// Whether TS frames of every given pitch lie within 2^31 bytes (what a thread's 32-bit offsets reach).
static bool near(const ssm_dims* d, std::initializer_list<int64_t> lds) {
  int64_t most = 0;
  for (int64_t ld : lds) most = std::max(most, ld);
  return most < (1 << 28) && (int64_t)TS * d->B * most * 4 < 0x7fffffff;
}

static void scan_stretches(const ScanPlan& pl, char* ws, ScanP* p) {
  p->nseg = pl.nseg;
  p->segt = pl.segt;
  p->ends = (float*)ws;
  p->starts = (float*)(ws + pl.ends);
  p->sums = (float*)(ws + 2 * pl.ends);
}
static unsigned join_blocks(const ssm_dims* d, const ScanPlan& pl) {
  return (unsigned)cdiv((int64_t)d->B * d->D * (pl.np / 4), 32);
}

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
  const int mode = !near(dims, {p.ldx, p.lddt, p.ldb, p.ldc, p.ldz, ldy}) ? FAR : p.z ? GATED : PLAIN;
  if ((uintptr_t)saved % 16 || (uintptr_t)ws % 16)
    return blstm_fail(BLSTM_EINVAL, "ssm_scan_fwd: saved and ws must be 16-byte aligned");
  if (pl.nseg > 1) {
    if (!ws) return blstm_fail(BLSTM_EINVAL, "ssm_scan_fwd: NULL pointer");
    scan_stretches(pl, (char*)ws, &p);
    const unsigned nb = (unsigned)(pl.blocks * (pl.nseg - 1));
#define ENDS(T, L, M) \
  BLSTM_LAUNCH("ssm_scan_ends", (ssm_scan_fwd_kernel<T, L, M, true>), dim3(nb), dim3(Tile<L>::NT), 0, stream, p)
    SCAN_DISPATCH(ENDS)
    BLSTM_LAUNCH("ssm_scan_join", ssm_scan_join_kernel<false>, dim3(join_blocks(dims, pl)), dim3(512), 0, stream, p.ends,
                 p.sums, p.starts, p.A, p.h0, (int64_t)dims->B * dims->D, dims->D, dims->N, pl.np, pl.nseg);
  }
#define FWD(T, L, M)                                                                                          \
  BLSTM_LAUNCH("ssm_scan_fwd", (ssm_scan_fwd_kernel<T, L, M, false>), dim3((unsigned)(pl.blocks * pl.nseg)), \
               dim3(Tile<L>::NT), 0, stream, p)
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
  if ((uintptr_t)saved % 16 || (uintptr_t)ws % 16)
    return blstm_fail(BLSTM_EINVAL, "ssm_scan_bwd: saved and ws must be 16-byte aligned");
  const size_t es = dims->precision == BLSTM_BF16 ? 2 : 4;
  char* w = (char*)ws;
  p.dy = dy; p.lddy = lddy; p.dhl = dh_last; p.saved = (float*)saved;
  p.dx = out->dx; p.ddt = out->ddt; p.dB = out->dBm; p.dC = out->dCm; p.dz = out->dz;
  p.lddx = out->lddx; p.ldddt = out->ldddt; p.lddB = out->lddb; p.lddC = out->lddc; p.lddz = out->lddz;
  p.dh0 = out->dh0;
  if (pl.nseg > 1) {
    scan_stretches(pl, w, &p);
    w += pl.fwd;
  }
  p.bc = pl.bc ? (float*)w : nullptr;
  p.dA = (float*)(w + pl.bc);
  p.par = (float*)(w + pl.bc + pl.dA);
  p.tpg = pl.tpg;
  const bool close = near(dims, {p.ldx, p.lddt, p.ldb, p.ldc, p.ldz, lddy, p.lddx, p.ldddt, p.lddz});
  const int mode = !close ? FAR : p.z ? GATED : PLAIN;
  if (pl.nseg > 1) {
    const unsigned nb = (unsigned)(pl.blocks * (pl.nseg - 1));
#define ADJ(T, L, M) \
  BLSTM_LAUNCH("ssm_scan_adj", (ssm_scan_adj_kernel<T, L, M>), dim3(nb), dim3(Tile<L>::NT), 0, stream, p)
    SCAN_DISPATCH(ADJ)
    BLSTM_LAUNCH("ssm_scan_join", ssm_scan_join_kernel<true>, dim3(join_blocks(dims, pl)), dim3(512), 0, stream, p.ends,
                 p.sums, p.starts, p.A, p.dhl, (int64_t)dims->B * dims->D, dims->D, dims->N, pl.np, pl.nseg);
  }
#define BWD(T, L, M)                                                                                  \
  BLSTM_LAUNCH("ssm_scan_bwd", (ssm_scan_bwd_kernel<T, L, M>), dim3((unsigned)(pl.blocks * pl.nseg)), \
               dim3(Tile<L>::NT), 0, stream, p)
  SCAN_DISPATCH(BWD)
  ScanSum s{};
  s.bc = p.bc; s.dA = p.dA; s.par = p.par;
  s.dB = p.dB; s.dC = p.dC; s.lddB = p.lddB; s.lddC = p.lddC;
  s.oA = out->dA; s.oD = out->dDskip; s.ob = out->ddt_bias;
  s.tpg = pl.tpg; s.G = dims->G; s.N = dims->N; s.D = dims->D; s.rows = pl.nseg * dims->B;
  s.M = (int64_t)dims->T * dims->B;
  s.nbc = pl.bc ? s.M * dims->G * 2 * dims->N : 0;
  s.blocks_bc = cdiv(s.nbc, 256);
  const int64_t nb = s.blocks_bc + cdiv((int64_t)dims->D * (dims->N + 2), 16);
  if (es == 2) BLSTM_LAUNCH("ssm_scan_sum", ssm_scan_sum_kernel<bf16>, dim3((unsigned)nb), dim3(256), 0, stream, s);
  else BLSTM_LAUNCH("ssm_scan_sum", ssm_scan_sum_kernel<float>, dim3((unsigned)nb), dim3(256), 0, stream, s);
  return blstm_check_launch("ssm_scan_bwd");
}

extern "C" int ssm_scan_step(const ssm_dims* dims, const ssm_scan_in* in, const int32_t* slots, int32_t n_slots,
                             float* state, void* y, int64_t ldy, hipStream_t stream) {
  ScanP p;
  int rc = ssm_check_dims(dims, "ssm_scan_step");
  if (!rc) rc = scan_in(dims, in, "ssm_scan_step", &p);
  if (rc) return rc;
  if (!state || !y) return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: NULL pointer");
  if (dims->T != 1) return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: T must be 1");
  if (n_slots < 1 || (!slots && n_slots < dims->B))
    return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: %d slots for %d streams", n_slots, dims->B);
  if (ldy < dims->D) return blstm_fail(BLSTM_EINVAL, "ssm_scan_step: a row pitch is below its row");
  p.y = y; p.ldy = ldy;
  const int lpc = lanes_of(dims->N, 4);
  p.tpg = (int)cdiv(p.Dg, 256 / lpc * CPT);
  const int64_t blocks = (int64_t)dims->B * dims->G * p.tpg;
  if (blocks > 0x7fffffff) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan_step: B*D too large");
#define STEP(T, L)                                                                                                \
  case L:                                                                                                         \
    BLSTM_LAUNCH("ssm_scan_step", (ssm_scan_step_kernel<T, L>), dim3((unsigned)blocks), dim3(256), 0, stream, p, \
                 slots, n_slots, state);                                                                          \
    break;
#define STEPS(T) switch (lpc) { STEP(T, 1) STEP(T, 2) STEP(T, 4) STEP(T, 8) STEP(T, 16) }
  if (dims->precision == BLSTM_BF16) { STEPS(bf16) } else { STEPS(float) }
  return blstm_check_launch("ssm_scan_step");
}
