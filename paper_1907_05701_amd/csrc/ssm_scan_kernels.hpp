// Kernels of the selective scan for SCAN_NS states a lane (included once for
// each, in a namespace of its own).
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
// channel, each with NS of its states in registers, so N <= NS LPC.  What is
// per channel and frame (the step, the gate, the outputs) is computed once, by
// the lane whose turn the frame is (frame r of a tile: lane r % LPC), and
// reaches the others as a DPP operand: no activation goes through LDS.  B and
// C, which every channel of the group shares, do, staged a tile ahead.
//
// The vector unit bounds these kernels (N = 16: an exponential, three
// multiply-adds and a product a state and frame forward, three times that
// backward), so what is beside the states is kept small.  Measured with 1024
// channels, 16 states, gates, bf16 (us; in brackets the share of it that the vector unit issues):
//   128 rows of 21 frames       forward 23 (0.54), backward 55 (0.80)
//   one row of 6000             ends 26 (0.75), forward 35 (0.71)
//   four padded rows of 1500    ends 26, forward 39 (0.42), adjoint ends 22, backward 79 (0.68)
// The rest is waiting for a tile's first loads and at its barriers, with four
// (backward: three) waves a SIMD.
#include <math.h>

#include <cmath>
#include <type_traits>

#include "dma.hpp"
#include "ssm_scan.hpp"

namespace SCAN_NAMESPACE {
static constexpr int NS = SCAN_NS;

template <int LPC> struct Tile {
  static constexpr int CT = SCAN_CT;                  // channels
  static constexpr int NT = CT * LPC;                 // threads
  static constexpr int NP = NS * LPC;                 // states, padded
  static constexpr int FL = (TS + LPC - 1) / LPC;     // frames of a tile that are a lane's
  static constexpr int BCI = (TS * NP + NT - 1) / NT; // elements of B of a tile that a thread stages
};
static_assert(TS % 8 == 0, "frames of a tile in whole turns of up to 8 lanes");

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
// The values of a lane's states in a staged row.
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
// LDS, the tiles of a group in a second launch.  Three waves a SIMD with four
// states a lane (36 registers for those of a tile), two with eight: tighter bounds spill and run slower.
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
      // can't see through this: carried over from above they would be three registers a state and frame
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
      // 0, 1 end with dB, of 2, 3 with dC; even rows with the first half of
      // their lane's states and odd ones with the other
      constexpr int H = NS / 2;
      typedef float fH __attribute__((ext_vector_type(H)));
      fH w;
#pragma unroll
      for (int j = 0; j < H; ++j)
        w[j] = stride_sum<LPC>(join2<4>(join2<5>(v[j], v[NS + j]), join2<5>(v[H + j], v[NS + H + j])));
      if ((lane & 15) < LPC) *(fH*)&red[buf][wave][R][(lane >> 5) * NP + part * NS + ((lane >> 4) & 1) * H] = w;
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

// LAUNCH(type, lanes, mode); four states a lane go with up to four lanes, eight
// states a lane in the backward with four and more
template <int NUM> struct Lanes { static constexpr int value = NUM; };
template <bool BACK, typename F> static void by_lanes(int lpc, F f) {
  if constexpr (NS == 4 || !BACK) {
    if (lpc == 1) return f(Lanes<1>{});
    if (lpc == 2) return f(Lanes<2>{});
  }
  if constexpr (NS == 8) {
    if (lpc == 8) return f(Lanes<8>{});
  }
  f(Lanes<4>{});
}
#define SCAN_BY_LANES(T, M, LAUNCH) \
  by_lanes<BACK>(lpc, [&](auto lanes) { LAUNCH(T, decltype(lanes)::value, M); });
#define SCAN_BY_MODE(T, LAUNCH)                        \
  if (mode == FAR) { SCAN_BY_LANES(T, FAR, LAUNCH) }   \
  else if (mode == PLAIN) { SCAN_BY_LANES(T, PLAIN, LAUNCH) } \
  else { SCAN_BY_LANES(T, GATED, LAUNCH) }
#define SCAN_DISPATCH(LAUNCH)                                 \
  if (precision == BLSTM_BF16) { SCAN_BY_MODE(bf16, LAUNCH) } \
  else { SCAN_BY_MODE(float, LAUNCH) }

static void launch(ScanPass pass, const ScanP& p, int lpc, int precision, int mode, unsigned blocks, hipStream_t s) {
#define FWD(T, L, M) \
  BLSTM_LAUNCH("ssm_scan_fwd", (ssm_scan_fwd_kernel<T, L, M, false>), dim3(blocks), dim3(Tile<L>::NT), 0, s, p)
#define ENDS(T, L, M) \
  BLSTM_LAUNCH("ssm_scan_ends", (ssm_scan_fwd_kernel<T, L, M, true>), dim3(blocks), dim3(Tile<L>::NT), 0, s, p)
#define ADJ(T, L, M) BLSTM_LAUNCH("ssm_scan_adj", (ssm_scan_adj_kernel<T, L, M>), dim3(blocks), dim3(Tile<L>::NT), 0, s, p)
#define BWD(T, L, M) BLSTM_LAUNCH("ssm_scan_bwd", (ssm_scan_bwd_kernel<T, L, M>), dim3(blocks), dim3(Tile<L>::NT), 0, s, p)
  if (pass == SCAN_FWD || pass == SCAN_ENDS) {
    constexpr bool BACK = false;
    if (pass == SCAN_FWD) { SCAN_DISPATCH(FWD) }
    else { SCAN_DISPATCH(ENDS) }
  } else {
    constexpr bool BACK = true;
    if (pass == SCAN_ADJ) { SCAN_DISPATCH(ADJ) }
    else { SCAN_DISPATCH(BWD) }
  }
}
}  // namespace SCAN_NAMESPACE
