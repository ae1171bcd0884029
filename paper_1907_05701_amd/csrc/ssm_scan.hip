// Selective state space scan: entry points, the plan of a launch, the single
// step, and what joins stretches and partial sums.  The scan's kernels and
// their mathematics are in ssm_scan_kernels.hpp.
#include <math.h>

#include <cmath>
#include <initializer_list>

#include "ssm_scan.hpp"

// The square root of 2^(2 e), by which a state is multiplied twice: any finite A is allowed, and over
// a whole stretch the power itself can pass float32's range where its product does not (a state of zero
// stays zero).  2^254 takes every normal float32 past the largest one, 2^-254 below the least, so
// exponents beyond are as good as these (a NaN among them is in the stretch's end, too).
__device__ __forceinline__ float root_decay(float e) { return __builtin_amdgcn_exp2f(__builtin_amdgcn_fmed3f(e, -127.f, 127.f)); }

// The states (REV: adjoints) that reach each stretch, from those that the
// stretches add.  A thread has four states of a channel and one of 16 runs of
// adjacent stretches: it joins its run, the runs meet in LDS, and it goes
// through its run again from what reaches it.  The loads of eight stretches
// are in flight at a time, and up to 129 stretches they are read once.  (One
// thread over all of 64 stretches waited for memory 26 us, eight runs that
// read twice took 15 us at 128.)  188 stretches of 1024 channels of 16 states, whose runs of 12 are read
// twice: 10 us for 26 MB of ends, sums and starts (20 MB of it HBM's), most of it the latency of dependent
// trips to memory.
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
  for (int j = 0; j < 4; ++j) A2.v[j] *= LOG2E_F / 2;
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
      for (int j = 0; j < 4; ++j) {
        const float w = root_decay(s[i] * A2.v[j]);
        h[j] = h[j] * w * w + v[i][j];
      }
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
    for (int j = 0; j < 4; ++j) {
      const float w = root_decay(ss[r][el] * A2.v[j]);
      h[j] = h[j] * w * w + sh[r][el][j];
    }
  }
  for (int k = k0; k < k1; k += 8) {
    if (len > 8) load(k);
    walk(h, sum, k, true);
  }
}

// Sums of the backward's partials: dB and dC over the tiles of a group; dA,
// dDskip and ddt_bias over the sequences and their stretches.  Bound by memory's
// latency: 5 us for 12 MB (128 rows of 21 frames, 1024 channels, 16 states).
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
// read and written once, which bounds the kernel (512 streams: 72 MB in 18.9 us, 3.8 TB/s;
// one stream: the launch).  A thread has CPT channels,
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
  int ns, lpc, np, tpg, nseg, segt;   // ns: states of a lane (forward)
  int bns, blpc;                      // of the backward, ns * lpc alike
  int64_t blocks;   // of one stretch
  // bytes; the stretches' ends, starts and sums lie first in either scratch,
  // then the backward's bc, dA, par
  size_t saved, ends, sums, fwd, bc, dA, par, bwd;
};
static void scan_plan(const ssm_dims* d, ScanPlan* o) {
  o->tpg = (int)cdiv(d->D / d->G, SCAN_CT);
  o->blocks = (int64_t)d->B * d->G * o->tpg;
  // Stretches: a sequence is split where its waves are few, so that 6144 run
  // (one row of 6000 frames / four padded ones of up to 1500 with their
  // backward, us: unsplit 1127 / 1104, 2048 waves 79 / 229, 4096 68 / 209, 6144 69 / 196,
  // 8192 70 / 191).  A stretch's ends cost the exponentials again, 0.75 of the
  // forward, and two more launches, about 64 frames' time: shorter sequences stay whole.
  o->ns = d->N <= 4 ? 4 : 8;
  o->lpc = lanes_of(d->N, o->ns);
  const int64_t waves = o->blocks * o->lpc, tiles = cdiv(d->T, TS);
  int64_t want = std::min(tiles, 6144 / waves);
  if (want < 2 || d->T * (1 - 1.75 / want) < 64) want = 1;
  // Where a SIMD has less than two waves all the same, a lane holds four
  // states: twice the waves of half the length, whose waits overlap.  (Forward
  // and backward of 50 rows of 37 frames, 640 channels, 10 states, fp32:
  // 8 states 56, 4 states 41 us; 8 of 60 frames, 1024, 16, bf16: 68, 48; with 2048 waves of 8 or
  // more: the same within 2 %; 17 to 32 states, which would be 512 threads a tile: 43, 49.)
  if (want * waves < 2048 && d->N <= 16) {
    o->ns = 4;
    o->lpc = lanes_of(d->N, 4);
  }
  o->np = o->ns * o->lpc;
  // The backward always: three waves a SIMD have room for half the states, two for all of
  // them (us, backward of 128 rows of 21 frames, 1024 channels, 16 states: 8 states 58, 4
  // states 55; 512 of 21, 512 channels 111, 102; 64 of 200, 640 channels, 12 states, fp32 151, 141).
  o->bns = d->N <= 16 ? 4 : 8;
  o->blpc = o->np / o->bns;
  o->segt = (int)(cdiv(tiles, want) * TS);
  o->nseg = (int)cdiv(d->T, o->segt);
  o->saved = (size_t)cdiv(d->T, TS) * d->B * d->D * o->np * 4;
  o->ends = o->nseg > 1 ? up256((size_t)o->nseg * d->B * d->D * o->np * 4) : 0;
  o->sums = o->nseg > 1 ? up256((size_t)o->nseg * d->B * d->D * 4) : 0;
  o->fwd = 2 * o->ends + o->sums;
  o->bc = o->tpg > 1 ? up256((size_t)o->tpg * d->T * d->B * d->G * 2 * d->N * 4) : 0;
  o->dA = up256((size_t)o->nseg * d->B * d->D * d->N * 4);
  o->par = up256((size_t)o->nseg * d->B * 2 * d->D * 4);
  o->bwd = o->fwd + o->bc + o->dA + o->par;
}
// Whether a launch has threads enough, for the forward and for the backward.
static int scan_fits(const ScanPlan& pl, int lanes, const char* fn) {
  return pl.blocks * pl.nseg * SCAN_CT * lanes > LAUNCH_THREADS
             ? blstm_fail(BLSTM_EUNSUPPORTED, "%s: B*D too large", fn) : BLSTM_OK;
}
static int scan_fits_fwd(const ScanPlan& pl, const char* fn) { return scan_fits(pl, pl.lpc, fn); }
static int scan_fits_bwd(const ssm_dims* d, const ScanPlan& pl, const char* fn) {
  // a thread of ssm_scan_sum for each element of dB and dC, and 16 for a column of dA
  if (2 * (int64_t)d->T * d->B * d->G * d->N + 16 * (int64_t)d->D * (d->N + 2) + 512 > LAUNCH_THREADS)
    return blstm_fail(BLSTM_EUNSUPPORTED, "%s: T*B*G*N too large", fn);
  return scan_fits(pl, pl.blpc, fn);
}

size_t ssm_conv_bwd_bytes(const ssm_dims* d);

extern "C" int ssm_workspace_bytes(const ssm_dims* dims, size_t* saved, size_t* fwd, size_t* bwd, size_t* conv_bwd) {
  ScanPlan pl;
  int rc = ssm_check_dims(dims, "ssm_workspace_bytes");
  if (rc) return rc;
  scan_plan(dims, &pl);
  if (saved || fwd || bwd) rc = scan_fits_fwd(pl, "ssm_workspace_bytes");
  if (!rc && bwd) rc = scan_fits_bwd(dims, pl, "ssm_workspace_bytes");
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

// Whether TS frames of every given pitch lie within 2^31 bytes (what a thread's 32-bit offsets reach).
static bool near(const ssm_dims* d, std::initializer_list<int64_t> lds) {
  int64_t most = 0;
  for (int64_t ld : lds) most = std::max(most, ld);
  return most < (1 << 28) && (int64_t)TS * d->B * most * 4 < 0x7fffffff;
}

static void scan_launch(ScanPass pass, const ssm_dims* d, const ScanPlan& pl, const ScanP& p, int mode, hipStream_t s) {
  const int stretches = pass == SCAN_ENDS || pass == SCAN_ADJ ? pl.nseg - 1 : pl.nseg;
  const bool back = pass == SCAN_ADJ || pass == SCAN_BWD;
  ((back ? pl.bns : pl.ns) == 4 ? scan_launch_ns4 : scan_launch_ns8)(pass, p, back ? pl.blpc : pl.lpc, d->precision, mode,
                                                                    (unsigned)(pl.blocks * stretches), s);
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
  if (rc) return rc;
  scan_plan(dims, &pl);
  rc = scan_fits_fwd(pl, "ssm_scan_fwd");
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
    scan_launch(SCAN_ENDS, dims, pl, p, mode, stream);
    BLSTM_LAUNCH("ssm_scan_join", ssm_scan_join_kernel<false>, dim3(join_blocks(dims, pl)), dim3(512), 0, stream, p.ends,
                 p.sums, p.starts, p.A, p.h0, (int64_t)dims->B * dims->D, dims->D, dims->N, pl.np, pl.nseg);
  }
  scan_launch(SCAN_FWD, dims, pl, p, mode, stream);
  return blstm_check_launch("ssm_scan_fwd");
}

extern "C" int ssm_scan_bwd(const ssm_dims* dims, const ssm_scan_in* in, const void* dy, int64_t lddy,
                            const float* dh_last, const void* saved, const ssm_scan_grads* out, void* ws,
                            hipStream_t stream) {
  ScanPlan pl;
  ScanP p;
  int rc = ssm_check_dims(dims, "ssm_scan_bwd");
  if (rc) return rc;
  scan_plan(dims, &pl);
  rc = scan_fits_bwd(dims, pl, "ssm_scan_bwd");
  if (!rc) rc = scan_in(dims, in, "ssm_scan_bwd", &p);
  if (rc) return rc;
  if (!dy || !saved || !ws || !out || !out->dx || !out->ddt || !out->dBm || !out->dCm || !out->dA || (in->z && !out->dz))
    return blstm_fail(BLSTM_EINVAL, "ssm_scan_bwd: NULL pointer");
  if (!in->z && out->dz) return blstm_fail(BLSTM_EINVAL, "ssm_scan_bwd: dz without z");
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
    scan_launch(SCAN_ADJ, dims, pl, p, mode, stream);
    BLSTM_LAUNCH("ssm_scan_join", ssm_scan_join_kernel<true>, dim3(join_blocks(dims, pl)), dim3(512), 0, stream, p.ends,
                 p.sums, p.starts, p.A, p.dhl, (int64_t)dims->B * dims->D, dims->D, dims->N, pl.np, pl.nseg);
  }
  scan_launch(SCAN_BWD, dims, pl, p, mode, stream);
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
  if (blocks * 256 > LAUNCH_THREADS) return blstm_fail(BLSTM_EUNSUPPORTED, "ssm_scan_step: B*D too large");
#define STEP(T, L)                                                                                                \
  case L:                                                                                                         \
    BLSTM_LAUNCH("ssm_scan_step", (ssm_scan_step_kernel<T, L>), dim3((unsigned)blocks), dim3(256), 0, stream, p, \
                 slots, n_slots, state);                                                                          \
    break;
#define STEPS(T) switch (lpc) { STEP(T, 1) STEP(T, 2) STEP(T, 4) STEP(T, 8) STEP(T, 16) }
  if (dims->precision == BLSTM_BF16) { STEPS(bf16) } else { STEPS(float) }
  return blstm_check_launch("ssm_scan_step");
}
