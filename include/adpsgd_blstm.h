/*
 * adpsgd_blstm.h -- C ABI of the MI355X (gfx950) learner-step library.
 *
 * One learner of H-ADPSGD (Zhang et al., "A Highly Efficient Distributed Deep
 * Learning System for Automatic Speech Recognition", arXiv 1907.05701)
 * repeats one SGD step of a bidirectional-LSTM acoustic model (Section 5.2):
 * the LSTM stack forward and back-propagation through time over fixed-length
 * chunks, a linear bottleneck, a softmax cross-entropy over context-dependent
 * states, then the super-learner gradient reduction (eq. 6) and the ADPSGD
 * local update, i.e. one column of eq. 7 (SGD plus 0.5/0.5 averaging with one
 * ring neighbour).
 *
 * Conventions shared by every call:
 *   - All pointers named theta/grad/x/y/dy/... are DEVICE pointers allocated by
 *     the caller; no call allocates device memory (the allocation-free head
 *     entry point works in a static device array of the library, held from
 *     the library's load on each device that runs it).  State carried
 *     between calls lives in the caller's act_ws (saved activations, the
 *     recurrence status flag).  Host-side, the library keeps a per-device
 *     side stream with its events (created on first use by an eager
 *     blstm_bwd that overlaps work, see there) and the bookkeeping of the
 *     optional timing hooks.  Workspace sizes come from
 *     blstm_workspace_bytes().
 *   - Every call only enqueues work on `stream` (no host synchronisation) and
 *     returns 0 on success or a negative BLSTM_E* code; blstm_last_error()
 *     then returns a message for the calling thread.  No C++ exception crosses
 *     the ABI.
 *   - Frame-major activation layout: element (t, b, j) of a [T][B][W] tensor
 *     is at (t*B + b)*W + j.
 *   - Parameters are one flat float32 vector in PyTorch nn.LSTM order: for
 *     layer l = 0..L-1, direction 0 (forward) then 1 (reverse): W_ih [4H][D_l],
 *     W_hh [4H][H], b_ih [4H], b_hh [4H] with gate row blocks i, f, g, o
 *     (D_0 = D, D_l = 2H above); then W_l [P][2H], b_l [P], W_s [K][P], b_s [K].
 *   - precision BLSTM_BF16: GEMM operands (weights and activations) are bf16,
 *     accumulation and the cell state are float32, master weights and
 *     gradients are float32.  precision BLSTM_FP32: everything is float32.
 *     Activation buffers (y_top, workspaces) hold the precision's element type.
 */
#ifndef ADPSGD_BLSTM_H
#define ADPSGD_BLSTM_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { BLSTM_FP32 = 0, BLSTM_BF16 = 1 };

enum {
  BLSTM_OK = 0,
  BLSTM_EINVAL = -1,       /* null pointer, bad dims, bad argument */
  BLSTM_EUNSUPPORTED = -2, /* shape/alignment the kernels do not handle */
  BLSTM_EHIP = -3          /* a HIP launch or runtime call failed */
};

/* adpsgd_step flags */
enum {
  ADPSGD_ORDER_EQ7 = 1u,   /* new = 0.5*(theta + peer) - lr*g (eq. 7 as printed);
                              default: new = 0.5*((theta - lr*g) + peer) */
  ADPSGD_WRITE_PEER = 2u   /* also store the averaged weights into theta_peer
                              (both columns of the pairing in T_k change) */
};

/* L layers, D input features, H cells per direction, P bottleneck units,
 * K classes, T frames per chunk, B sequences; precision BLSTM_FP32/BF16.
 * The paper's model is L=6, D=260, H=512, P=256, K=32000, T=21. */
typedef struct blstm_dims {
  int32_t L, D, H, P, K, T, B, precision;
} blstm_dims;

/* Number of float32 parameters in the flat layout (Section 5.2's "over 43
 * million parameters": 43,154,944 for the paper's model), or BLSTM_EINVAL. */
int64_t blstm_param_count(const blstm_dims* dims);

/* Sizes in bytes of the caller-allocated buffers for these dims:
 *   act_ws   -- activations saved by blstm_fwd for blstm_bwd, plus the
 *               backward's scratch; owned by the caller, opaque layout except
 *               for its last 256 bytes (the recurrence status flag, see
 *               blstm_recurrence_ok).
 *   head_ws  -- scratch of softmax_ce_fwd_bwd (logits, partial sums).
 *   theta_lp -- the bf16 operand copy of theta (n * 2 bytes; 0 for FP32).
 *   y_top    -- blstm_fwd output [T][B][2H] in the precision's element type.
 * Any output pointer may be NULL.  Returns 0 or BLSTM_EINVAL/EUNSUPPORTED. */
int blstm_workspace_bytes(const blstm_dims* dims, size_t* act_ws, size_t* head_ws,
                          size_t* theta_lp, size_t* y_top);

/* theta_lp[i] = bf16 round-to-nearest-even of theta[i], for i < n (the flat
 * layout, unpadded).  BF16 only; a no-op returning 0 for FP32. */
int blstm_pack_params(const blstm_dims* dims, const float* theta, void* theta_lp,
                      hipStream_t stream);

/* Forward pass of the LSTM stack (Section 5.2; cell as PyTorch nn.LSTM, each
 * chunk starting from h = c = 0).
 *   theta    [n] float32;  theta_lp [n] bf16 (BF16; ignored for FP32)
 *   x        [T][B][D] float32 features
 *   act_ws   workspace, written (saved gate pre-activations, cell states, hidden states)
 *   y_top    [T][B][2H] output of the top layer, forward half first. */
int blstm_fwd(const blstm_dims* dims, const float* theta, const void* theta_lp,
              const float* x, void* act_ws, void* y_top, hipStream_t stream);

/* Bottleneck, softmax and frame cross-entropy with their backward
 * (Section 5.2; eqs. 1-2 and 4).  With s = W_s (W_l y + b_l) + b_s per frame:
 *   *loss   = loss_scale * sum over frames of (logsumexp(s) - s[label])
 *   dy_top  [T][B][2H] float32 = dloss/dy_top
 *   grad    the head slots (W_l, b_l, W_s, b_s) of the flat float32 gradient
 *           are overwritten; the LSTM slots are not touched.
 * labels [T][B] int32 in [0, K) (not checked: out-of-range labels give an
 * undefined loss).  loss_scale is 1/(B*T) for the mean frame loss.
 * loss is a device float. */
int softmax_ce_fwd_bwd(const blstm_dims* dims, const float* theta, const void* theta_lp,
                       const void* y_top, const int32_t* labels, float loss_scale,
                       float* loss, float* dy_top, float* grad, void* head_ws,
                       hipStream_t stream);

/* softmax_ce_fwd_bwd without a head_ws argument, for callers that cannot
 * allocate device memory (code under stream capture, tight serving loops,
 * harnesses that forbid allocation).  The head workspace is a static device
 * array of HEAD_STATIC_SCRATCH_BYTES held by each device the library runs on
 * until the process ends; dims whose head workspace (blstm_workspace_bytes'
 * head_ws) exceeds it are rejected with BLSTM_EUNSUPPORTED.  Same arguments,
 * results and errors as softmax_ce_fwd_bwd otherwise.  The call allocates
 * nothing (its first call on a device looks the array's address up once).
 * Calls that overlap on one device share the array and race: serialise them
 * (one stream, or events). */
#define HEAD_STATIC_SCRATCH_BYTES ((size_t)64 << 20)
int softmax_ce_fwd_bwd_static(const blstm_dims* dims, const float* theta, const void* theta_lp,
                              const void* y_top, const int32_t* labels, float loss_scale,
                              float* loss, float* dy_top, float* grad, hipStream_t stream);

/* Back-propagation through time of the LSTM stack (Section 5.2 model; the
 * gradient g of eq. 4 for the LSTM parameters) given dy_top = dloss/dy_top.
 * Per layer, top-down: the gate-gradient recurrence in reverse time
 * (dh = dy + W_hh^T da of the next step, dc, da for gates i, f, g, o), then
 * dW_ih = sum_t da x^T, dW_hh = sum_t da h_prev^T, db = sum_t da and the
 * gradient reaching the layer below, dX = W_ih^T da.
 *   theta, theta_lp  as for blstm_fwd
 *   act_ws  from blstm_fwd with the same theta and dims (saved gate
 *           pre-activations, cell and hidden states); also used as scratch,
 *           so a second blstm_bwd needs a new blstm_fwd first
 *   y_top   [T][B][2H] in the precision's type, from that blstm_fwd
 *   dy_top  [T][B][2H] float32
 *   grad    [n] float32: the LSTM slots are overwritten (b_ih and b_hh
 *           receive the same bias gradient); head slots are not touched.
 * Returns 0, BLSTM_EINVAL (NULL pointer, bad dims) or BLSTM_EHIP (launch
 * failure).  When not under stream capture the call may also run work on an
 * internal stream of the current device (created once, default priority);
 * that work is joined into `stream` before the call returns, so stream order
 * holds as for any other call.  ADPSGD_BLSTM_OVERLAP=0 disables it. */
int blstm_bwd(const blstm_dims* dims, const float* theta, const void* theta_lp,
              void* act_ws, const void* y_top, const float* dy_top, float* grad,
              hipStream_t stream);

/* Whether every recurrent exchange wait of the persistent kernels completed
 * since the previous blstm_recurrence_ok on act_ws (or since act_ws was first
 * used): the flag is sticky, so one query after many steps (or after replays
 * of a captured graph) covers all of them.  The workgroups of a persistent
 * launch that wait for each other start only once all of them run, and where
 * other streams, graphs or processes keep some of them from that, one of them
 * does the work of all, with the same results; so calls may overlap with any
 * other work on the device.  Every wait is bounded all the same: should one
 * give up, the kernel still ends, the flag is set, and the results of that call
 * are not valid.  The flag lives in the last 256 bytes of act_ws (an int32 at
 * offset act_ws_bytes - 256, nonzero after a give-up, one behind it that is
 * nonzero if work was done by one workgroup in that way, and an initialisation
 * tag); the query reads it, clears both, and returns BLSTM_OK or BLSTM_EHIP
 * with a message.  Synchronises `stream`; not during stream capture.
 * ADPSGD_BLSTM_COOPERATIVE=1 makes every persistent launch cooperative (about
 * 15 us more per launch), for comparisons. */
int blstm_recurrence_ok(const blstm_dims* dims, const void* act_ws, hipStream_t stream);

/* Super-learner reduction (eq. 6): out = scale * sum_{r=0}^{R-1} grads[r],
 * summed left to right in float32.  grads is a HOST array of R device
 * pointers (1 <= R <= 16), each to n floats; out may equal grads[0]. */
int replica_grad_reduce(const float* const* grads, int32_t R, int64_t n, float scale,
                        float* out, hipStream_t stream);

/* ADPSGD local update, one column of eq. 7, fused with the reduction above.
 * g = scale * sum_r grads[r] (float32, left to right), t = lr*g, then
 *   default:          theta = ((theta - t) + theta_peer) * 0.5
 *   ADPSGD_ORDER_EQ7: theta = ((theta + theta_peer) * 0.5) - t
 * every operation a single float32 rounding, no fused multiply-add.
 * ADPSGD_WRITE_PEER also stores the result into theta_peer.  theta_lp, if
 * not NULL, receives the bf16 copy of the new theta (as blstm_pack_params).
 * R = 1 with scale = 1 is the plain update.  theta, theta_peer and theta_lp
 * must not alias each other or the gradients. */
int adpsgd_step(float* theta, float* theta_peer, const float* const* grads, int32_t R,
                float scale, int64_t n, float lr, uint32_t flags, void* theta_lp,
                hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Selective state space scan and its short causal convolution: the recurrence
 * of a causal (streaming) acoustic model, where the LSTM stack above needs
 * the whole chunk.  Frame-major as above, each activation tensor with a row
 * pitch of its own: element (t, b, j) is at (t*B + b)*ld + j, so halves and
 * columns of a wider projection are read and written where they lie.
 * Activations hold the precision's type, parameters and their gradients are
 * float32, the scan's state is float32, sums and states are float32 inside.
 *   D channels in G groups of D/G adjacent ones, N states per channel
 *   (1..64), W convolution taps (1..8), T frames, B sequences; T*B at most
 *   2^24, D at most 2^20, and no more of them together than a launch has
 *   threads for, 2^32 - 1 (EUNSUPPORTED).  The scan takes 64 a tile of 64
 *   channels of a group, stretch of a sequence and lane of a channel, with up to
 *   8 states a lane forward, 4 backward where N <= 16: 2^24 sequences of one tile of
 *   16 states go forward and not back.  The backward also refuses
 *   2 T B G N + 16 D (N + 2) above 2^32 - 513.  The convolution and the single
 *   steps take a thread for 4 channels of 8 frames, 4 channels, and 2 channels' 4 states.
 *   lens (NULL, or B int32 on the device): frames t >= lens[b] do not belong
 *   to sequence b (values outside 0..T count as the nearer end).  Their inputs
 *   are not read, outputs and gradients there are zero, and the state
 *   behind the last frame is the one after frame lens[b] - 1.
 * Outputs must not overlap each other or an input, except where said.
 * ------------------------------------------------------------------------- */
typedef struct ssm_dims {
  int32_t T, B, D, N, G, W, precision;
} ssm_dims;

enum {
  SSM_SOFTPLUS = 1u,   /* scan: step = softplus(dt + dt_bias), else dt + dt_bias */
  SSM_SILU = 2u        /* convolution: y = silu(pre), else y = pre */
};

/* Sizes in bytes of caller-allocated buffers (16-byte aligned; a size of 0
 * needs none):
 *   saved    -- states that ssm_scan_fwd keeps for ssm_scan_bwd
 *   fwd, bwd -- scratch of ssm_scan_fwd and ssm_scan_bwd
 *   conv_bwd -- scratch of ssm_conv_bwd
 * A buffer belongs to one call (or one captured graph) at a time.  Any output
 * pointer may be NULL: a size that is not asked for is not held to its call's
 * limits.  Returns 0 or BLSTM_EINVAL/EUNSUPPORTED. */
int ssm_workspace_bytes(const ssm_dims* dims, size_t* saved, size_t* fwd, size_t* bwd, size_t* conv_bwd);

/* pre[t] = bias + sum_j w[j] x[t - W + 1 + j] per channel, y = silu(pre) or pre.
 *   w [D][W] float32 (the last tap meets the current frame), bias [D] or NULL
 *   state      [B][W-1][D] (precision's type): the W-1 inputs before frame 0,
 *              oldest first; NULL for zeros
 *   state_out  the same behind the last frame, or NULL; another buffer than state. */
int ssm_conv_fwd(const ssm_dims* dims, const void* x, int64_t ldx, const float* w, const float* bias,
                 const int32_t* lens, const void* state, void* y, int64_t ldy, void* state_out, uint32_t flags,
                 hipStream_t stream);

/* Gradients of ssm_conv_fwd: dx, dw [D][W], dbias [D] (or NULL) and dstate
 * [B][W-1][D] (or NULL) given dy and, where the loss depends on state_out,
 * dstate_out [B][W-1][D] (or NULL), both in the precision's type.  All are
 * overwritten. */
int ssm_conv_bwd(const ssm_dims* dims, const void* x, int64_t ldx, const float* w, const float* bias,
                 const int32_t* lens, const void* state, const void* dy, int64_t lddy, const void* dstate_out,
                 void* dx, int64_t lddx, float* dw, float* dbias, void* dstate, void* ws, uint32_t flags,
                 hipStream_t stream);

/* One frame (T = 1) of B streams.  state [n_slots][W-1][D] is updated in
 * place; stream b's is row slots[b] (device int32), or row b where slots is
 * NULL (n_slots >= B then).  A slot outside 0..n_slots-1 means no stream: its y is
 * zero and no state changes.  Where several rows name one slot, the first of
 * them is the stream and the others count as none. */
int ssm_conv_step(const ssm_dims* dims, const void* x, int64_t ldx, const float* w, const float* bias,
                  const int32_t* slots, int32_t n_slots, void* state, void* y, int64_t ldy, uint32_t flags,
                  hipStream_t stream);

/* The scan's inputs.  Per sequence, channel d of group g and state n:
 *   s_t = softplus(dt_t + dt_bias) (SSM_SOFTPLUS) or dt_t + dt_bias
 *   h_t[n] = exp(s_t A[d][n]) h_{t-1}[n] + s_t x_t B_t[g][n],   h_{-1} = h0 or 0
 *   o_t = sum_n C_t[g][n] h_t[n] + Dskip[d] x_t
 *   y_t = o_t silu(z_t)   (z given), else o_t
 * x, dt, z [T][B][D]; Bm, Cm [T][B][G*N]; A [D][N], finite, and exp(s_t A) of any one
 * frame within float32 (s_t A below 88: past it 0 * inf makes NaN of a zero state);
 * Dskip, dt_bias [D];
 * h0 [B][D][N].  z, Dskip, dt_bias, h0 and lens may be NULL. */
typedef struct ssm_scan_in {
  const void *x, *dt, *Bm, *Cm, *z;
  int64_t ldx, lddt, ldb, ldc, ldz;
  const float *A, *Dskip, *dt_bias, *h0;
  const int32_t* lens;
  uint32_t flags;
} ssm_scan_in;

/* y [T][B][D]; h_last [B][D][N] (or NULL; may equal h0): the state behind each sequence's last
 * frame; saved: what ssm_scan_bwd reads, or NULL where there is no backward;
 * ws: scratch. */
int ssm_scan_fwd(const ssm_dims* dims, const ssm_scan_in* in, void* y, int64_t ldy, float* h_last, void* saved,
                 void* ws, hipStream_t stream);

/* Gradients of ssm_scan_fwd's inputs, all overwritten.  dx, ddt, dz [T][B][D]
 * and dBm, dCm [T][B][G*N] in the precision's type, the others float32.
 * dz is required with z and refused without; dDskip, ddt_bias and dh0 may be NULL.
 * dh_last [B][D][N]: the loss gradient of h_last, NULL for zeros. */
typedef struct ssm_scan_grads {
  void *dx, *ddt, *dBm, *dCm, *dz;
  int64_t lddx, ldddt, lddb, lddc, lddz;
  float *dA, *dDskip, *ddt_bias, *dh0;
} ssm_scan_grads;

/* in: as given to that ssm_scan_fwd (h0 itself is not read again), saved: as
 * it left it; dy [T][B][D] in the precision's type. */
int ssm_scan_bwd(const ssm_dims* dims, const ssm_scan_in* in, const void* dy, int64_t lddy, const float* dh_last,
                 const void* saved, const ssm_scan_grads* out, void* ws, hipStream_t stream);

/* One frame (T = 1) of B streams; in->h0 and in->lens are ignored.  state
 * [n_slots][D][N] float32 is updated in place; slots as in ssm_conv_step. */
int ssm_scan_step(const ssm_dims* dims, const ssm_scan_in* in, const int32_t* slots, int32_t n_slots, float* state,
                  void* y, int64_t ldy, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Distillation: a student's head trained on a teacher's top logits.
 * ------------------------------------------------------------------------- */
#define SOFTMAX_MAX_TOP 256
#define SOFTMAX_MAX_CLASSES (1 << 18)

/* The k largest logits of every row and what the others weigh:
 *   top  [M][k] float32, the logits themselves in descending order
 *   idx  [M][k] int32, their classes; among equal logits the lower class first
 *   rest [M] float32 (or NULL), log of the sum over the other classes of
 *        exp(logit / temperature); -inf where there are none
 * logits [M][K] of the precision's type, row pitch ld; 1 <= k <= K and
 * k <= SOFTMAX_MAX_TOP, K <= SOFTMAX_MAX_CLASSES, M < 2^22.  A NaN orders above +inf. */
int softmax_topk_rows(const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision, int32_t k,
                      float temperature, float* top, int32_t* idx, float* rest, hipStream_t stream);

/* What a row is trained on.  With u = logits / temperature and the k listed
 * classes' top / temperature and rest (NULL: -inf) normalised to
 * probabilities p_i and r, the soft loss is the Kullback-Leibler divergence
 * of the student's softmax(u) from them, the classes that are not listed as one
 * bucket; the hard loss is the cross-entropy of softmax(logits) with labels:
 *   row_loss = weight (soft temperature^2 KL + hard CE)
 * An entry whose idx is outside 0..K-1 is absent; a class listed twice has
 * both probabilities; a row without entries and rest has no soft loss; one whose
 * entries or rest hold a NaN or +inf has no probabilities, and its loss and gradient
 * are NaN (unless its weight or soft is 0).
 * labels (NULL: none) outside 0..K-1: the row has no hard loss.
 * weights [M] float32 (NULL: ones): a row of weight 0, or with neither loss, has loss
 * and gradient 0 whatever it holds (on the head, whose products sum over frames, its y_top
 * has to be finite all the same). */
typedef struct softmax_teacher {
  const float* top;       /* [M][k] */
  const int32_t* idx;     /* [M][k] */
  const float* rest;      /* [M] or NULL */
  const int32_t* labels;  /* [M] or NULL */
  const float* weights;   /* [M] or NULL */
  int32_t k;              /* 1..SOFTMAX_MAX_TOP */
  float temperature, soft, hard;
} softmax_teacher;

/* row_loss [M] float32 as above (without loss_scale) and dlogits [M][K] =
 * loss_scale * d(sum of row losses)/dlogits in the precision's type, row pitch
 * ldd.  dlogits may equal logits where ldd = ld, and overlaps no input otherwise. */
int softmax_distill_rows(const void* logits, int64_t ld, int64_t M, int32_t K, int32_t precision,
                         const softmax_teacher* teacher, float loss_scale, float* row_loss, void* dlogits,
                         int64_t ldd, hipStream_t stream);

/* The two on the acoustic model's head, from y_top, for dims as above (bf16:
 * the logits are float32 throughout, as in softmax_ce_fwd_bwd).
 * softmax_head_ws_bytes: size of ws for either. */
int softmax_head_ws_bytes(const blstm_dims* dims, size_t* bytes);

/* softmax_topk_rows of the head's logits for the T*B frames of y_top. */
int softmax_topk(const blstm_dims* dims, const float* theta, const void* theta_lp, const void* y_top, int32_t k,
                 float temperature, float* top, int32_t* idx, float* rest, void* ws, hipStream_t stream);

/* softmax_ce_fwd_bwd with the teacher's loss in place of the cross-entropy:
 * *loss = loss_scale * sum of the row losses, dy_top and the head slots of
 * grad as there. */
int softmax_distill_fwd_bwd(const blstm_dims* dims, const float* theta, const void* theta_lp, const void* y_top,
                            const softmax_teacher* teacher, float loss_scale, float* loss, float* dy_top,
                            float* grad, void* ws, hipStream_t stream);

/* Message describing the last failure on the calling thread ("" if none). */
const char* blstm_last_error(void);

/* Optional kernel timing.  After blstm_timing_begin(prefix), every library
 * kernel whose name starts with prefix ("" = all) is bracketed by HIP events
 * on the stream it is launched on; a run of consecutive launches of one
 * per-time-step kernel shares one event pair (counted as that many
 * launches).  blstm_timing_end() waits for those events, fills up to cap
 * entries (one per kernel name: launches and summed milliseconds), stores
 * the number of names in *count and stops recording.  Host-side bookkeeping
 * only; not thread-safe. */
typedef struct blstm_kernel_time {
  char name[48];
  int32_t launches;
  double total_ms;
} blstm_kernel_time;

int blstm_timing_begin(const char* prefix);
int blstm_timing_end(blstm_kernel_time* out, int32_t cap, int32_t* count);

#ifdef __cplusplus
}
#endif

#endif /* ADPSGD_BLSTM_H */
