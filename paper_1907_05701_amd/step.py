"""One learner step on the GPU through the C ABI.

``LearnerStep`` owns the device buffers of one learner (torch allocations:
memory only) and runs, per step, the five library calls in order:
blstm_fwd -> softmax_ce_fwd_bwd -> blstm_bwd -> adpsgd_step (which also
refreshes the bf16 operand copy for the next step).  Nothing here computes
anything; it only marshals arguments."""

from __future__ import annotations

import numpy as np
import torch

from . import binding as bd


def _given(teacher):
    """A teacher as an argument where there is one: a learner whose step() or
    gradient() knows of none is called as it is."""
    return () if teacher is None else (teacher,)


def new_scores(M, ids, k, entropy, device):
    """Output tensors of the scoring calls for M rows, by argument name: those
    that are asked for."""
    out = {}
    if ids is not None:
        out["logprob"] = torch.empty(ids.shape, dtype=torch.float32, device=device)
    if entropy:
        out["entropy"] = torch.empty(M, dtype=torch.float32, device=device)
    if k:
        out["top"] = torch.empty((M, k), dtype=torch.float32, device=device)
        out["idx"] = torch.empty((M, k), dtype=torch.int32, device=device)
    return out


class LearnerStep:
    def __init__(self, L, D, H, P, K, T, B, precision="bf16", device="cuda:0"):
        self.dims = bd.make_dims(L, D, H, P, K, T, B, precision)
        self.shape = dict(L=L, D=D, H=H, P=P, K=K, T=T, B=B)
        self.precision = precision
        self.device = torch.device(device)
        self.n = bd.blstm_param_count(self.dims)
        sizes = bd.blstm_workspace_bytes(self.dims)
        self.sizes = sizes
        dev = self.device
        act_dtype = torch.bfloat16 if precision == "bf16" else torch.float32
        self.act_dtype = act_dtype
        self.theta = torch.empty(self.n, dtype=torch.float32, device=dev)
        self.peer = torch.empty(self.n, dtype=torch.float32, device=dev)
        self.grad = torch.empty(self.n, dtype=torch.float32, device=dev)
        self.theta_lp = (torch.empty(self.n, dtype=torch.bfloat16, device=dev)
                         if precision == "bf16" else None)
        self.x = torch.empty((T, B, D), dtype=torch.float32, device=dev)
        self.labels = torch.empty((T, B), dtype=torch.int32, device=dev)
        self.y_top = torch.empty((T, B, 2 * H), dtype=act_dtype, device=dev)
        self.dy_top = torch.empty((T, B, 2 * H), dtype=torch.float32, device=dev)
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        self.act_ws = torch.empty(max(sizes["act_ws"], 1), dtype=torch.uint8, device=dev)
        self.head_ws = torch.empty(max(sizes["head_ws"], 1), dtype=torch.uint8, device=dev)
        self.distill_ws = None   # on first use
        self.loss_scale = 1.0 / (T * B)

    # ---------------------------------------------------------------- data ---
    def load(self, theta, x, labels, peer=None):
        self.theta.copy_(torch.from_numpy(np.ascontiguousarray(theta, dtype=np.float32)))
        self.x.copy_(torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)))
        self.labels.copy_(torch.from_numpy(np.ascontiguousarray(labels, dtype=np.int32)))
        if peer is not None:
            self.peer.copy_(torch.from_numpy(np.ascontiguousarray(peer, dtype=np.float32)))
        self.pack()

    def pack(self):
        if self.theta_lp is not None:
            bd.blstm_pack_params(self.dims, self.theta, self.theta_lp)

    # ---------------------------------------------------------- the calls ---
    def forward(self):
        bd.blstm_fwd(self.dims, self.theta, self.theta_lp, self.x, self.act_ws, self.y_top)

    def head(self, y_top=None):
        bd.softmax_ce_fwd_bwd(self.dims, self.theta, self.theta_lp,
                              self.y_top if y_top is None else y_top, self.labels,
                              self.loss_scale, self.loss, self.dy_top, self.grad, self.head_ws)

    def _distill_ws(self):
        if self.distill_ws is None:
            self.distill_ws = torch.empty(bd.softmax_head_ws_bytes(self.dims), dtype=torch.uint8, device=self.device)
        return self.distill_ws

    def top_logits(self, k, temperature=1.0):
        """This learner as a teacher, after forward(): the k top logits of every
        frame, their classes and the log-sum-exp of the other logits over the
        temperature, as new tensors ([T*B][k], [T*B][k], [T*B])."""
        M = self.shape["T"] * self.shape["B"]
        top = torch.empty((M, k), dtype=torch.float32, device=self.device)
        idx = torch.empty((M, k), dtype=torch.int32, device=self.device)
        rest = torch.empty(M, dtype=torch.float32, device=self.device)
        bd.softmax_topk(self.dims, self.theta, self.theta_lp, self.y_top, top, idx, self._distill_ws(), rest,
                        temperature)
        return top, idx, rest

    def distill(self, top, idx, rest=None, weights=None, temperature=1.0, soft=1.0, hard=0.0):
        """head() against a teacher's top logits, mixed with the labels' cross-entropy."""
        bd.softmax_distill_fwd_bwd(self.dims, self.theta, self.theta_lp, self.y_top, top, idx, self.loss_scale,
                                   self.loss, self.dy_top, self.grad, self._distill_ws(), rest,
                                   self.labels.view(-1), weights, temperature, soft, hard)

    def log_probs(self, ids=None, k=0, entropy=True, temperature=1.0):
        """What this learner says of every frame, after forward(): the log
        probabilities of the classes ids [T*B][n] (int32; outside the classes:
        0), the entropy, and the log probabilities and classes of the k most
        likely ones, as new tensors in a dict ("logprob", "entropy", "top", "idx")."""
        out = new_scores(self.shape["T"] * self.shape["B"], ids, k, entropy, self.device)
        bd.softmax_logprob(self.dims, self.theta, self.theta_lp, self.y_top, self._distill_ws(), ids=ids,
                           temperature=temperature, **out)
        return out

    def score_head(self, ids=None, dlogprob=None, dentropy=None, temperature=1.0):
        """head() from the loss gradients of log_probs()' outputs, for losses of
        whole sequences: dy_top and the head's gradient, before backward()."""
        bd.softmax_logprob_bwd(self.dims, self.theta, self.theta_lp, self.y_top, self.dy_top, self.grad,
                               self._distill_ws(), ids=ids, dlogprob=dlogprob, dentropy=dentropy,
                               temperature=temperature)

    def backward(self, dy_top=None):
        bd.blstm_bwd(self.dims, self.theta, self.theta_lp, self.act_ws, self.y_top,
                     self.dy_top if dy_top is None else dy_top, self.grad)

    def gradient(self, teacher=None):
        """teacher: arguments of distill() in a dict, in place of the labels alone."""
        self.forward()
        if teacher is None:
            self.head()
        else:
            self.distill(**teacher)
        self.backward()

    def check_recurrence(self):
        """Raises if a recurrent exchange wait gave up since the last forward
        call (synchronises the current stream)."""
        bd.blstm_recurrence_ok(self.dims, self.act_ws)

    def update(self, lr, flags=0, grads=None, scale=1.0):
        bd.adpsgd_step(self.theta, self.peer, [self.grad] if grads is None else grads, scale, lr,
                       flags, self.theta_lp)

    def step(self, lr, flags=0, teacher=None):
        """The whole learner step: gradient, then the fused update."""
        self.gradient(*_given(teacher))
        self.update(lr, flags)

    def capture(self, lr, steps=1, flags=0, teacher=None):
        """Record `steps` learner steps into a HIP graph (replaying it runs
        them again on the current buffers, i.e. continues training).  Each replay
        reads `teacher`'s tensors where they lie, too: keep them."""
        if teacher is not None:
            self._distill_ws()   # allocated outside the graph's memory
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(steps):
                self.step(lr, flags, *_given(teacher))
        return graph
