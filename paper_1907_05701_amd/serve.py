"""A learner's head in 8 bits, for scoring frames.

``Int8Head`` keeps the bottleneck and the output layer of a ``LearnerStep`` as
8-bit integers with a scale for each output, and answers with log
probabilities of given classes, entropies and most likely classes of any
number of frames, without their logits in memory.  Nothing here computes
anything; it only marshals arguments."""

from __future__ import annotations

import torch

from . import binding as bd
from .step import new_scores


def _quantized(w):
    """(integers [N][K rounded up to 16], scales [N]) of a float32 matrix [N][K]."""
    N, K = w.shape
    q = torch.empty((N, (K + 15) // 16 * 16), dtype=torch.int8, device=w.device)
    scale = torch.empty(N, dtype=torch.float32, device=w.device)
    bd.int8_quantize_rows(w, q, scale)
    return q, scale


class Int8Head:
    def __init__(self, learner):
        """learner: a LearnerStep with its weights loaded; later changes to them
        do not reach this head (make a new one)."""
        P, K, H2 = learner.shape["P"], learner.shape["K"], 2 * learner.shape["H"]
        w_l, b_l, w_s, b_s = torch.split(learner.theta[learner.n - (P * H2 + P + K * P + K):], [P * H2, P, K * P, K])
        self.w_l, self.scale_l = _quantized(w_l.view(P, H2))
        self.w_s, self.scale_s = _quantized(w_s.view(K, P))
        self.b_l, self.b_s = b_l.clone(), b_s.clone()
        self.P, self.K, self.H2, self.device = P, K, H2, learner.device
        self.ws, self._older = None, []

    def _buffers(self, M):
        """A workspace for M frames: one for both calls, which follow each other on a stream.
        Smaller ones stay, since a captured graph may hold them; each is at least twice
        the one before, so that they are less than the newest together."""
        n = max(bd.int8_linear_ws_bytes(M, self.w_l.shape[1]), bd.int8_logprob_ws_bytes(M, self.K, self.w_s.shape[1]))
        if self.ws is None or self.ws.numel() < n:
            if self.ws is not None:
                self._older.append(self.ws)
                n = max(n, 2 * self.ws.numel())
            self.ws = torch.empty(n, dtype=torch.uint8, device=self.device)
        return self.ws

    def log_probs(self, y_top, ids=None, k=0, entropy=True, temperature=1.0):
        """As LearnerStep.log_probs, from y_top [..., 2H] (bfloat16 or float32)
        of any number of frames; ids [frames][n].  Calls of one head follow
        each other on one stream (they share a workspace)."""
        y = y_top.reshape(-1, self.H2)
        M = y.shape[0]
        ws = self._buffers(M)
        z = torch.empty((M, self.P), dtype=y.dtype, device=self.device)
        bd.int8_linear_rows(y, self.w_l, self.scale_l, z, ws, bias=self.b_l)
        out = new_scores(M, ids, k, entropy, self.device)
        bd.int8_logprob_rows(z, self.w_s, self.scale_s, ws, bias=self.b_s, ids=ids, temperature=temperature, **out)
        return out
