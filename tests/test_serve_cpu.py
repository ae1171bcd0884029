"""Host-side checks of the 8-bit head's workspaces: what calls of growing numbers of frames keep."""

import torch

from paper_1907_05701_amd import binding as bd
from paper_1907_05701_amd.serve import Int8Head


def _head(P=256, K=32000, H2=1024):
    """A head without weights, on the CPU: workspaces are sized on the host."""
    h = Int8Head.__new__(Int8Head)
    h.w_l, h.w_s = (torch.empty((1, c), dtype=torch.int8).expand(n, c) for n, c in ((P, H2), (K, P)))
    h.P, h.K, h.H2, h.device = P, K, H2, "cpu"
    h.ws, h._older = None, []
    return h


def _need(h, M):
    return max(bd.int8_linear_ws_bytes(M, h.H2), bd.int8_logprob_ws_bytes(M, h.K, h.P))


def test_a_head_whose_frames_rise_one_by_one_keeps_a_few_times_what_it_needs():
    """Kept workspaces double, so that all of them together are below twice the newest, which is below twice the need."""
    h, most = _head(), 0
    for M in range(1, 2689):
        most = max(most, _need(h, M))
        assert h._buffers(M).numel() >= _need(h, M)
        kept = h.ws.numel() + sum(w.numel() for w in h._older)
        assert kept < 4 * most, M


def test_a_workspace_stays_while_it_is_large_enough():
    h = _head()
    most = h._buffers(300)
    assert all(h._buffers(M) is most for M in (1, 7, 299, 300)) and h._older == []
    assert h._buffers(3000) is not most and h._older[0] is most
