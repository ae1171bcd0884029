"""GPU: scoring by a learner and by its 8-bit head, as they are used together:
forward, scores, the gradient of a loss of the scores, and the head in 8 bits
at batch and single-frame sizes."""

import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import score_models as sm  # noqa: E402

pytestmark = pytest.mark.gpu
TOL = 64 * 2.0 ** -24   # as in test_gpu_score.py
SHAPE = dict(L=2, D=40, H=64, P=40, K=203, T=21, B=6)


def learner(precision, **over):
    from paper_1907_05701_amd import inputs
    from paper_1907_05701_amd.step import LearnerStep
    shape = dict(SHAPE, **over)
    st = LearnerStep(**shape, precision=precision)
    x = inputs.features(shape["T"], shape["B"], shape["D"])
    st.load(inputs.params(st.n), x, inputs.labels(shape["T"], shape["B"], shape["K"]))
    st.forward()
    return st


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_a_learner_scores_its_frames(gpu_lib, precision):
    """The label's log probability against the loss, and the most likely classes against the top logits."""
    st = learner(precision)
    M, labels = SHAPE["T"] * SHAPE["B"], st.labels.view(-1, 1)
    s = st.log_probs(ids=labels, k=4)
    st.head()
    top, idx, _ = st.top_logits(4)
    torch.cuda.synchronize()
    assert s["logprob"].shape == (M, 1) and s["entropy"].shape == (M,) and s["top"].shape == (M, 4)
    loss = float(st.loss)
    assert abs(float(-s["logprob"].double().mean()) - loss) <= TOL * (1 + loss)
    assert torch.equal(s["idx"], idx)
    gaps = (s["top"][:, :1] - s["top"]) - (top[:, :1] - top)
    assert float(gaps.abs().max()) <= 2 * TOL * (1 + float(s["top"].abs().max()))
    assert set(st.log_probs(k=2, entropy=False)) == {"top", "idx"}


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_a_step_from_scores_is_a_step_from_labels(gpu_lib, precision):
    """The loss as the labels' mean negative log probability: the gradient of every parameter is the cross-entropy's,
    up to the roundings of ds and dz that both make (bf16) and of sums."""
    st = learner(precision)
    M = SHAPE["T"] * SHAPE["B"]
    st.gradient()
    want = st.grad.clone()
    st.forward()
    st.score_head(ids=st.labels.view(-1, 1), dlogprob=torch.full((M, 1), -1.0 / M, device="cuda"))
    st.backward()
    torch.cuda.synchronize()
    tol = 1e-5 if precision == "fp32" else 4 * 2.0 ** -8
    assert float((st.grad - want).norm() / want.norm()) <= tol


def test_sequence_step_in_a_graph(gpu_lib):
    """Scores, the gradient given from outside and the backward in one graph, replayed beside eager steps."""
    st, ref = learner("bf16"), learner("bf16")
    M = SHAPE["T"] * SHAPE["B"]
    ids = torch.randint(0, SHAPE["K"], (M, 3), dtype=torch.int32, device="cuda")
    dl, dh = torch.randn(M, 3, device="cuda") / M, torch.randn(M, device="cuda") / M

    def step(s):
        s.forward()
        out = s.log_probs(ids=ids, k=3)
        s.score_head(ids=ids, dlogprob=dl, dentropy=dh, temperature=2.0)
        s.backward()
        return out
    step(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(st)
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = torch.randn(st.x.shape, generator=g, device="cuda")
        dl.copy_(torch.randn(M, 3, generator=g, device="cuda") / M)
        st.x.copy_(x)
        ref.x.copy_(x)
        graph.replay()
        want = step(ref)
        torch.cuda.synchronize()
        assert torch.equal(st.grad, ref.grad)
        assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("frames", [1, 6, 40, 126])
def test_the_head_in_8_bits(gpu_lib, precision, frames):
    """Against exact arithmetic: integers of the weights and of the frames, the bottleneck's outputs rounded to the
    precision, their integers, the logits, and float64 log probabilities of those."""
    from paper_1907_05701_amd.serve import Int8Head
    st = learner(precision)
    head = Int8Head(st)
    P, K, H2, n = SHAPE["P"], SHAPE["K"], 2 * SHAPE["H"], st.n
    y = st.y_top.view(-1, H2)[:frames]
    ids = torch.randint(-1, K, (frames, 2), dtype=torch.int32, device="cuda")
    got = head.log_probs(y, ids=ids, k=5, temperature=1.5)
    torch.cuda.synchronize()

    theta = st.theta.cpu().numpy()
    at = n - (P * H2 + P + K * P + K)
    w_l, b_l, w_s, b_s = np.split(theta[at:], np.cumsum([P * H2, P, K * P]))
    q, qs = sm.quantize(y.float().cpu().numpy())
    wq, ws = sm.quantize(w_l.reshape(P, H2))
    z = torch.from_numpy(sm.linear(q, qs, wq, ws, b_l)).to(y.dtype)
    q, qs = sm.quantize(z.float().numpy())
    wq, ws = sm.quantize(w_s.reshape(K, P))
    rows = torch.from_numpy(sm.linear(q, qs, wq, ws, b_s)).double()
    lps = [sm.log_probs(r, 1.5) for r in rows]
    orders = [sm.order(r)[:5] for r in rows]
    want = {"logprob": torch.stack([sm.listed(lp, i) for lp, i in zip(lps, ids.cpu())]),
            "entropy": torch.stack([sm.entropy(r, 1.5) for r in rows]),
            "top": torch.stack([lp[o] for lp, o in zip(lps, orders)])}
    assert torch.equal(got["idx"].cpu().long(), torch.stack(orders))
    for name, w in want.items():
        assert bool(((got[name].double().cpu() - w).abs() <= TOL * (1 + w.abs())).all()), name


def test_the_head_in_8_bits_takes_any_number_of_frames_in_turn(gpu_lib):
    """The workspace grows and is used again; the order of the calls does not matter."""
    from paper_1907_05701_amd.serve import Int8Head
    st = learner("bf16")
    head, H2 = Int8Head(st), 2 * SHAPE["H"]
    y = st.y_top.view(-1, H2)
    whole = head.log_probs(st.y_top, k=3)
    for n in (1, 50, 3, 126):
        part = head.log_probs(y[:n], k=3)
        torch.cuda.synchronize()
        assert torch.equal(part["idx"], whole["idx"][:n])
        assert float((part["entropy"] - whole["entropy"][:n]).abs().max()) <= 2 * TOL * 8


def test_the_head_in_8_bits_in_a_graph_beside_larger_calls(gpu_lib):
    """What a graph holds stays when a later call needs a larger workspace."""
    from paper_1907_05701_amd.serve import Int8Head
    st = learner("bf16")
    head, H2 = Int8Head(st), 2 * SHAPE["H"]
    y = st.y_top.view(-1, H2)
    few = y[:2].clone()
    want = head.log_probs(few, k=3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = head.log_probs(few, k=3)
    held = head.ws.data_ptr()
    head.log_probs(y, k=3)
    assert head.ws.data_ptr() != held
    others = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in (512, 4096, 1 << 16, 1 << 20) for _ in range(8)]
    for _ in range(3):
        for t in got.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)
        assert not any(bool(t.any()) for t in others)
