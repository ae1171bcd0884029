"""GPU: log probabilities and their gradient on the model's head where its frames are taken in more than one part:
every frame has its own list, gradients and answers.

Tolerances.  A bf16 logit s = z W_s + b_s carries the roundings of z, of W_s and of W_l, 2^-8 each at most, as in
test_gpu_distill.py: 3 * 2^-8 of the largest one (`off`); a log probability at a temperature tau is a difference of
two such values over tau.  dH = -sum p (log p + H) ds / tau, and of second order the square of a change of the exponents.
Gradients are the head's (2e-2, test_gpu_parity.py); that of the entropy alone, -p (log p + H) / tau, is relative to differences
of logits, and has the three roundings, p's off / tau, and those of ds and of dz, 2^-8 each: 5 * 2^-8 + off."""

import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_gpu_distill as td  # noqa: E402

pytestmark = pytest.mark.gpu
TAU = 2.0


def lists(M, K, n, g):
    """n classes a frame, a list of ends and classes that are none, frames without a gradient."""
    ids = torch.randint(0, K, (M, n), generator=g, device="cuda", dtype=torch.int32)
    ids[::5, n - 1] = -1
    ids[1::7, 0] = K
    dl, dh = torch.randn(M, n, generator=g, device="cuda") / M, torch.randn(M, generator=g, device="cuda") / M
    dl[::3], dh[::3] = 0.0, 0.0
    return ids, dl, dh


@pytest.mark.parametrize("M,P,K,k,parts", [(1475, 16, 32008, 8, 2), (2900, 8, 40000, 5, 3)])
def test_bf16_scores_of_several_parts(gpu_lib, M, P, K, k, parts):
    from paper_1907_05701_amd import binding as bd
    st, par, g = td.head_case("bf16", M, 64, P, K, k, seed=8)
    assert bd.softmax_head_ws_bytes(st.dims) - bd.blstm_workspace_bytes(st.dims)["head_ws"] < M * K * 4 / (parts - 1)
    ids, dl, dh = lists(M, K, 3, g)
    got = st.log_probs(ids=ids, k=k, temperature=TAU)
    v = {n: st.theta[sl].double().view(shape).requires_grad_() for n, (sl, shape) in par.items()}
    y = st.y_top.double().view(M, -1).requires_grad_()
    s = (y @ v["W_l"].t() + v["b_l"]) @ v["W_s"].t() + v["b_s"]
    lp = torch.log_softmax(s / TAU, 1)
    p, ok = lp.exp(), (ids >= 0) & (ids < K)
    H = -(p * lp).sum(1)
    at = torch.where(ok, ids, 0).long()
    listed = torch.where(ok, lp.gather(1, at), 0.0)

    off = 3 * 2.0 ** -8 * float(s.detach().abs().max())
    with torch.no_grad():
        assert float((got["logprob"].double() - listed).abs().max()) <= 2 * off / TAU
        assert bool((got["logprob"][~ok] == 0).all())
        slope = (p * (lp + H[:, None]).abs()).sum(1)
        assert bool(((got["entropy"].double() - H).abs() <= off / TAU * slope + 2 * (off / TAU) ** 2 + 1e-5).all())
        assert float((lp.gather(1, got["idx"].long()) - got["top"].double()).abs().max()) <= 2 * off / TAU
        assert float((torch.topk(lp, k, 1).values - got["top"].double()).abs().max()) <= 2 * off / TAU

    rel = lambda a, b: float((a - b).norm() / b.norm())  # noqa: E731

    def gradients(loss, bound, keep):
        for t in (*v.values(), y):
            t.grad = None
        loss.backward(retain_graph=keep)
        err = {n: rel(st.grad[sl].double().view(shape), v[n].grad) for n, (sl, shape) in par.items()}
        dy = st.dy_top.double().view(M, -1)
        for r0 in range(0, M, 400):
            err[f"dy{r0}"] = rel(dy[r0:r0 + 400], y.grad[r0:r0 + 400])
        print("[head]", {a: f"{b:.1e}" for a, b in err.items()}, flush=True)
        assert max(err.values()) <= bound, err
        assert bool((dy[::3] == 0).all())
    st.score_head(ids=ids, dlogprob=dl, dentropy=dh, temperature=TAU)
    gradients((dl * listed).sum() + (dh * H).sum(), 2e-2, True)
    st.score_head(dentropy=dh, temperature=TAU)
    gradients((dh * H).sum(), 5 * 2.0 ** -8 + off, False)


def test_float32_scores_of_more_frames_than_a_launch_takes(gpu_lib):
    """2^21 frames and some: rows on either side of the parts, in 64 bits (sums of 32, 8 and 136 float32 products: 1e-5
    for logits, as for the top logits there, and the head's 1e-4 for gradients)."""
    from paper_1907_05701_amd import binding as bd
    T, B, H, P, K, k, n = 2049, 1024, 16, 8, 136, 5, 3
    M = T * B
    d = bd.make_dims(1, 8, H, P, K, T, B, "fp32")
    g = torch.Generator(device="cuda").manual_seed(5)
    theta = torch.rand(bd.blstm_param_count(d), generator=g, device="cuda") - 0.5
    y = torch.rand(T, B, 2 * H, generator=g, device="cuda") * 2 - 1
    ws = torch.empty(bd.softmax_head_ws_bytes(d), dtype=torch.uint8, device="cuda")
    ids, dl, dh = lists(M, K, n, g)
    dl, dh = dl * M, dh * M
    o = {"logprob": torch.full((M, n), 99.0, device="cuda"), "entropy": torch.full((M,), 99.0, device="cuda"),
         "top": torch.full((M, k), 99.0, device="cuda"), "idx": torch.full((M, k), -7, dtype=torch.int32, device="cuda")}
    bd.softmax_logprob(d, theta, None, y, ws, ids=ids, temperature=TAU, **o)
    dy, grad = torch.full_like(y, 99.0), torch.zeros_like(theta)
    bd.softmax_logprob_bwd(d, theta, None, y, dy, grad, ws, ids=ids, dlogprob=dl, dentropy=dh, temperature=TAU)
    rows = [0, 1] + [(1 << 21) + e for e in (-2, -1, 0, 1)] + [M - 2, M - 1]
    at = torch.tensor(rows, device="cuda")
    th = theta[-(P * 2 * H + P + K * P + K):].double().cpu()
    Wl, bl, Ws, bs = torch.split(th, [P * 2 * H, P, K * P, K])
    x = y.view(M, -1)[at].double().cpu().requires_grad_()
    s = (x @ Wl.view(P, -1).t() + bl) @ Ws.view(K, P).t() + bs
    lp = torch.log_softmax(s / TAU, 1)
    H_ = -(lp.exp() * lp).sum(1)
    i = ids[at].cpu()
    ok = (i >= 0) & (i < K)
    listed = torch.where(ok, lp.gather(1, torch.where(ok, i, 0).long()), 0.0)
    got = {name: t[at].cpu().double() for name, t in o.items()}
    with torch.no_grad():
        assert float((got["logprob"] - listed).abs().max()) <= 2e-5 and float((got["entropy"] - H_).abs().max()) <= 2e-5
        assert float((lp.gather(1, got["idx"].long()) - got["top"]).abs().max()) <= 2e-5
        assert float((torch.topk(lp, k, 1).values - got["top"]).abs().max()) <= 2e-5
    ((dl[at].cpu().double() * listed).sum() + (dh[at].cpu().double() * H_).sum()).backward()
    for r, row in enumerate(rows):
        want, have = x.grad[r], dy.view(M, -1)[row].double().cpu()
        assert float((have - want).norm()) <= 1e-4 * float(want.norm()), row
        assert (row % 3 == 0) == bool((have == 0).all())
    for name, t in o.items():
        assert int((t == (-7 if name == "idx" else 99.0)).sum()) == 0, name
    assert int((dy == 99.0).sum()) == 0 and math.isfinite(float(grad.double().sum()))
