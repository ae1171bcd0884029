"""GPU: a teacher's top logits and the distillation loss and gradients against
float64 forms (tests/operator_models.py), row by row, and on the head.

Tolerances, as in om.far: half a step of the output's type, and 64 * 2^-24 for
the float32 work: an exponent of up to 2^5 (base 2) carries up to 2^5 half-steps
of its own rounding into the exponential, doubled by the scaling; sums add in a
tree.  Temperatures and logits here keep the exponents of what counts within
that."""

import math
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_models as om  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
TOL = 64 * 2.0 ** -24


def run_topk(s, k, tau=1.0, rest=True):
    from paper_1907_05701_amd import binding as bd
    M = s.shape[0]
    top = torch.full((M, k), 99.0, device="cuda")
    idx = torch.full((M, k), -7, dtype=torch.int32, device="cuda")
    r = torch.full((M,), 99.0, device="cuda") if rest else None
    bd.softmax_topk_rows(s, top, idx, r, temperature=tau)
    torch.cuda.synchronize()
    return top, idx, r


def check_topk(s, k, tau=1.0):
    top, idx, rest = run_topk(s, k, tau)
    want = [om.topk(row, k, tau) for row in s.cpu()]
    wt, wi, wr = (torch.stack([w[i] for w in want]) for i in range(3))
    assert torch.equal(idx.cpu().long(), wi)
    assert torch.equal(torch.nan_to_num(top.double().cpu(), nan=1e300), torch.nan_to_num(wt, nan=1e300))
    r = rest.double().cpu()
    assert torch.equal(torch.isnan(r), torch.isnan(wr))
    ok = torch.isfinite(wr)
    assert torch.equal(r[~ok & ~torch.isnan(wr)], wr[~ok & ~torch.isnan(wr)])
    # a logarithm: what its argument is off by, relatively, beside its own rounding
    assert bool(((r - wr).abs()[ok] <= TOL * (1 + wr.abs()[ok])).all())


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,k,tau", [(1, 1, 1, 1.0), (3, 2, 1, 0.5), (4, 7, 7, 2.0), (5, 100, 8, 2.0), (2, 513, 256, 1.0),
                                       (3, 4001, 33, 1.0), (2, 32000, 32, 1.0), (2, 32000, 200, 3.0), (2, 40007, 64, 1.0)])
def test_topk(gpu_lib, M, K, k, tau, precision):
    g = torch.Generator().manual_seed(K + k)
    check_topk((torch.randn(M, K, generator=g) * 3).to(TYPES[precision]).cuda(), k, tau)


def test_topk_of_the_most_classes(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    g = torch.Generator().manual_seed(1)
    check_topk((torch.randn(2, bd.SOFTMAX_MAX_CLASSES, generator=g) * 3).bfloat16().cuda(), 16)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_topk_where_logits_bunch(gpu_lib, precision):
    """Ties over whole rows, ascending and descending rows, all large logits in
    the columns of a few threads, the lowest value, infinities and NaN."""
    K, t = 6000, TYPES[precision]
    low = torch.finfo(t).min
    s = torch.zeros(9, K)
    s[1] = torch.arange(K) / 64
    s[2] = -torch.arange(K) / 64
    s[3, :16] = 5.0
    s[3, 4096:4112] = 7.0
    s[4] = low
    s[4, 70] = 1.0
    s[5] = -math.inf
    s[5, [3, 4000]] = torch.tensor([2.0, 1.0])
    s[6, 100:3000] = math.nan
    s[7] = -0.0
    s[7, ::2] = 0.0
    s[8, [9, 17]] = math.inf
    for k in (1, 40, 256):
        check_topk(s.to(t).cuda(), k)


@pytest.mark.parametrize("precision,K", [("fp32", 300), ("bf16", 9001), ("fp32", 40007), ("bf16", 70001)])
@pytest.mark.parametrize("mask", [None, -1e9, -1e4, 1e9])
def test_topk_of_masked_rows(gpu_lib, mask, precision, K):
    """A few ordinary logits beside a mask's value (None: the type's lowest), fewer of them than k, and a row of nothing
    else.  The rest of the lowest value over a temperature below one is past float32, so it starts at one."""
    t = TYPES[precision]
    m = torch.finfo(t).min if mask is None else mask
    s = torch.full((3, K), m)
    s[0, 5:45] = torch.linspace(-3, 3, 40)
    s[1, [7, K - 1]] = torch.tensor([1.0, 2.0])
    for tau in (1.0, 2.0, 3.0) if mask is None else (0.5, 1.0, 3.0):
        for k in (4, 40, 130):
            top, idx, rest = run_topk(s.to(t).cuda(), k, tau)
            w, at = torch.sort(s.to(t).double(), dim=1, descending=True, stable=True)   # the lower class first
            assert torch.equal(idx.cpu().long(), at[:, :k]) and torch.equal(top.double().cpu(), w[:, :k])
            wr = torch.logsumexp(w[:, k:] / tau, 1)
            assert bool(((rest.double().cpu() - wr).abs() <= TOL * (1 + wr.abs())).all())


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("k", [64, 65, 128])
@pytest.mark.parametrize("K", [130, 4097, 8195, 16391, 32768, 33001])
def test_topk_of_adjacent_large_logits(gpu_lib, K, k, precision):
    """Several of the k within the same 16 bytes; k on either side of where maxima are joined."""
    g = torch.Generator().manual_seed(K)
    s = torch.randn(3, K, generator=g)
    s[1, 16:16 + 40] += 20
    s[2, K - 60:] = torch.arange(60) / 4.0 + 5
    check_topk(s.to(TYPES[precision]).cuda(), k, 2.0)


@pytest.mark.parametrize("K", [33000, 70001])
def test_topk_of_long_rows_that_bunch(gpu_lib, K):
    """The same for rows that 1024 threads hold, and for those that no registers hold."""
    s = torch.zeros(4, K)
    s[1] = torch.arange(K) / 64
    s[2, 4000:5500] = 3.0
    s[2, 9000] = math.nan
    s[3] = -80.0
    s[3, [5, K - 1]] = torch.tensor([90.0, 95.0])     # the others far below the threshold
    for t in (torch.float32, torch.bfloat16):
        check_topk(s.to(t).cuda(), 2)
        check_topk(s.to(t).cuda(), 200, tau=0.5)


def test_topk_is_the_same_every_time(gpu_lib):
    """Candidates arrive in any order; sums over those that are left do not depend on it."""
    g = torch.Generator(device="cuda").manual_seed(8)
    for K in (900, 32000, 70000):
        s = torch.randn(64, K, generator=g, device="cuda") * 3
        first = run_topk(s, 100)
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(first, run_topk(s, 100)))


def test_topk_of_strided_rows(gpu_lib):
    g = torch.Generator().manual_seed(5)
    wide = (torch.randn(4, 1200, generator=g) * 3).cuda()
    for lo, hi in ((1, 1101), (8, 1000)):
        check_topk(wide[:, lo:hi], 20)
    top, idx, _ = run_topk(wide, 5, rest=False)
    assert torch.equal(top, torch.gather(wide, 1, idx.long()))


def make_rows(M, K, k, precision, seed, rest=True):
    g = torch.Generator().manual_seed(seed)
    s = torch.randn(M, K, generator=g) * 2
    top = torch.sort(torch.randn(M, k, generator=g) * 2 + 4, descending=True).values
    idx = torch.stack([torch.randperm(K, generator=g)[:k] for _ in range(M)]).to(torch.int32)
    r = torch.randn(M, generator=g) + 2 if rest else None
    lab = torch.randint(0, K, (M,), generator=g, dtype=torch.int32)
    return s.to(TYPES[precision]), top, idx, r, lab


def check_distill(s, top, idx, rest, labels, weights=None, tau=1.0, soft=1.0, hard=0.0, scale=0.25, inplace=False,
                  view=None):
    from paper_1907_05701_amd import binding as bd
    M, K = s.shape
    gs = s.cuda()
    d = torch.full_like(gs, 99.0)
    if view is not None:
        wide = torch.full((M, K + 9), 99.0, dtype=s.dtype, device="cuda")
        wide[:, view:view + K] = gs
        gs = wide[:, view:view + K]
        d = torch.full_like(wide, 99.0)[:, view:view + K]
    if inplace:
        d = gs
    loss = torch.full((M,), 99.0, device="cuda")
    c = lambda v: None if v is None else v.cuda()  # noqa: E731
    bd.softmax_distill_rows(gs, c(top), c(idx), loss, d, rest=c(rest), labels=c(labels), weights=c(weights),
                            temperature=tau, soft=soft, hard=hard, loss_scale=scale)
    torch.cuda.synchronize()
    wl, wd = [], []
    for m in range(M):
        w = 1.0 if weights is None else float(weights[m])
        row = s[m].double().requires_grad_()
        if w == 0:
            wl.append(torch.zeros((), dtype=torch.float64))
            wd.append(torch.zeros(K, dtype=torch.float64))
            continue
        r = torch.tensor(-math.inf, dtype=torch.float64) if rest is None else rest[m].double()
        l = w * om.distill_row(row, top[m].double(), idx[m].long(), r, -1 if labels is None else int(labels[m]), tau,
                               soft, hard)
        g = torch.autograd.grad(l, row)[0] if l.requires_grad else torch.zeros(K, dtype=torch.float64)
        wl.append(l.detach())
        wd.append(g * scale)
    wl, wd = torch.stack(wl), torch.stack(wd)
    far = {"loss": om.far(loss, wl, TOL * soft * tau * tau + TOL), "dlogits": om.far(d, wd, TOL)}
    print("[distill]", {k: f"{v:.2f}" for k, v in far.items()}, flush=True)
    assert max(far.values()) <= 1.0, far
    if view is not None:
        assert int((d._base == 99.0).sum()) == M * 9


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,k", [(2, 2, 1), (3, 7, 7), (3, 100, 8), (2, 2001, 64), (2, 3000, 256), (2, 32000, 32), (1, 40007, 20)])
def test_distill(gpu_lib, M, K, k, precision):
    s, top, idx, rest, lab = make_rows(M, K, k, precision, K + k, rest=k < K)
    check_distill(s, top, idx, rest, lab, tau=2.0, soft=0.7, hard=0.3)
    check_distill(s, top, idx, None, None)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0, 3.0])
@pytest.mark.parametrize("K", [100, 4097, 8195, 16391, 20003])
def test_distill_at_every_temperature_and_length(gpu_lib, K, tau, precision):
    """Labels among the listed classes, beside them and missing; a row whose
    others lie 200 below its listed ones, one whose listed ones lie below, one of spread logits."""
    s, top, idx, rest, lab = make_rows(5, K, 6, precision, K)
    lab[0], lab[1] = idx[0, 2], -1
    s[2] -= 200
    s[2, idx[2].long()] += 200
    s[3, idx[3].long()] -= 60
    s[4] *= 20
    check_distill(s, top, idx, rest, lab, tau=tau, soft=0.6, hard=0.4)
    check_distill(s, top, idx, rest, lab, tau=tau, soft=0.0, hard=1.0)


@pytest.mark.parametrize("K", [33001, 65537, 100000, 131072])
def test_distill_of_long_rows(gpu_lib, K):
    for precision in ("fp32", "bf16"):
        s, top, idx, rest, lab = make_rows(1, K, 12, precision, K)
        lab[0] = K - 1
        idx[0, 0] = K - 1
        idx[0, 1:] = idx[0, 1:].clamp(max=K - 2)
        check_distill(s, top, idx, rest, lab, tau=2.0, soft=0.5, hard=0.5, inplace=K == 33001)


def test_a_loss_that_is_not_asked_for_may_be_infinite(gpu_lib):
    """The teacher is sure of a class that the student excludes: the soft loss is
    infinite and its gradient finite; with soft = 0 neither is there."""
    s, top, idx, rest, lab = make_rows(2, 50, 3, "fp32", 31)
    s[:, idx[0, 0]] = -math.inf
    idx[1] = idx[0]
    lab[:] = (idx[0, 0] + 1) % 50
    check_distill(s, top, idx, rest, lab, soft=0.0, hard=1.0)
    from paper_1907_05701_amd import binding as bd
    loss, d = torch.empty(2, device="cuda"), torch.empty(2, 50, device="cuda")
    bd.softmax_distill_rows(s.cuda(), top.cuda(), idx.cuda(), loss, d, rest=rest.cuda())
    assert bool(torch.isinf(loss).all()) and bool(torch.isfinite(d).all())


def test_distill_of_the_most_classes(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    s, top, idx, rest, lab = make_rows(1, bd.SOFTMAX_MAX_CLASSES, 9, "bf16", 3)
    check_distill(s, top, idx, rest, lab, tau=3.0, soft=0.5, hard=0.5)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_distill_rows_of_every_kind(gpu_lib, precision):
    """A class listed twice, entries outside the classes, no entry at all, only
    the rest, a label outside, weights (0 over rows of NaN, too)."""
    s, top, idx, rest, lab = make_rows(8, 500, 6, precision, 11)
    idx[0, 3] = idx[0, 0]
    idx[1] = idx[1, 0]
    idx[2, 2:4] = torch.tensor([-1, 500], dtype=torch.int32)
    idx[3] = -1
    idx[4] = -1
    rest[4] = -math.inf
    lab[[0, 5]] = torch.tensor([-1, 500], dtype=torch.int32)
    lab[6] = idx[6, 1]
    w = torch.tensor([1.0, 0.5, 2.0, 1.0, 1.0, 1.0, 0.25, 0.0])
    s[7] = math.nan
    check_distill(s, top, idx, rest, lab, w, tau=1.5, soft=0.8, hard=0.4)
    check_distill(s, top, idx, rest, None, w)
    check_distill(s, top, idx, rest, lab, w, soft=0.0, hard=1.0)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_distill_of_masked_and_far_logits(gpu_lib, precision):
    """Classes masked by the type's lowest value or by -inf; listed logits far above the others, and below."""
    s, top, idx, rest, lab = make_rows(5, 300, 4, precision, 12)
    s[0, 50:] = torch.finfo(s.dtype).min
    idx[0] = torch.tensor([3, 9, 11, 20], dtype=torch.int32)
    s[1, 50:] = -math.inf
    idx[1] = idx[0]
    lab[:2] = 5
    s[2, idx[2].long()] += 150.0       # the others' sum beside e^150
    s[3, idx[3].long()] -= 150.0
    s[4] += 1000.0
    check_distill(s, top, idx, rest, lab, soft=0.5, hard=0.5)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_distill_in_place_and_strided(gpu_lib, precision):
    s, top, idx, rest, lab = make_rows(3, 1001, 16, precision, 13)
    check_distill(s, top, idx, rest, lab, tau=2.0, hard=0.5, inplace=True)
    check_distill(s, top, idx, rest, lab, tau=2.0, hard=0.5, view=1)
    check_distill(s, top, idx, rest, lab, tau=2.0, hard=0.5, view=8, inplace=True)
    s, top, idx, rest, lab = make_rows(3, 4000, 16, precision, 14)
    check_distill(s, top, idx, rest, lab, hard=0.5, inplace=True)


def test_a_teacher_that_is_the_student(gpu_lib):
    """The top logits of the student's own rows: no loss, and gradients that are roundings beside softmax's."""
    from paper_1907_05701_amd import binding as bd
    g = torch.Generator().manual_seed(9)
    s = (torch.randn(5, 3001, generator=g) * 2).cuda()
    top, idx, rest = run_topk(s, 24, tau=2.0)
    loss, d = torch.empty(5, device="cuda"), torch.empty_like(s)
    bd.softmax_distill_rows(s, top, idx, loss, d, rest=rest, temperature=2.0)
    assert float(loss.abs().max()) <= 4 * TOL
    assert bool((d.abs() <= 2 * TOL * torch.softmax(s / 2, 1)).all())


def closed_row(s, top, idx, rest, label, tau, soft, hard):
    """Loss and gradient of a row of distinct classes in float64, from differences
    alone.  (Autograd of logsumexp forms exp(x - (max + log n)), and beside a max of 3.4e38 log n
    is lost in 64 bits, too: n equal classes would weigh 1 each.)"""
    u = (s - s.max()) / tau
    lz = u.exp().sum().log()
    other = torch.ones_like(s, dtype=torch.bool)
    other[idx] = False
    mo = u[other].max()
    w = (u[other] - mo).exp()
    p = torch.softmax(torch.cat((top / tau, rest.view(1))), 0)
    kl = (p[:-1] * (p[:-1].log() - u[idx] + lz)).sum() + p[-1] * (p[-1].log() - mo - w.sum().log() + lz)
    d = (u - lz).exp()
    d[idx] -= p[:-1]
    d[other] -= p[-1] * w / w.sum()
    loss, d = soft * tau * tau * kl, soft * tau * d
    if label >= 0 and hard:
        v = s - s.max()
        lse = v.exp().sum().log()
        loss = loss + hard * (lse - v[label])
        d += hard * (v - lse).exp()
        d[label] -= hard
    return loss, d


MASKS = {"lowest": None, "-1e9": -1e9, "-1e4": -1e4, "1e9": 1e9}


@pytest.mark.parametrize("precision,K", [("fp32", 300), ("bf16", 300), ("bf16", 33001), ("fp32", 65540), ("bf16", 131080)])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0, 3.0])
@pytest.mark.parametrize("mask", MASKS)
def test_distill_where_a_mask_leaves_nothing(gpu_lib, mask, tau, precision, K):
    """Every class that is not listed at the mask's value, and the whole row at it,
    with and without labels; rows that registers hold and rows that none do.
    Equal logits are equal probabilities however large they are: the bounds are the others'.
    A row a call: the loss of one (up to 1e38) is no measure for another."""
    s, top, idx, rest, lab = make_rows(2, K, 4, precision, 41)
    m = torch.finfo(s.dtype).min if MASKS[mask] is None else MASKS[mask]
    keep = s[0, idx[0].long()].clone()
    rest[0] = -1.0   # a small share, so that what it costs is below float32's largest
    s[:] = m
    s[0, idx[0].long()] = keep
    lab[0] = idx[0, 1]
    from paper_1907_05701_amd import binding as bd
    for i in (0, 1):
        gs, *t = (v[i:i + 1].cuda() for v in (s, top, idx, rest))
        for labels, soft, hard in ((lab, 0.5, 0.5), (None, 1.0, 0.0)):
            loss, d = torch.full((1,), 99.0, device="cuda"), torch.full_like(gs, 99.0)
            bd.softmax_distill_rows(gs, t[0], t[1], loss, d, rest=t[2], temperature=tau, soft=soft, hard=hard,
                                    labels=None if labels is None else labels[i:i + 1].cuda())
            wl, wd = closed_row(s[i].double(), top[i].double(), idx[i].long(), rest[i].double(), int(lab[i]), tau, soft, hard)
            far = {"loss": om.far(loss[0], wl, TOL * soft * tau * tau + TOL), "dlogits": om.far(d[0], wd, TOL)}
            print("[mask]", i, {k: f"{v:.2f}" for k, v in far.items()}, flush=True)
            assert max(far.values()) <= 1.0, (i, far)


@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
def test_a_teacher_of_lowest_values(gpu_lib, tau):
    """Listed logits at float32's lowest value: equal among themselves, nothing beside an ordinary one or a rest."""
    s, top, idx, rest, lab = make_rows(5, 200, 4, "fp32", 43)
    low = torch.finfo(torch.float32).min
    top[0], rest[0] = low, -math.inf
    top[1] = low
    top[2, 1:], rest[2] = low, -math.inf
    rest[3] = low
    top[4], rest[4] = 1e9, -math.inf
    check_distill(s, top, idx, rest, lab, tau=tau, soft=0.5, hard=0.5)
    check_distill(s, top, idx, rest, None, tau=tau)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("tau", [1.0, 2.0, 3.0])
def test_a_teacher_that_has_diverged_is_seen(gpu_lib, tau, precision):
    """A NaN or +inf among the listed logits or as the rest: no probabilities, so
    the loss and every gradient of the row are NaN, with labels, too.  Not where the
    entry is absent, the row weighs nothing or the soft loss is not wanted."""
    from paper_1907_05701_amd import binding as bd
    s, top, idx, rest, lab = make_rows(9, 500, 4, precision, 44)
    top[0, 2] = math.nan
    top[1] = math.nan
    top[2], rest[2] = math.nan, -math.inf
    top[3, 0] = math.inf
    rest[4] = math.nan
    rest[5] = math.inf
    idx[5, 1] = idx[5, 0]
    top[6, 3], idx[6, 3] = math.nan, -1
    top[7] = math.nan
    w = torch.ones(9)
    w[7] = 0
    bad = torch.tensor([True] * 6 + [False] * 3)
    s, top, idx, rest, lab, w = (v.cuda() for v in (s, top, idx, rest, lab, w))
    for labels, soft, hard in ((None, 1.0, 0.0), (lab, 0.5, 0.5)):
        loss, d = torch.zeros(9, device="cuda"), torch.zeros_like(s)
        bd.softmax_distill_rows(s, top, idx, loss, d, rest=rest, labels=labels, weights=w, temperature=tau, soft=soft,
                                hard=hard)
        assert torch.equal(torch.isnan(loss).cpu(), bad), loss
        n = torch.isnan(d).sum(1).cpu()
        assert bool((n[bad] == 500).all()) and bool((n[~bad] == 0).all()), n
        assert float(loss[7]) == 0 and not bool(d[7].any())
    check_distill(s.cpu(), top.cpu(), idx.cpu(), rest.cpu(), lab.cpu(), w.cpu(), tau=tau, soft=0.0, hard=1.0)


@pytest.mark.parametrize("precision,K", [("fp32", 130), ("bf16", 9001), ("fp32", 70001)])
def test_a_row_with_neither_loss_has_no_gradient(gpu_lib, precision, K):
    """No entry, no rest and no label, over logits that a mask has left nothing of, NaN or ordinary: zeros,
    in place, too."""
    from paper_1907_05701_amd import binding as bd
    s, top, idx, rest, lab = make_rows(5, K, 6, precision, 51)
    idx[:4], rest[:4], lab[:4] = -1, -math.inf, -1
    s[0], s[1], s[3, 7] = -math.inf, math.nan, math.inf
    for labels, soft, hard in ((None, 1.0, 0.0), (lab, 0.5, 0.5), (lab, 0.0, 1.0)):
        for inplace in (False, True):
            g = s.cuda()
            loss, d = torch.full((5,), 99.0, device="cuda"), g if inplace else torch.full_like(g, 99.0)
            bd.softmax_distill_rows(g, top.cuda(), idx.cuda(), loss, d, rest=rest.cuda(), soft=soft, hard=hard,
                                    labels=None if labels is None else labels.cuda(), temperature=2.0)
            assert not bool(loss[:4].any()) and not bool(d[:4].any())
            assert float(loss[4]) > 0 and bool(torch.isfinite(d[4]).all()) and bool(d[4].any())


# ------------------------------------------------------------------ the head ---
def head_case(precision, M, H, P, K, k, seed=0):
    from paper_1907_05701_amd.step import LearnerStep
    st = LearnerStep(L=1, D=8, H=H, P=P, K=K, T=1, B=M, precision=precision)
    g = torch.Generator(device="cuda").manual_seed(seed)
    st.theta.copy_(torch.rand(st.n, generator=g, device="cuda") * 0.2 - 0.1)
    st.pack()
    st.y_top.copy_(torch.rand(1, M, 2 * H, generator=g, device="cuda") * 2 - 1)
    st.grad.fill_(7.0)
    n = 2 * (4 * H * 8 + 4 * H * H + 8 * H)
    par, off = {}, n
    for name, shape in (("W_l", (P, 2 * H)), ("b_l", (P,)), ("W_s", (K, P)), ("b_s", (K,))):
        par[name] = slice(off, off + math.prod(shape)), shape
        off += math.prod(shape)
    assert off == st.n
    return st, par, g


def head_model(st, par):
    """float64 leaves and logits of the head, on the unrounded weights."""
    v = {k: st.theta[sl].double().view(shape).cpu().requires_grad_() for k, (sl, shape) in par.items()}
    y = st.y_top.double().cpu().view(-1, st.y_top.shape[-1]).requires_grad_()
    z = y @ v["W_l"].t() + v["b_l"]
    return v, y, z @ v["W_s"].t() + v["b_s"]


@pytest.mark.parametrize("precision,bound", [("fp32", 1e-4), ("bf16", 2e-2)])   # the head's own (test_gpu_parity.py)
@pytest.mark.parametrize("M,H,P,K,k", [(5, 64, 16, 133, 9), (168, 64, 32, 100, 8), (150, 96, 24, 1003, 20), (1100, 64, 64, 500, 16)])
def test_head_distillation(gpu_lib, M, H, P, K, k, precision, bound):
    st, par, g = head_case(precision, M, H, P, K, k)
    top = torch.randn(M, k, generator=g, device="cuda") * 2 + 3
    idx = torch.argsort(torch.rand(M, K, generator=g, device="cuda"), 1)[:, :k].to(torch.int32).contiguous()
    rest = torch.randn(M, generator=g, device="cuda")
    st.labels.copy_(torch.randint(0, K, (1, M), generator=g, device="cuda"))
    w = (torch.rand(M, generator=g, device="cuda") < 0.8).float()
    st.distill(top, idx, rest, weights=w, temperature=2.0, soft=0.6, hard=0.4)
    torch.cuda.synchronize()
    v, y, s = head_model(st, par)
    c = lambda t: t.double().cpu()  # noqa: E731
    p = torch.softmax(torch.cat((c(top) / 2, c(rest)[:, None]), 1), 1)
    lq = torch.log_softmax(s / 2, 1)
    at = idx.long().cpu()
    hit = torch.zeros(M, K, dtype=torch.bool).scatter_(1, at, True)
    lo = torch.logsumexp(lq.masked_fill(hit, -math.inf), 1)
    kl = (p[:, :-1] * (torch.log(p[:, :-1]) - lq.gather(1, at))).sum(1) + p[:, -1] * (torch.log(p[:, -1]) - lo)
    ce = -torch.log_softmax(s, 1).gather(1, st.labels.view(-1, 1).long().cpu())[:, 0]
    loss = (c(w) * (0.6 * 4 * kl + 0.4 * ce)).sum() / M
    loss.backward()
    rel = lambda a, b: float((a - b).norm() / b.norm())  # noqa: E731
    err = {k2: rel(c(st.grad[sl]).view(shape), v[k2].grad) for k2, (sl, shape) in par.items()}
    err["dy"] = rel(c(st.dy_top).view(M, -1), y.grad)
    loss = loss.detach()
    err["loss"] = abs(float(st.loss) - float(loss)) / abs(float(loss))
    print("[head]", {a: f"{b:.1e}" for a, b in err.items()}, flush=True)
    assert max(err.values()) <= bound, err
    assert bool((st.grad[:par["W_l"][0].start] == 7).all())   # the stack's slots are not the head's


def test_head_distillation_at_the_paper_batch(gpu_lib):
    """2688 frames of 32000 states in bf16: three pieces of the logits, the last a short one."""
    M, K, k = 2688, 32000, 32
    st, par, g = head_case("bf16", M, 512, 256, K, k, seed=2)
    top = torch.randn(M, k, generator=g, device="cuda") * 2 + 8
    idx = ((torch.randint(0, K, (M, 1), generator=g, device="cuda") + 991 * torch.arange(k, device="cuda")) % K).int()
    rest = torch.randn(M, generator=g, device="cuda") + 8
    st.labels.copy_(torch.randint(0, K, (1, M), generator=g, device="cuda"))
    st.distill(top, idx, rest, temperature=2.0, soft=0.6, hard=0.4)
    p = {n: st.theta[sl].double().view(shape) for n, (sl, shape) in par.items()}
    y = st.y_top.double().view(M, -1)
    z = y @ p["W_l"].t() + p["b_l"]
    s = z @ p["W_s"].t() + p["b_s"]
    t = torch.softmax(torch.cat((top.double() / 2, rest.double()[:, None]), 1), 1)
    q = torch.softmax(s / 2, 1)
    at = torch.zeros_like(q).scatter_(1, idx.long(), 1.0)
    qr = (q * (1 - at)).sum(1, keepdim=True)
    lab = st.labels.view(-1, 1).long()
    q1 = torch.softmax(s, 1)
    kl = (t[:, :-1] * (t[:, :-1].log() - q.gather(1, idx.long()).log())).sum(1) + t[:, -1] * (t[:, -1:].log() - qr.log())[:, 0]
    loss = float((0.6 * 4 * kl - 0.4 * q1.gather(1, lab).log()[:, 0]).mean())
    ds = 0.6 * 2 * (q - (1 - at) * q * (t[:, -1:] / qr)).scatter_add(1, idx.long(), -t[:, :-1])
    ds = (ds + 0.4 * q1.scatter_add(1, lab, torch.full_like(qr, -1.0))) / M
    dz = ds @ p["W_s"]
    want = {"W_l": dz.t() @ y, "b_l": dz.sum(0), "W_s": ds.t() @ z, "b_s": ds.sum(0)}
    rel = lambda a, b: float((a - b).norm() / b.norm())  # noqa: E731
    err = {n: rel(st.grad[sl].double().view(shape), want[n]) for n, (sl, shape) in par.items()}
    err["dy"] = rel(st.dy_top.double().view(M, -1), dz @ p["W_l"])
    err["loss"] = abs(float(st.loss) - loss) / loss
    print("[head]", {a: f"{b:.1e}" for a, b in err.items()}, flush=True)
    assert max(err.values()) <= 2e-2, err


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_head_top_logits(gpu_lib, precision):
    M, K, k = 1100, 700, 12
    st, par, _ = head_case(precision, M, 64, 32, K, k, seed=4)
    top, idx, rest = st.top_logits(k, temperature=2.0)
    _, _, s = head_model(st, par)
    s = s.detach()
    # float32: sums of 128 and 32 products; bf16: operands and z rounded, 2^-8 each
    off = 1e-5 if precision == "fp32" else 3 * 2.0 ** -8 * float(s.abs().max())
    assert float((s.gather(1, idx.long().cpu()) - top.double().cpu()).abs().max()) <= off
    want, order = torch.sort(s, 1, descending=True)
    assert float((want[:, :k] - top.double().cpu()).abs().max()) <= off
    assert float((torch.logsumexp(want[:, k:] / 2, 1) - rest.double().cpu()).abs().max()) <= off
    assert bool((top[:, 1:] <= top[:, :-1]).all())
    assert all(len(set(r)) == k for r in idx.tolist())


@pytest.mark.parametrize("M,P,K,k,parts", [(1475, 16, 32008, 8, 2), (2900, 8, 40000, 5, 3), (2900, 24, 75, 5, 1)])
def test_bf16_heads_of_several_parts(gpu_lib, M, P, K, k, parts):
    """Frames past one part of the logits, the last part shorter than the others:
    targets, weights and labels of every frame are its own.  Bounds: the head's (2e-2, test_gpu_parity.py),
    and, for single logits, operands and z rounded, 2^-8 each, as in test_head_top_logits."""
    from paper_1907_05701_amd import binding as bd
    st, par, g = head_case("bf16", M, 64, P, K, k, seed=6)
    more = bd.softmax_head_ws_bytes(st.dims) - bd.blstm_workspace_bytes(st.dims)["head_ws"]
    assert more < M * K * 4 / (parts - 1) if parts > 1 else more >= M * K * 4   # the logits of a part (and sums)
    top = torch.randn(M, k, generator=g, device="cuda") * 2 + 3
    idx = torch.argsort(torch.rand(M, K, generator=g, device="cuda"), 1)[:, :k].to(torch.int32).contiguous()
    rest = torch.randn(M, generator=g, device="cuda")
    st.labels.copy_(torch.randint(0, K, (1, M), generator=g, device="cuda"))
    w = torch.rand(M, generator=g, device="cuda") * (torch.rand(M, generator=g, device="cuda") < 0.8)
    st.distill(top, idx, rest, weights=w, temperature=2.0, soft=0.6, hard=0.4)
    v = {n: st.theta[sl].double().view(shape).requires_grad_() for n, (sl, shape) in par.items()}
    y = st.y_top.double().view(M, -1).requires_grad_()
    s = (y @ v["W_l"].t() + v["b_l"]) @ v["W_s"].t() + v["b_s"]
    p = torch.softmax(torch.cat((top.double() / 2, rest.double()[:, None]), 1), 1)
    lq, at = torch.log_softmax(s / 2, 1), idx.long()
    hit = torch.zeros(M, K, dtype=torch.bool, device="cuda").scatter_(1, at, True)
    lo = torch.logsumexp(lq.masked_fill(hit, -math.inf), 1)
    kl = (p[:, :-1] * (torch.log(p[:, :-1]) - lq.gather(1, at))).sum(1) + p[:, -1] * (torch.log(p[:, -1]) - lo)
    ce = -torch.log_softmax(s, 1).gather(1, st.labels.view(-1, 1).long())[:, 0]
    loss = (w.double() * (0.6 * 4 * kl + 0.4 * ce)).sum() / M
    loss.backward()
    rel = lambda a, b: float((a - b).norm() / b.norm())  # noqa: E731
    err = {n: rel(st.grad[sl].double().view(shape), v[n].grad) for n, (sl, shape) in par.items()}
    dy = st.dy_top.double().view(M, -1)
    for r0 in range(0, M, 400):
        err[f"dy{r0}"] = rel(dy[r0:r0 + 400], y.grad[r0:r0 + 400])
    assert bool((dy[w == 0] == 0).all())
    err["loss"] = abs(float(st.loss) - float(loss.detach())) / float(loss.detach())
    print("[head]", {a: f"{b:.1e}" for a, b in err.items()}, flush=True)
    assert max(err.values()) <= 2e-2, err
    got, gi, gr = st.top_logits(k, temperature=2.0)
    s = s.detach()
    off = 3 * 2.0 ** -8 * float(s.abs().max())
    want = torch.sort(s, 1, descending=True).values
    assert float((s.gather(1, gi.long()) - got.double()).abs().max()) <= off
    assert float((want[:, :k] - got.double()).abs().max()) <= off
    assert float((torch.logsumexp(want[:, k:] / 2, 1) - gr.double()).abs().max()) <= off


def test_float32_head_of_more_rows_than_a_launch_holds(gpu_lib):
    """2^23 frames and more at 512 threads a row: rows on either side of the parts, as in test_head_top_logits."""
    from paper_1907_05701_amd import binding as bd
    T, B, H, P, K, k = 8195, 1024, 16, 8, 136, 129
    M = T * B
    d = bd.make_dims(1, 8, H, P, K, T, B, "fp32")
    g = torch.Generator(device="cuda").manual_seed(5)
    theta = torch.rand(bd.blstm_param_count(d), generator=g, device="cuda") - 0.5
    y = torch.rand(T, B, 2 * H, generator=g, device="cuda") * 2 - 1
    ws = torch.empty(bd.softmax_head_ws_bytes(d), dtype=torch.uint8, device="cuda")
    top, rest = torch.full((M, k), 99.0, device="cuda"), torch.full((M,), 99.0, device="cuda")
    idx = torch.full((M, k), -7, dtype=torch.int32, device="cuda")
    bd.softmax_topk(d, theta, None, y, top, idx, ws, rest, temperature=2.0)
    at = torch.tensor([0, 1] + [n * (1 << 21) + e for n in (1, 2, 3, 4) for e in (-1, 0, 1)] + [M - 2, M - 1])
    th = theta[-(P * 2 * H + P + K * P + K):].double().cpu()
    Wl, bl, Ws, bs = torch.split(th, [P * 2 * H, P, K * P, K])
    s = (y.view(M, -1)[at.cuda()].double().cpu() @ Wl.view(P, -1).t() + bl) @ Ws.view(K, P).t() + bs
    t, i, r = top[at.cuda()].double().cpu(), idx[at.cuda()].long().cpu(), rest[at.cuda()].double().cpu()
    want = torch.sort(s, 1, descending=True).values
    assert float((s.gather(1, i) - t).abs().max()) <= 1e-5
    assert float((want[:, :k] - t).abs().max()) <= 1e-5
    assert float((torch.logsumexp(want[:, k:] / 2, 1) - r).abs().max()) <= 1e-5
    assert int((idx < 0).sum()) == 0 and int((rest == 99.0).sum()) == 0


# -------------------------------------------------- the operators as one run ---
def test_a_causal_student_learns_from_the_blstm_teacher(gpu_lib):
    """Teacher's forward and top logits, then the student's convolution, scan and
    head against them and back: every gradient against float64 autograd of the
    same student (float32 path: the head's 1e-4)."""
    from paper_1907_05701_amd import binding as bd
    from paper_1907_05701_amd.step import LearnerStep
    T, B, H, P, K, k, N, W = 12, 4, 32, 16, 60, 6, 8, 4
    D, M, tau = 2 * H, T * B, 2.0
    g = torch.Generator(device="cuda").manual_seed(21)
    teacher = LearnerStep(L=2, D=8, H=H, P=P, K=K, T=T, B=B, precision="fp32")
    teacher.theta.copy_(torch.rand(teacher.n, generator=g, device="cuda") * 0.6 - 0.3)
    teacher.x.normal_(generator=g)
    teacher.forward()
    teacher.check_recurrence()
    top, idx, rest = teacher.top_logits(k, tau)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x, dt, z, Bm, Cm = r(T, B, D), r(T, B, D) * 0.5, r(T, B, D), r(T, B, N), r(T, B, N)
    w, bias, A, Ds, dtb = r(D, W) * 0.5, r(D) * 0.1, -torch.exp(r(D, N) * 0.3), r(D), r(D) * 0.3 - 2
    student = LearnerStep(L=1, D=8, H=H, P=P, K=K, T=T, B=B, precision="fp32")
    student.theta.copy_(torch.rand(student.n, generator=g, device="cuda") * 0.2 - 0.1)
    student.labels.copy_(torch.randint(0, K, (T, B), generator=g, device="cuda"))
    d = bd.make_ssm_dims(T=T, B=B, D=D, N=N, W=W, precision="fp32")
    ws = {n: torch.empty(max(v, 1), dtype=torch.uint8, device="cuda") for n, v in bd.ssm_workspace_bytes(d).items()}
    e = torch.empty_like
    xc, dxc, dx, ddt, dz, dB, dC = e(x), e(x), e(x), e(x), e(x), e(Bm), e(Cm)
    dw, dbias, dA, dD, ddtb = e(w), e(bias), e(A), e(Ds), e(dtb)
    bd.ssm_conv_fwd(d, x, w, bias, xc)
    bd.ssm_scan_fwd(d, xc, dt, A, Bm, Cm, student.y_top, ws["fwd"], Dskip=Ds, z=z, dt_bias=dtb, saved=ws["saved"])
    student.distill(top, idx, rest, temperature=tau, soft=0.7, hard=0.3)
    bd.ssm_scan_bwd(d, xc, dt, A, Bm, Cm, student.dy_top, ws["saved"], ws["bwd"], dxc, ddt, dA, dB, dC, Dskip=Ds,
                    dDskip=dD, z=z, dz=dz, dt_bias=dtb, ddt_bias=ddtb)
    bd.ssm_conv_bwd(d, x, w, bias, dxc, dx, dw, dbias, ws["conv_bwd"])
    torch.cuda.synchronize()
    c = lambda t: t.double().cpu()  # noqa: E731
    v = {n: c(t).requires_grad_() for n, t in dict(x=x, dt=dt, z=z, Bm=Bm, Cm=Cm, w=w, bias=bias, A=A, Ds=Ds, dtb=dtb).items()}
    y, _ = om.scan(om.conv(v["x"], v["w"], v["bias"])[0], v["dt"], v["A"], v["Bm"], v["Cm"], v["Ds"], v["z"], v["dtb"])
    th = c(student.theta)
    n = 2 * (4 * H * 8 + 4 * H * H + 8 * H)
    Wl, bl, Ws, bs = torch.split(th[n:], [P * D, P, K * P, K])
    s = (y.reshape(M, D) @ Wl.view(P, D).t() + bl) @ Ws.view(K, P).t() + bs
    lab = student.labels.view(-1).cpu()
    loss = sum(om.distill_row(s[m], c(top)[m], idx[m].long().cpu(), c(rest)[m], int(lab[m]), tau, 0.7, 0.3) for m in range(M)) / M
    loss.backward()
    got = dict(x=dx, dt=ddt, z=dz, Bm=dB, Cm=dC, w=dw, bias=dbias, A=dA, Ds=dD, dtb=ddtb)
    err = {a: float((c(t) - v[a].grad).norm() / v[a].grad.norm()) for a, t in got.items()}
    loss = loss.detach()
    err["loss"] = abs(float(student.loss) - float(loss)) / float(loss)
    print("[student]", {a: f"{b:.1e}" for a, b in err.items()}, flush=True)
    assert max(err.values()) <= 1e-4, err


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_a_trainer_with_a_teacher_takes_the_teachers_step(gpu_lib, precision):
    """One epoch of one batch moves the weights as distill()'s gradient says, and
    a captured step repeats an eager one."""
    from paper_1907_05701_amd.step import LearnerStep
    from paper_1907_05701_amd.train import Trainer
    shape = dict(L=1, D=8, H=64, P=16, K=50, T=5, B=4)
    rng = np.random.default_rng(3)
    steps = []
    for i in range(3):
        st = LearnerStep(**shape, precision=precision)
        theta = rng.uniform(-0.2, 0.2, st.n).astype(np.float32) if i != 2 else steps[1].theta.cpu().numpy()
        x = rng.standard_normal((5, 4, 8), dtype=np.float32)
        st.load(theta, x, np.zeros((5, 4), np.int32), theta)
        steps.append(st)
    teacher, a, b = steps
    lab = rng.integers(0, 50, (5, 4)).astype(np.int32)
    Trainer(a, [(x, lab)], 0.1, 4, warmup_epochs=1, teacher=teacher, top=7, temperature=2.0, soft=0.5, hard=0.5).run(1)
    b.x.copy_(torch.from_numpy(x))
    b.labels.copy_(torch.from_numpy(lab))
    teacher.x.copy_(b.x)
    teacher.forward()
    top, idx, rest = teacher.top_logits(7, 2.0)
    t = dict(top=top, idx=idx, rest=rest, temperature=2.0, soft=0.5, hard=0.5)
    start = b.theta.clone()
    b.step(0.1, teacher=t)
    torch.cuda.synchronize()
    assert torch.equal(a.theta, b.theta) and torch.equal(a.loss, b.loss) and not torch.equal(b.theta, start)
    first = b.theta.clone()
    graph = b.capture(0.1, teacher=t)
    for _ in range(3):
        b.theta.copy_(start)
        b.pack()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.theta, first)
