"""GPU: log probabilities of given classes, entropy and most likely classes, and
the gradient of the logits, against float64 forms (tests/score_models.py), row
by row, and on the head.

Tolerances.  TOL = 64 * 2^-24 for the float32 work: an exponent of up to 2^5 (base 2) of what counts carries up to
2^5 half-steps of its own rounding into the exponential, doubled by the scaling; sums add in a tree.  A log
probability and an entropy are off by TOL relative to 1 and their own size; a gradient by TOL relative to the size of
the terms that add up to it, and half a step of its type."""

import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import operator_models as om  # noqa: E402
import score_models as sm  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
TOL = 64 * 2.0 ** -24


def run(s, ids=None, k=0, tau=1.0, entropy=True, stream=None):
    from paper_1907_05701_amd import binding as bd
    M = s.shape[0]
    o = {"logprob": torch.full(ids.shape, 99.0, device="cuda") if ids is not None else None,
         "entropy": torch.full((M,), 99.0, device="cuda") if entropy else None,
         "top": torch.full((M, k), 99.0, device="cuda") if k else None,
         "idx": torch.full((M, k), -7, dtype=torch.int32, device="cuda") if k else None}
    bd.softmax_logprob_rows(s, ids=ids, temperature=tau, stream=stream, **o)
    return o


def near(got, want):
    """Within TOL of 1 and the value; infinities and NaN in the same places."""
    g, w = got.double().cpu(), want.double()
    assert torch.equal(torch.isnan(g), torch.isnan(w))
    ok = torch.isfinite(w)
    rest = ~ok & ~torch.isnan(w)
    assert torch.equal(torch.isfinite(g), ok) and torch.equal(g[rest], w[rest])
    assert bool(((g - w).abs()[ok] <= TOL * (1 + w.abs()[ok])).all()), float(((g - w).abs()[ok]).max())


def check(s, ids, k, tau=1.0, only=None):
    """`only`: the rows looked at."""
    o = run(s, ids, k, tau)
    torch.cuda.synchronize()
    if only is not None:
        o = {n: None if t is None else t[only] for n, t in o.items()}
        s, ids = s[only], None if ids is None else ids[only]
    rows = s.double().cpu()
    lps = [sm.log_probs(r, tau) for r in rows]
    near(o["entropy"], torch.stack([sm.entropy(r, tau) for r in rows]))
    if ids is not None:
        near(o["logprob"], torch.stack([sm.listed(lp, i) for lp, i in zip(lps, ids.cpu())]))
    if k:
        at = [sm.order(r)[:k] for r in rows]
        assert torch.equal(o["idx"].cpu().long(), torch.stack(at))
        near(o["top"], torch.stack([lp[i] for lp, i in zip(lps, at)]))


def some_ids(M, K, n, seed=0):
    """Classes at random, some listed twice, some that are none."""
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(-2, K + 2, (M, n), generator=g, dtype=torch.int32)
    if n > 2:
        ids[:, 2] = ids[:, 0]
    return ids.cuda()


SHAPES = [(1, 1, 1, 1, 1.0), (3, 2, 2, 1, 0.5), (4, 7, 3, 7, 2.0), (5, 63, 1, 0, 1.0), (5, 64, 5, 64, 1.0), (6, 65, 0, 2, 3.0),
          (9, 100, 8, 8, 2.0), (2, 511, 256, 256, 1.0), (7, 700, 2, 33, 1.0), (5, 1024, 1, 5, 1.0), (5, 1025, 1, 5, 0.7),
          (3, 2049, 4, 9, 1.0), (3, 4001, 33, 33, 1.0), (2, 16391, 3, 64, 1.0), (2, 32000, 32, 32, 1.0),
          (2, 32000, 7, 200, 3.0), (2, 40007, 64, 64, 1.0), (1, 131072, 3, 8, 1.0), (2, 70001, 0, 130, 2.0)]


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,n,k,tau", SHAPES)
def test_rows(gpu_lib, M, K, n, k, tau, precision):
    g = torch.Generator().manual_seed(K + k)
    s = (torch.randn(M, K, generator=g) * 3).to(TYPES[precision]).cuda()
    check(s, some_ids(M, K, n) if n else None, k, tau)


def test_rows_of_the_most_classes(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    g = torch.Generator().manual_seed(1)
    check((torch.randn(2, bd.SOFTMAX_MAX_CLASSES, generator=g) * 3).bfloat16().cuda(), some_ids(2, bd.SOFTMAX_MAX_CLASSES, 9), 16)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [90, 800, 3000, 20000, 70001])
def test_rows_that_masks_or_ties_bend(gpu_lib, K, precision):
    """Ties over whole rows, ascending and descending rows, masks of -inf, of the type's lowest value and of -1e9, rows
    with nothing left, infinities and NaN."""
    t = TYPES[precision]
    low = torch.finfo(t).min
    s = torch.zeros(14, K)
    s[1] = torch.arange(K) / 64
    s[2] = -torch.arange(K) / 64
    s[3, :16] = 5.0
    s[3, K - 16:] = 7.0
    s[4] = low
    s[4, 70] = 1.0
    s[5] = -math.inf
    s[5, [3, K - 2]] = torch.tensor([2.0, 1.0])
    s[6, 10:K - 4] = math.nan
    s[7] = -0.0
    s[7, ::2] = 0.0
    s[8, [9, 17]] = math.inf
    s[9] = -math.inf
    s[10] = low
    s[11] = -1e9
    s[12] = -1e9
    s[12, 5:45] = torch.linspace(-3, 3, 40)
    s[13, :] = 100.0
    s[13, K - 1] = -math.inf
    s = s.to(t).cuda()
    for k in (0, 1, 40, 80):
        check(s, some_ids(14, K, 6, seed=k), k)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K,k,n", [(200, 32, 64), (500, 33, 1), (1030, 32, 64), (2000, 5, 65), (2049, 0, 3), (4001, 32, 2), (4097, 7, 1)])
def test_many_rows(gpu_lib, K, k, n, precision):
    """Rows enough to fill the card: ties over all classes and over a part, rows with nothing left, infinities, NaN."""
    t = TYPES[precision]
    s = torch.randn(1100, K, generator=torch.Generator().manual_seed(K)) * 3
    s[3] = 0.0
    s[500, 10:K - 90] = 9.0
    s[501] = torch.arange(K) / 64
    s[700] = -math.inf
    s[701] = torch.finfo(t).min
    s[702, :K - 2] = -math.inf
    s[900, K // 2] = math.nan
    s[1098, 7] = math.inf
    s[1099] = math.nan
    check(s.to(t).cuda(), some_ids(1100, K, n), k, only=[*range(0, 1100, 37), 3, 500, 501, 700, 701, 702, 900, 1098, 1099])


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K,k", [(300, 32), (4000, 20), (9001, 130), (32000, 8), (140001, 32)])
def test_rows_of_many_ties(gpu_lib, K, k, precision):
    """Fewer classes above the ties than are asked for, ties at the end of a row alone, at any place, beside NaN and infinities,
    several levels of them, and more than fit above the threshold."""
    s = torch.full((9, K), -3.0)
    s[0, torch.arange(k // 2) * 7 % K] = torch.linspace(1, 2, k // 2)
    s[1] = torch.arange(K) % 2 * -1.0
    s[2, :] = -50.0 - torch.arange(K) % 64
    s[2, K - 3 * k // 2:] = 1.0
    s[3, [5, K - 1, K // 2]] = math.nan
    s[4, [6, K - 2]] = math.inf
    s[4, 7] = math.nan
    s[5] = torch.arange(K) % 5 * 1.0
    s[6, : K // 3] = -math.inf
    s[6, K // 3: K // 3 + 3] = 4.0
    s[7, :K - k // 2] = -math.inf
    s[8] = (torch.arange(K) // 16) * 0.0
    s[8, torch.randperm(K, generator=torch.Generator().manual_seed(3))[:K // 2]] = -0.0
    check(s.to(TYPES[precision]).cuda(), some_ids(9, K, 2), k)


def test_logits_far_from_zero(gpu_lib):
    """Only differences count: the same rows 1e4 and 1e6 away, where float32 still holds them."""
    g = torch.Generator().manual_seed(4)
    base = torch.round(torch.randn(3, 3001, generator=g) * 64) / 16
    for off in (0.0, 1e4, -1e6):
        check((base + off).cuda(), some_ids(3, 3001, 4), 7)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [130, 900, 9001, 33001])
def test_views_and_what_is_not_asked_for(gpu_lib, K, precision):
    """Rows of a wider matrix, at odd offsets.  A subset of the outputs may be another kernel's (short rows, by k), whose sums
    add up in another order: both are within TOL of the exact values, and so within twice that of each other."""
    g = torch.Generator().manual_seed(K)
    wide = (torch.randn(6, K + 37, generator=g) * 3).to(TYPES[precision]).cuda()
    s, ids = wide[1:, 3:3 + K], some_ids(5, K, 5)
    check(s, ids, 9)
    full = run(s, ids, 9)
    for n, k, e in ((0, 9, True), (5, 0, True), (5, 9, False), (0, 0, True), (5, 0, False), (0, 9, False)):
        part = run(s, ids if n else None, k, entropy=e)
        for name, v in part.items():
            if name == "idx":
                assert v is None or torch.equal(v, full[name])
            elif v is not None:
                assert bool(((v - full[name]).abs() <= 2 * TOL * (1 + v.abs())).all())


def grad(s, ids, g, h, tau=1.0, out=None, stream=None):
    from paper_1907_05701_amd import binding as bd
    d = torch.full_like(s, 7.0) if out is None else out
    bd.softmax_logprob_bwd_rows(s, d, ids=ids, dlogprob=g, dentropy=h, temperature=tau, stream=stream)
    return d


def check_grad(s, ids, g, h, tau=1.0, d=None):
    if d is None:
        d = grad(s, ids, g, h, tau)
    torch.cuda.synchronize()
    M = s.shape[0]
    for m in range(M):
        i = ids[m].cpu() if ids is not None else torch.zeros(0, dtype=torch.int32)
        gm = g[m].double().cpu() if g is not None else torch.zeros(0, dtype=torch.float64)
        want, size = sm.gradient(s[m].double().cpu(), i, gm, float(h[m]) if h is not None else 0.0, tau)
        got = d[m].double().cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        bound = om.half_step(s.dtype) * want.abs() + TOL * size + 1e-30
        assert bool((((got - want).abs() <= bound) | torch.isnan(want)).all()), m


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K,n,tau", [(1, 1, 1, 1.0), (3, 2, 1, 0.5), (4, 7, 3, 2.0), (5, 100, 8, 2.0), (2, 513, 256, 1.0),
                                       (7, 700, 2, 1.0), (3, 4001, 33, 1.0), (2, 16391, 3, 0.7), (2, 32000, 1, 1.0),
                                       (2, 40007, 64, 1.0), (1, 131073, 3, 1.0)])
def test_gradient(gpu_lib, M, K, n, tau, precision):
    g = torch.Generator().manual_seed(K + n)
    s = (torch.randn(M, K, generator=g) * 3).to(TYPES[precision]).cuda()
    ids, dl, dh = some_ids(M, K, n), torch.randn(M, n, generator=g).cuda(), torch.randn(M, generator=g).cuda()
    check_grad(s, ids, dl, dh, tau)
    check_grad(s, ids, dl, None, tau)
    check_grad(s, None, None, dh, tau)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [90, 3000, 70001])
def test_gradient_of_rows_that_masks_bend(gpu_lib, K, precision):
    """Rows without a gradient stay zero whatever they hold; masked rows, rows with nothing left, NaN and infinities."""
    t = TYPES[precision]
    g = torch.Generator().manual_seed(K)
    s = torch.randn(10, K, generator=g)
    s[1, ::3] = -math.inf
    s[2] = -math.inf
    s[3, 5] = math.nan
    s[4, 6] = math.inf
    s[5] = math.nan
    s[6] = torch.finfo(t).min
    s[7] = -1e9
    s[7, 3] = 4.0
    ids = some_ids(10, K, 4)
    ids[1, 1] = 3          # a masked class
    dl, dh = torch.randn(10, 4, generator=g), torch.randn(10, generator=g)
    dl[5], dh[5] = 0.0, 0.0
    dl[8], dh[8] = 0.0, 0.0
    ids[9] = -1
    dh[9] = 0.0
    s = s.to(t).cuda()
    check_grad(s, ids, dl.cuda(), dh.cuda())
    d = grad(s, ids, dl.cuda(), dh.cuda())
    assert bool((d[[2, 5, 8, 9]] == 0).all())


def test_gradient_against_differences_of_the_forward(gpu_lib):
    """Central differences of the kernel's own log probabilities and entropy, float32: a step of 2^-6 has a truncation
    error of 2^-12 / 6 of the third derivative (at most 1), and the outputs' TOL over the step."""
    K, e = 90, 2.0 ** -6
    g = torch.Generator().manual_seed(0)
    s = torch.randn(1, K, generator=g)
    ids = torch.tensor([[3, 50, 3]], dtype=torch.int32)
    dl, dh = torch.tensor([[0.5, -1.0, 0.25]]), torch.tensor([0.7])
    both = torch.cat([s + e * torch.eye(K), s - e * torch.eye(K)])
    o = run(both.cuda(), ids.expand(2 * K, 3).contiguous().cuda())
    loss = (o["logprob"].cpu() * dl).sum(1) + o["entropy"].cpu() * dh
    want = (loss[:K] - loss[K:]) / (2 * e)
    got = grad(s.cuda(), ids.cuda(), dl.cuda(), dh.cuda())[0].cpu()
    assert float((got - want).abs().max()) <= 2 * 2.0 ** -12 / 6 * 8 + 4 * TOL * 6 / e


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [100, 9001, 70003])
def test_gradient_in_place_and_between_guards(gpu_lib, K, precision):
    t = TYPES[precision]
    g = torch.Generator().manual_seed(K)
    s = (torch.randn(4, K, generator=g) * 2).to(t).cuda()
    ids, dl, dh = some_ids(4, K, 5), torch.randn(4, 5, generator=g).cuda(), torch.randn(4, generator=g).cuda()
    want = grad(s, ids, dl, dh)
    wide = torch.full((6, K + 11), 5.0, dtype=t, device="cuda")
    grad(s, ids, dl, dh, out=wide[1:5, 4:4 + K])
    assert torch.equal(wide[1:5, 4:4 + K], want)
    wide[1:5, 4:4 + K] = 5.0
    assert bool((wide == 5.0).all())
    work = s.clone()
    grad(work, ids, dl, dh, out=work)
    assert torch.equal(work, want)


def test_the_same_every_time_on_another_stream_and_in_a_graph(gpu_lib):
    g = torch.Generator(device="cuda").manual_seed(8)
    for K in (300, 900, 32000, 70000):
        s = torch.randn(64, K, generator=g, device="cuda") * 3
        ids, dl = some_ids(64, K, 4), torch.randn(64, 4, generator=g, device="cuda")
        first, dfirst = run(s, ids, 9), grad(s, ids, dl, None)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        again, dagain = run(s, ids, 9, stream=other), torch.empty_like(s)
        other.wait_stream(torch.cuda.current_stream())
        grad(s, ids, dl, None, out=dagain, stream=other)
        torch.cuda.synchronize()
        assert all(torch.equal(first[n], again[n]) for n in first) and torch.equal(dfirst, dagain)
        again["top"].zero_()
        dagain.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            from paper_1907_05701_amd import binding as bd
            bd.softmax_logprob_rows(s, ids=ids, **again)
            grad(s, ids, dl, None, out=dagain)
        for seed in range(3):
            s.copy_(torch.randn(64, K, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            first, dfirst = run(s, ids, 9), grad(s, ids, dl, None)
            assert all(torch.equal(first[n], again[n]) for n in first) and torch.equal(dfirst, dagain)


@pytest.mark.parametrize("K", [200, 3000])
def test_rows_past_32_bits(gpu_lib, K):
    """A pitch of 2^24 elements: the last rows lie past 2^32 bytes and 2^31 elements."""
    M, ld = 140, 1 << 24
    far = torch.empty(M * ld, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(far, (M, K), (ld, 1))
    g = torch.Generator(device="cuda").manual_seed(K)
    small = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    rows.copy_(small)
    ids, dl = some_ids(M, K, 2), torch.randn(M, 2, generator=g, device="cuda")
    a, b = run(rows, ids, 3), run(small, ids, 3)
    d = grad(small, ids, dl, None)
    grad(rows, ids, dl, None, out=rows)
    torch.cuda.synchronize()
    assert all(torch.equal(a[n], b[n]) for n in a) and torch.equal(rows, d)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K,n", [(500, 64), (513, 65), (700, 64), (1030, 64), (2000, 3), (2049, 65), (4001, 1), (4097, 2)])
def test_gradients_of_many_rows(gpu_lib, K, n, precision):
    M, only = 1100, [*range(0, 1100, 37), 3, 500, 700, 702, 900, 1098]
    g = torch.Generator().manual_seed(K)
    s = torch.randn(M, K, generator=g) * 3
    s[3] = 0.0
    s[500] = torch.finfo(TYPES[precision]).min
    s[700] = -math.inf
    s[702, :K - 2] = -math.inf
    s[1098, 5] = math.nan
    s = s.to(TYPES[precision]).cuda()
    dl, dh = torch.randn(M, n, generator=g), torch.randn(M, generator=g)
    dl[900], dh[900] = 0.0, 0.0
    ids = some_ids(M, K, n)
    d = grad(s, ids, dl.cuda(), dh.cuda())
    check_grad(s[only], ids[only], dl[only], dh[only], d=d[only])
    assert not d[900].any()
    over = s.clone()
    assert torch.equal(grad(over, ids, dl.cuda(), dh.cuda(), out=over).nan_to_num(9.0), d.nan_to_num(9.0))


@pytest.mark.parametrize("K", [90, 3000, 33000])
def test_extreme_temperatures(gpu_lib, K):
    s = torch.randn(5, K, generator=torch.Generator().manual_seed(K))
    s[1, ::3] = -math.inf
    s[2] = torch.finfo(torch.float32).min
    s[3] = -math.inf
    for tau in (2.0 ** 100, 2.0 ** 40, 2.0 ** -20, 2.0 ** -31, 2.0 ** -60, 2.0 ** -100):
        check(s.cuda(), some_ids(5, K, 3), 5, tau)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("K,n", [(2, 64), (40, 64), (64, 65), (200, 17), (512, 9), (700, 64), (3000, 256), (9001, 130), (32768, 256), (40007, 200)])
def test_gradients_of_lists_that_repeat(gpu_lib, K, n, precision):
    """Few classes listed many times, the same one throughout, classes a power of two apart, ids that are none."""
    g = torch.Generator().manual_seed(n)
    s = (torch.randn(7, K, generator=g) * 2).to(TYPES[precision]).cuda()
    ids = torch.randint(0, K, (7, n), generator=g, dtype=torch.int32)
    ids[0] = K - 1
    ids[1] = torch.arange(n) % 3 * (K // 2) % K
    ids[2] = torch.arange(n).flip(0) % K
    ids[3] = (1 << torch.arange(n) % 18) % K
    ids[4, ::2] = -1
    ids[4, 1::2] = K - 1
    ids[5] = torch.where(torch.arange(n) % 2 == 0, K, -5 - torch.arange(n))
    ids[6, n // 2:] = -1
    check_grad(s, ids.cuda(), torch.randn(7, n, generator=g).cuda(), torch.randn(7, generator=g).cuda())
    check_grad(s, ids.cuda(), torch.randn(7, n, generator=g).cuda(), None, 0.7)


def test_many_rows_of_few_classes(gpu_lib):
    """More rows than 16 bits count, each by a wave."""
    M, K = 70001, 5
    g = torch.Generator(device="cuda").manual_seed(2)
    s = torch.randn(M, K, generator=g, device="cuda")
    ids = torch.randint(0, K, (M, 1), generator=g, device="cuda", dtype=torch.int32)
    o = run(s, ids, 2)
    d = grad(s, ids, torch.ones(M, 1, device="cuda"), None)
    lp = torch.log_softmax(s.double(), 1)
    near(o["logprob"], lp.gather(1, ids.long()).cpu())
    near(o["top"], lp.topk(2).values.cpu())
    want = torch.zeros_like(lp).scatter_(1, ids.long(), 1.0) - lp.exp()
    assert float((d - want).abs().max()) <= 2 * TOL


def test_refusals_of_tensors(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    s = torch.zeros(4, 50, device="cuda")
    f, i = torch.zeros(4, 3, device="cuda"), torch.zeros(4, 3, dtype=torch.int32, device="cuda")
    for kw in (dict(ids=i), dict(logprob=f), dict(ids=i.long(), logprob=f), dict(ids=i, logprob=f[:, :2]), dict(top=f),
               dict(idx=i), dict(top=f, idx=i.t()), dict(entropy=f), dict(ids=i.cpu(), logprob=f), dict(ids=i[:3], logprob=f)):
        with pytest.raises(ValueError):
            bd.softmax_logprob_rows(s, **kw)
    with pytest.raises(bd.BlstmError):
        bd.softmax_logprob_rows(s)
    for bad in (s.double(), s.t()[:, :3], s[:, ::2], s[0]):
        with pytest.raises(ValueError):
            bd.softmax_logprob_rows(bad, entropy=torch.zeros(bad.shape[0], device="cuda"))
    for kw in (dict(ids=i), dict(dlogprob=f), dict(ids=i, dlogprob=f.double()), dict(dentropy=f)):
        with pytest.raises(ValueError):
            bd.softmax_logprob_bwd_rows(s, torch.empty_like(s), **kw)
    with pytest.raises(ValueError):
        bd.softmax_logprob_bwd_rows(s, s.bfloat16(), ids=i, dlogprob=f)
    with pytest.raises(bd.BlstmError):   # over the logits at another pitch
        wide = torch.zeros(4, 100, device="cuda")
        bd.softmax_logprob_bwd_rows(wide[:, :40], torch.as_strided(wide, (4, 40), (50, 1)), ids=i, dlogprob=f)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("P,K", [(32, 100), (24, 203)])
def test_on_the_head(gpu_lib, P, K, precision):
    """Forward: as the rows of the head's own logits, which its top logits show.  Backward: the head's gradients are linear in
    dlogits, so that those of the label's log probability are those of the cross-entropy, of the other sign."""
    from paper_1907_05701_amd import binding as bd
    T, B, H = 21, 8, 64
    dims = bd.make_dims(2, 40, H, P, K, T, B, precision)
    g = torch.Generator(device="cuda").manual_seed(P)
    n, M, t = bd.blstm_param_count(dims), T * B, TYPES[precision]
    theta = (torch.rand(n, generator=g, device="cuda") - 0.5) * 0.4
    lp = theta.to(torch.bfloat16) if precision == "bf16" else None
    y = (torch.randn(T, B, 2 * H, generator=g, device="cuda") * 0.7).to(t)
    ws = torch.empty(bd.softmax_head_ws_bytes(dims), dtype=torch.uint8, device="cuda")
    # every logit, in descending order
    top, idx = torch.empty(M, K, device="cuda"), torch.empty(M, K, dtype=torch.int32, device="cuda")
    bd.softmax_topk(dims, theta, lp, y, top, idx, ws)
    logits = torch.empty(M, K, device="cuda").scatter_(1, idx.long(), top)
    ids, k = some_ids(M, K, 3), 5
    o = {"logprob": torch.empty(M, 3, device="cuda"), "entropy": torch.empty(M, device="cuda"),
         "top": torch.empty(M, k, device="cuda"), "idx": torch.empty(M, k, dtype=torch.int32, device="cuda")}
    bd.softmax_logprob(dims, theta, lp, y, ws, ids=ids, temperature=2.0, **o)
    want = run(logits, ids, k, 2.0)
    for name in o:
        assert torch.equal(o[name], want[name]), name

    labels = torch.randint(0, K, (M,), generator=g, device="cuda", dtype=torch.int32)
    loss, hws = torch.zeros(1, device="cuda"), torch.empty(bd.blstm_workspace_bytes(dims)["head_ws"], dtype=torch.uint8, device="cuda")
    dy, grad_ = torch.zeros(T, B, 2 * H, device="cuda"), torch.zeros(n, device="cuda")
    bd.softmax_ce_fwd_bwd(dims, theta, lp, y, labels.view(T, B), 1.0 / M, loss, dy, grad_, hws)
    dy2, grad2 = torch.zeros_like(dy), torch.zeros_like(grad_)
    bd.softmax_logprob_bwd(dims, theta, lp, y, dy2, grad2, ws, ids=labels.view(M, 1),
                           dlogprob=torch.full((M, 1), -1.0 / M, device="cuda"))
    torch.cuda.synchronize()
    # bf16: dlogits rounded on both sides from float32 values that differ in their last bits, and so dz
    tol = 3e-6 if precision == "fp32" else 2 * 2.0 ** -8
    assert float((dy2 - dy).norm() / dy.norm()) <= tol and float((grad2 - grad_).norm() / grad_.norm()) <= tol

    # the entropy's gradient, along a direction of the head's parameters, float32: against differences in 64 bits
    if precision == "fp32":
        bd.softmax_logprob_bwd(dims, theta, lp, y, dy2, grad2, ws, dentropy=torch.full((M,), 1.0 / M, device="cuda"))
        torch.cuda.synchronize()
        H2, at = 2 * H, n - (P * 2 * H + P + K * P + K)
        way = torch.randn(n - at, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
        base, yd = theta[at:].double().cpu(), y.view(M, H2).double().cpu()

        def ent(v):
            Wl, bl, Ws, bs = torch.split(v, [P * H2, P, K * P, K])
            s = (yd @ Wl.view(P, H2).t() + bl) @ Ws.view(K, P).t() + bs
            lpd = torch.log_softmax(s, 1)
            return float(-(lpd.exp() * lpd).sum(1).mean())
        e = 1e-5
        d = (ent(base + e * way) - ent(base - e * way)) / (2 * e)
        got = float((grad2[at:].double().cpu() * way).sum())
        size = float((grad2[at:].double().cpu() * way).norm())
        assert abs(got - d) <= 1e-4 * size
