"""GPU: tokens to 8-bit integers, products of integers with scales, and the
8-bit head's log probabilities.  The integers and the products are compared bit
by bit with exact arithmetic (tests/score_models.py): sums of integers are
exact, and each step behind them is one rounding that numpy's float32 makes too."""

import math
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import score_models as sm  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
TOL = 64 * 2.0 ** -24   # as in test_gpu_score.py


def up16(n):
    return -(-n // 16) * 16


def quantize(x, Kq=None):
    from paper_1907_05701_amd import binding as bd
    M, K = x.shape
    q = torch.full((M, up16(K) if Kq is None else Kq), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((M,), 99.0, device="cuda")
    bd.int8_quantize_rows(x, q, scale)
    torch.cuda.synchronize()
    return q, scale


def check_quantize(x, Kq=None):
    q, scale = quantize(x, Kq)
    K = x.shape[1]
    wq, ws = sm.quantize(x.float().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), ws, equal_nan=True)
    assert np.array_equal(q[:, :K].cpu().numpy(), wq)
    assert not bool(q[:, K:].any())


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 1), (3, 15), (5, 16), (6, 17), (5, 260), (4, 511), (3, 1024), (2, 1030), (2, 4100),
                                 (2, 9000), (1, 40000)])
def test_integers(gpu_lib, M, K, precision):
    g = torch.Generator().manual_seed(K)
    x = (torch.randn(M, K, generator=g) * torch.exp(2 * torch.randn(M, 1, generator=g))).to(TYPES[precision]).cuda()
    check_quantize(x)
    check_quantize(x, up16(K) + 48)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("Kq", [16, 4096, 20000])
def test_integers_of_short_rows_in_wide_ones(gpu_lib, Kq, precision):
    """Fewer columns than 16 bytes hold, at the end of their memory, and integers' rows of any length."""
    g = torch.Generator().manual_seed(Kq)
    for K in (1, 3, 7, 9):
        check_quantize(torch.randn(5, K, generator=g).to(TYPES[precision]).cuda(), Kq)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_integers_at_borders(gpu_lib, precision):
    """Ties, values next to them, rows of zeros, the smallest and largest numbers, NaN and infinities."""
    t = TYPES[precision]
    x = torch.zeros(16, 300)
    x[0, 0], x[0, 1:128], x[0, 128:255] = 127.0, torch.arange(127) + 0.5, -(torch.arange(127) + 0.5)
    x[1] = x[0] * (1 + 2.0 ** -7)
    x[2, 0], x[2, 1:128] = 127.0, (torch.arange(127) + 0.5) * (1 - 2.0 ** -23)
    x[3, 0], x[3, 1:128] = 127.0, (torch.arange(127) + 0.5) * (1 + 2.0 ** -23)
    x[4] = -0.0
    x[5] = torch.arange(300) * 2.0 ** -140
    x[6] = torch.arange(300) * 2.0 ** -120
    x[7] = torch.finfo(t).max
    x[7, ::2] = -1.0
    x[8] = torch.finfo(t).max * torch.linspace(-1, 1, 300)
    x[9, 250] = math.nan
    x[10, 3] = math.inf
    x[11, 3] = -math.inf
    x[12] = 1.0
    x[13] = torch.linspace(-1, 1, 300) * 0.3
    x[14, 299] = 5.0
    x[15] = torch.arange(300) / 299.0
    check_quantize(x.to(t).cuda())


def test_integers_of_many_values(gpu_lib):
    """float32 values within a few roundings of a half of a step, a million of them."""
    g = torch.Generator().manual_seed(2)
    top = torch.rand(40, 1, generator=g) + 0.5
    half = torch.randint(0, 127, (40, 25000), generator=g) + 0.5
    x = (half.double() * top.double() / 127).float()
    x = x * (1 + torch.randint(-3, 4, x.shape, generator=g) * 2.0 ** -24).float()
    x[:, :1] = top
    q, scale = quantize(x.cuda())
    v = x.double() * 127 / top.double()                # off by 2^-53 of it, and no border is nearer than 2^-33
    assert torch.equal(q[:, :25000].cpu().double(), torch.round(v))


def ints(M, K, g, full=False):
    return torch.randint(-128 if full else -127, 128, (M, K), generator=g, dtype=torch.int8)


def check_linear(q, w, xs, ws, bias, t, ldpad=0):
    from paper_1907_05701_amd import binding as bd
    M, N = q.shape[0], w.shape[0]
    want = torch.from_numpy(sm.linear(q.numpy(), xs.numpy(), w.numpy(), ws.numpy(), None if bias is None else bias.numpy())).to(t)
    wide = torch.full((M + 2, N + ldpad), 7.0, dtype=t, device="cuda")
    y = wide[1:M + 1, :N]
    bd.int8_linear(q.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y, bias=None if bias is None else bias.cuda())
    torch.cuda.synchronize()
    got = y.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))
    y.fill_(7.0)
    assert bool((wide == 7.0).all())


SIZES = [(1, 1, 16), (1, 16, 64), (1, 4096, 1024), (2, 33, 48), (7, 100, 260 // 16 * 16), (16, 17, 128), (17, 40, 80),
         (33, 50, 272), (64, 256, 1024), (65, 130, 144), (100, 1003, 272), (128, 128, 128), (129, 127, 1024),
         (300, 77, 2064), (257, 300, 112), (520, 260, 16), (1, 3, 16384), (70, 5, 5008)]


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_products(gpu_lib, M, N, K, precision):
    g = torch.Generator().manual_seed(M + N + K)
    q, w = ints(M, K, g, True), ints(N, K, g, True)
    xs, ws, bias = torch.rand(M, generator=g) * 0.01, torch.rand(N, generator=g) * 0.01, torch.randn(N, generator=g)
    check_linear(q, w, xs, ws, bias, TYPES[precision], ldpad=N % 5)
    check_linear(q, w, xs, ws, None, TYPES[precision])


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(4100, 4000, 208), (3900, 4001, 1040), (2000, 2310, 144), (1700, 1600, 80)])
def test_products_that_fill_the_chip(gpu_lib, M, N, K, precision):
    """Each size of tile with ragged ends; outputs whose rows no 16 bytes divide.  float64 products of these are exact."""
    from paper_1907_05701_amd import binding as bd
    t = TYPES[precision]
    g = torch.Generator(device="cuda").manual_seed(M)
    q = torch.randint(-127, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-127, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    xs, ws = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
    bias = torch.randn(N, generator=g, device="cuda")
    s = (q.double() @ w.double().t().contiguous()).float()
    for b in (bias, None):
        want = s * (xs[:, None] * ws)
        want = (want if b is None else want + b).to(t)
        y = torch.full((M + 1, N), 7.0, dtype=t, device="cuda")
        bd.int8_linear(q, xs, w, ws, y[:M], bias=b)
        torch.cuda.synchronize()
        assert torch.equal(y[:M], want) and bool((y[M] == 7.0).all())


def test_the_largest_sums(gpu_lib):
    """Sums next to 2^31, and beyond 2^24, where the float32 of a sum is a rounding."""
    K = 131056
    for M in (2, 70):
        q, w = torch.full((M, K), -128, dtype=torch.int8), torch.full((3, K), -128, dtype=torch.int8)
        w[1, 1000:] = 127
        w[2, ::2] = 127
        q[1, 5::7] = 3
        check_linear(q, w, torch.ones(M), torch.ones(3), None, torch.float32)


def test_scales_of_any_kind(gpu_lib):
    """Scales of zero, NaN, infinities and denormal products travel as float32 says."""
    g = torch.Generator().manual_seed(7)
    q, w = ints(6, 64, g), ints(5, 64, g)
    q[3] = 0
    xs = torch.tensor([0.0, math.nan, 1e-30, math.nan, math.inf, 1.0])
    ws = torch.tensor([1.0, 1e-12, 0.0, 1e30, 2.0])
    bias = torch.tensor([0.0, -math.inf, 1.0, 3.0, math.nan])
    check_linear(q, w, xs, ws, bias, torch.float32)
    check_linear(q, w, xs, ws, None, torch.bfloat16)


def test_rows_at_a_pitch(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    g = torch.Generator().manual_seed(9)
    for M, N in ((5, 40), (90, 200)):
        wide, weights = ints(M, 400, g).cuda(), ints(N, 320, g).cuda()
        q, w = wide[:, 32:240], weights[:, 64:272]
        xs, ws = torch.rand(M, generator=g), torch.rand(N, generator=g)
        y = torch.empty(M, N, device="cuda")
        bd.int8_linear(q, xs.cuda(), w, ws.cuda(), y)
        want = sm.linear(q.cpu().numpy(), xs.numpy(), w.cpu().numpy(), ws.numpy())
        assert np.array_equal(y.cpu().numpy(), want)


def linear_rows(x, w, ws, bias=None, stream=None, y=None, buf=None):
    from paper_1907_05701_amd import binding as bd
    M, N = x.shape[0], w.shape[0]
    y = torch.full((M, N), 7.0, dtype=x.dtype, device="cuda") if y is None else y
    buf = torch.empty(bd.int8_linear_ws_bytes(M, w.shape[1]), dtype=torch.uint8, device="cuda") if buf is None else buf
    bd.int8_linear_rows(x, w, ws, y, buf, bias=bias, stream=stream)
    return y


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 100, 260), (1, 4096, 1024), (3, 50, 1000), (16, 64, 4096), (17, 64, 1024),
                                   (64, 128, 333), (65, 100, 260), (300, 520, 100), (2, 20, 12001), (9, 30, 2500),
                                   (40, 70, 600), (48, 33, 512), (33, 40, 50), (20, 40, 1024), (32, 33, 1025),
                                   (5, 40, 2048), (16, 20, 2049), (1, 40, 5000)])
def test_tokens_times_weights(gpu_lib, M, N, K, precision):
    """Rows of a wider matrix, one of zeros, one with a NaN."""
    t = TYPES[precision]
    g = torch.Generator().manual_seed(M + K)
    wide = torch.randn(M, K + 5, generator=g).to(t)
    if M > 2:
        wide[1] = 0.0
        wide[2, 3] = math.nan
    x, w, ws, bias = wide.cuda()[:, 3:3 + K], ints(N, up16(K), g), torch.rand(N, generator=g) * 0.01, torch.randn(N, generator=g)
    w[:, K:] = 0
    y = linear_rows(x, w.cuda(), ws.cuda(), bias.cuda()).cpu()
    q, xs = sm.quantize(x.float().cpu().numpy())
    want = torch.from_numpy(sm.linear(q, xs, w[:, :K].numpy(), ws.numpy(), bias.numpy())).to(t)
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and bool(torch.isnan(want[2:3]).all())
    assert torch.equal(torch.nan_to_num(y, nan=0.0), torch.nan_to_num(want, nan=0.0))


def test_tokens_of_wider_weights(gpu_lib):
    """Weights with more columns of zeros than their padding."""
    g = torch.Generator().manual_seed(4)
    for M in (2, 40, 90):
        x, w, ws = torch.randn(M, 20, generator=g).cuda(), ints(30, 160, g), torch.rand(30, generator=g).cuda()
        w[:, 20:] = 0
        assert torch.equal(linear_rows(x, w.cuda(), ws), linear_rows(x, w[:, :32].contiguous().cuda(), ws))


def head(x, w, ws, bias, ids=None, k=0, tau=1.0, entropy=True, stream=None, out=None, buf=None):
    from paper_1907_05701_amd import binding as bd
    M = x.shape[0]
    o = out or {"logprob": torch.full(ids.shape, 99.0, device="cuda") if ids is not None else None,
                "entropy": torch.full((M,), 99.0, device="cuda") if entropy else None,
                "top": torch.full((M, k), 99.0, device="cuda") if k else None,
                "idx": torch.full((M, k), -7, dtype=torch.int32, device="cuda") if k else None}
    buf = torch.empty(bd.int8_logprob_ws_bytes(M, *w.shape), dtype=torch.uint8, device="cuda") if buf is None else buf
    bd.int8_logprob_rows(x, w, ws, buf, bias=bias, ids=ids, temperature=tau, stream=stream, **o)
    return o


def near(got, want):
    g, w = got.double().cpu(), want.double().cpu()
    assert torch.equal(torch.isnan(g), torch.isnan(w))
    ok = torch.isfinite(w)
    rest = ~ok & ~torch.isnan(w)
    assert torch.equal(torch.isfinite(g), ok) and torch.equal(g[rest], w[rest])
    assert bool(((g - w).abs()[ok] <= TOL * (1 + w.abs()[ok])).all()), float((g - w).abs()[ok].max())


def check_head(x, w, ws, bias, ids, k, tau=1.0):
    """Against float64 forms of the float32 logits, whose bits the operator's are by its definition."""
    o = head(x, w, ws, bias, ids, k, tau)
    torch.cuda.synchronize()
    q, xs = sm.quantize(x.float().cpu().numpy())
    logits = torch.from_numpy(sm.linear(q, xs, w[:, :x.shape[1]].cpu().numpy(), ws.cpu().numpy(),
                                        None if bias is None else bias.cpu().numpy()))
    rows = logits.double()
    lps = [sm.log_probs(r, tau) for r in rows]
    near(o["entropy"], torch.stack([sm.entropy(r, tau) for r in rows]))
    if ids is not None:
        near(o["logprob"], torch.stack([sm.listed(lp, i) for lp, i in zip(lps, ids.cpu())]))
    if k:
        at = [sm.order(r)[:k] for r in rows]
        assert torch.equal(o["idx"].cpu().long(), torch.stack(at))
        near(o["top"], torch.stack([lp[i] for lp, i in zip(lps, at)]))


def head_case(M, P, K, n, precision, seed=0):
    g = torch.Generator().manual_seed(seed + M + K)
    x = (torch.randn(M, P, generator=g) * 2).to(TYPES[precision]).cuda()
    w, ws = ints(K, up16(P), g), (torch.rand(K, generator=g) + 0.5) * 0.02 / math.sqrt(P)
    w[:, P:] = 0
    ids = torch.randint(-1, K + 1, (M, n), generator=g, dtype=torch.int32).cuda() if n else None
    return x, w.cuda(), ws.cuda(), torch.randn(K, generator=g).cuda(), ids


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("M,P,K,n,k,tau", [(1, 1, 1, 1, 1, 1.0), (1, 256, 1000, 1, 8, 1.0), (3, 16, 40, 2, 40, 2.0),
                                           (16, 256, 3001, 1, 5, 1.0), (33, 100, 515, 3, 0, 0.7), (70, 260, 700, 0, 20, 1.0),
                                           (5, 512, 9001, 256, 256, 1.0), (130, 64, 333, 1, 1, 1.0), (300, 24, 129, 1, 3, 3.0),
                                           (2, 1000, 400, 1, 6, 1.0), (3, 1500, 200, 2, 4, 1.0), (17, 512, 1025, 1, 33, 1.0)])
def test_head(gpu_lib, M, P, K, n, k, tau, precision):
    x, w, ws, bias, ids = head_case(M, P, K, n, precision)
    check_head(x, w, ws, bias, ids, k, tau)
    check_head(x, w, ws, None, ids, k, tau)


@pytest.mark.parametrize("M", [3, 40, 70])
@pytest.mark.parametrize("K,k", [(319, 30), (319, 8), (512, 32), (513, 32), (1000, 30), (1000, 64), (1000, 200), (2100, 65), (8192, 64), (8300, 64)])
def test_head_of_few_classes_and_many_of_them(gpu_lib, M, K, k):
    """Groups of classes fewer than the likely ones, or hardly more; logits that tie."""
    x, w, ws, bias, ids = head_case(M, 64, K, 2, "bf16")
    check_head(x, w, ws, bias, ids, k)
    w[:K // 2], ws[:K // 2] = w[:1], ws[0]
    check_head(x, w, ws, None, None, k)


def test_head_of_the_paper(gpu_lib):
    x, w, ws, bias, ids = head_case(40, 256, 32000, 2, "bf16")
    check_head(x, w, ws, bias, ids, 8)


def test_head_of_the_most_classes(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    x, w, ws, bias, ids = head_case(2, 64, bd.SOFTMAX_MAX_CLASSES, 3, "fp32")
    check_head(x, w, ws, bias, ids, 12)


@pytest.mark.parametrize("K", [60, 2000, 33000])
def test_head_where_logits_bunch(gpu_lib, K):
    """Equal weights, masks of -inf, of -1e9 and of the lowest value, classes that are all masked, NaN in a token and in
    the bias, tokens of zeros, few distinct logits."""
    x, w, ws, bias, ids = head_case(9, 48, K, 3, "fp32")
    x[3] = 0.0
    x[4, 7] = math.nan
    ks = (1, 7, 50)
    for k in ks:
        check_head(x, w, ws, bias, ids, k)
        check_head(x, w[:1].expand(K, 48).contiguous(), ws[:1].expand(K).contiguous(), None, ids, k)
        check_head(x, w, ws, torch.full_like(bias, -math.inf), ids, k)
        check_head(x, w, ws, torch.full_like(bias, torch.finfo(torch.float32).min), ids, k)
        b = bias.clone()
        b[::2] = -math.inf
        b[1::4] = -1e9
        check_head(x, w, ws, b, ids, k)
        b[:] = -1e9
        b[5] = 0.0
        check_head(x, w, ws, b, ids, k)
        b[:] = torch.finfo(torch.float32).min
        b[[2, 11]] = 0.0
        check_head(x, w, ws, b, ids, k)
        b = bias.clone()
        b[17] = math.nan
        b[18] = math.inf
        check_head(x, w, ws, b, ids, k)
        b = bias.clone()
        b[19] = math.inf
        check_head(x, w, ws, b, ids, k)
        check_head(x, (w // 100), ws * 0 + 1.0, torch.round(bias), ids, k)   # whole logits: many ties


def test_head_of_large_logits(gpu_lib):
    """Logits of several thousands, and one class that has all the probability."""
    x, w, ws, bias, ids = head_case(6, 64, 900, 2, "fp32")
    check_head(x, w, ws * 300, bias, ids, 9)
    bias[700] = 5000.0
    check_head(x, w, ws, bias, ids, 9)


def test_head_at_extreme_temperatures(gpu_lib):
    """At 2^100 every class that is not at -inf is alike; at 2^-20 the largest has it all."""
    x, w, ws, bias, ids = head_case(5, 64, 900, 2, "fp32")
    bias[::7] = -math.inf
    check_head(x, w, ws, bias, ids, 9, 2.0 ** 100)
    check_head(x, w, ws, bias, ids, 9, 2.0 ** 40)
    check_head(x, w, ws, bias, ids, 9, 2.0 ** -20)


@pytest.mark.parametrize("M", [1, 20, 70])
def test_head_next_to_no_temperature(gpu_lib, M):
    """Exponents, and the sums' first reference, past what float32 holds."""
    x, w, ws, bias, ids = head_case(M, 64, 900, 2, "fp32")
    bias[::7] = -math.inf
    for tau in (2.0 ** -29, 2.0 ** -31, 2.0 ** -60, 2.0 ** -100):
        check_head(x, w, ws, bias, ids, 9, tau)
        check_head(x, w, ws, None, ids, 0, tau)


def test_head_asks_for_parts_and_leaves_the_rest(gpu_lib):
    x, w, ws, bias, ids = head_case(50, 256, 2000, 4, "bf16")
    full = head(x, w, ws, bias, ids, 6)
    for n, k, e in ((0, 6, True), (4, 0, True), (4, 6, False), (0, 0, True), (4, 0, False), (0, 6, False)):
        part = head(x, w, ws, bias, ids if n else None, k, entropy=e)
        for name, v in part.items():
            if name == "idx":
                assert v is None or torch.equal(v, full[name])
            elif v is not None:
                near(v, full[name])


def test_the_same_every_time_on_another_stream_and_in_graphs(gpu_lib):
    """Two captured graphs with a workspace each, replayed in turn, beside eager calls."""
    from paper_1907_05701_amd import binding as bd
    for M in (1, 12, 50, 300):
        x, w, ws, bias, ids = head_case(M, 256, 3000, 2, "bf16")
        first, y1 = head(x, w, ws, bias, ids, 5), linear_rows(x, w, ws, bias)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        again = {n: torch.zeros_like(v) for n, v in first.items()}
        y2 = torch.zeros_like(y1)
        bufs = [torch.empty(bd.int8_logprob_ws_bytes(M, 3000, 256), dtype=torch.uint8, device="cuda") for _ in range(2)]
        other.wait_stream(torch.cuda.current_stream())
        head(x, w, ws, bias, ids, stream=other, out=again, buf=bufs[0])
        linear_rows(x, w, ws, bias, stream=other, y=y2, buf=bufs[0])
        torch.cuda.synchronize()
        assert torch.equal(y1, y2) and all(torch.equal(first[n], again[n]) for n in first)
        outs, graphs = [{n: torch.zeros_like(v) for n, v in first.items()} for _ in range(2)], []
        ys = [torch.zeros_like(y1) for _ in range(2)]
        for o, y, buf in zip(outs, ys, bufs):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                linear_rows(x, w, ws, bias, y=y, buf=buf)
                head(x, w, ws, bias, ids, out=o, buf=buf)
            graphs.append(graph)
        g = torch.Generator(device="cuda").manual_seed(M)
        for _ in range(3):
            x.copy_(torch.randn(M, 256, generator=g, device="cuda"))
            for graph in graphs:
                graph.replay()
            torch.cuda.synchronize()
            first, y1 = head(x, w, ws, bias, ids, 5), linear_rows(x, w, ws, bias)
            for o, y in zip(outs, ys):
                assert torch.equal(y1, y) and all(torch.equal(first[n], o[n]) for n in first)


@pytest.mark.parametrize("M", [3, 20, 40, 150])
def test_head_of_views(gpu_lib, M):
    """Tokens that are columns of a wider matrix at an odd offset, weights at a pitch, lists that are not all there."""
    for precision in TYPES:
        x, w, ws, bias, ids = head_case(M, 100, 700, 3, precision)
        wide = torch.full((M + 2, 117), math.nan, dtype=x.dtype, device="cuda")
        wide[1:M + 1, 5:105] = x
        far = torch.full((700, 400), 55, dtype=torch.int8, device="cuda")
        far[:, 32:144] = w
        want = head(x, w, ws, bias, ids, 6)
        got = head(wide[1:M + 1, 5:105], far[:, 32:144], ws, bias, ids, 6)
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want)


def test_rows_past_32_bits(gpu_lib):
    """Pitches of 2^22, so that the last rows lie past 2^32 bytes."""
    from paper_1907_05701_amd import binding as bd
    g = torch.Generator().manual_seed(1)
    M, K, ld = 1100, 48, 1 << 22
    far = torch.empty(M * ld, dtype=torch.int8, device="cuda")
    rows = torch.as_strided(far, (M, K), (ld, 1))
    small = ints(M, K, g).cuda()
    rows.copy_(small)
    xs, ys = torch.rand(M, generator=g).cuda(), torch.rand(40, generator=g).cuda()
    few = ints(40, K, g).cuda()
    for q, s, w, t in ((rows, xs, few, ys), (few, ys, rows, xs)):
        a, b = (torch.empty(q.shape[0], w.shape[0], device="cuda") for _ in range(2))
        bd.int8_linear(q, s, w, t, a)
        bd.int8_linear(q.contiguous(), s, w.contiguous(), t, b)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
    x = torch.randn(5, K, generator=g).cuda()
    ids = torch.randint(0, M, (5, 2), generator=g, dtype=torch.int32).cuda()
    a, b = head(x, rows, xs, None, ids, 4), head(x, small, xs, None, ids, 4)
    torch.cuda.synchronize()
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_refusals_of_tensors(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    x, w, ws, bias, ids = head_case(4, 64, 100, 2, "fp32")
    q, s = quantize(x)
    y = torch.empty(4, 100, device="cuda")
    buf = torch.empty(bd.int8_logprob_ws_bytes(4, 100, 64), dtype=torch.uint8, device="cuda")
    for a in ((x, None, ws, y, buf), (x, w[0, 0], ws, y, buf), (x, w[0], ws, y, buf)):
        with pytest.raises(ValueError):
            bd.int8_linear_rows(*a)
        with pytest.raises(ValueError):
            bd.int8_logprob_rows(*a[:3], buf, entropy=torch.empty(4, device="cuda"))
    for a in ((q, s, w, ws, y.double()), (q, s, w, ws, y.t()), (q, s, w, ws, y[:3]), (q, s[:3], w, ws, y), (q, s, w[:99], ws, y),
              (q, s, w, ws[1:], y), (q.float(), s, w, ws, y), (q[:, :48], s, w, ws, y), (q.cpu(), s, w, ws, y),
              (q, s, w.t(), ws, y)):
        with pytest.raises(ValueError):
            bd.int8_linear(*a)
    with pytest.raises(ValueError):
        bd.int8_linear(q, s, w, ws, y, bias=bias.double())
    with pytest.raises(bd.BlstmError):
        bd.int8_linear(q[:, :40], s, w[:, :40], ws, y)                      # 16 does not divide 40
    with pytest.raises(bd.BlstmError):
        bd.int8_linear(q[:, 8:56], s, w[:, :48], ws, y)                     # not aligned
    for a in ((x, w, ws, y.bfloat16(), buf), (x, w, ws, y, buf[:8]), (x, w, ws, y, buf[8:]), (x, w, ws, y, None),
              (x.double(), w, ws, y, buf)):
        with pytest.raises(ValueError):
            bd.int8_linear_rows(*a)
    with pytest.raises(bd.BlstmError):
        bd.int8_linear_rows(torch.zeros(4, 65, device="cuda"), w, ws, y, buf)   # longer than the weights' rows
    e = torch.empty(4, device="cuda")
    for kw in (dict(), dict(entropy=e, ids=ids), dict(entropy=e[:3]), dict(entropy=e, top=y[:, :3].contiguous())):
        with pytest.raises((ValueError, bd.BlstmError)):
            bd.int8_logprob_rows(x, w, ws, buf, **kw)
    for bad in (buf[:64], buf[8:], None):
        with pytest.raises(ValueError):
            bd.int8_logprob_rows(x, w, ws, bad, entropy=e)
