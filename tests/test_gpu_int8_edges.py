"""GPU: the 8-bit head where its logits, products or sizes are far from a trained model's.  Compared with float64
forms of the float32 logits as in test_gpu_int8.py."""

import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_gpu_int8 as t8  # noqa: E402

pytestmark = pytest.mark.gpu
LOG2E = 1.4426950408889634


@pytest.mark.parametrize("M", [1, 6, 20, 40, 150])
def test_head_of_classes_far_above_the_others(gpu_lib, M):
    """One class, two alike, or several at powers of two and other numbers up to 10^37: their log probability is 0, or
    what they share, and the others' the distance."""
    x, w, ws, bias, ids = t8.head_case(M, 64, 900, 2, "fp32")
    ids[:, 0] = 700
    for tau in (1.0, LOG2E, 0.25, 3.0):
        for top in (2.0 ** 27, 2.0 ** 40, 2.0 ** 100, 3e30, 1e37):
            b = bias.clone()
            b[700] = top
            t8.check_head(x, w, ws, b, ids, 9, tau)
    for top in (2.0 ** 31, 2.0 ** 100, 1e37):
        b = bias.clone()
        b[[3, 700]] = top
        t8.check_head(x, w * 0, ws, b, ids, 9)
        b[:] = top
        t8.check_head(x, w, ws, b, ids, 9)


@pytest.mark.parametrize("M", [1, 6, 20, 40, 150])
@pytest.mark.parametrize("size", [1e7, 1e9, 1e12, 1e20, 1e30, 1e33, 1e36])
def test_head_of_logits_of_any_size(gpu_lib, M, size):
    """Scales that make every logit so large."""
    x, w, ws, bias, ids = t8.head_case(M, 64, 900, 2, "fp32")
    t8.check_head(x, w, ws * size, bias, ids, 9)
    t8.check_head(x, w, ws * size, bias * size, ids, 9, 2.0)


@pytest.mark.parametrize("M", [1, 6, 40, 150])
@pytest.mark.parametrize("top", [-1e29, 0.0, 1e27, 5e28, 2e29, 5e29])
def test_head_of_masks_below_large_logits(gpu_lib, M, top):
    """Classes at -2e30, -1.1e30 and the type's lowest value below a largest logit of up to 5e29, listed and likely."""
    x, w, ws, bias, ids = t8.head_case(M, 64, 100, 3, "fp32")
    ids[:] = torch.tensor([10, 40, 70], dtype=torch.int32)
    b = torch.full_like(bias, -2e30)
    b[30:60], b[60:] = -1.1e30, torch.finfo(torch.float32).min / 4
    b[5] = top
    t8.check_head(x, w, ws, b, ids, 70)


@pytest.mark.parametrize("M", [1, 6, 20, 40, 150])
def test_head_of_masks_that_products_lift(gpu_lib, M):
    """A bias of -2e30 with a product of exactly 10^30, or of more, or of -3e38, beside ordinary classes: the class is at
    the sum of both."""
    x, w, ws, bias, ids = t8.head_case(M, 64, 900, 2, "fp32")
    x[:, 0], x[:, 1] = 127.0, 1.0                       # integers are the values themselves: a scale of 1
    x[:, 2:] = torch.round(x[:, 2:])
    ws = ws / 1000                                      # the others' logits are next to their biases
    ids[:, 0] = 700
    w[700] = 0
    w[700, 1] = 1                                       # the sum is 1, the product the scale
    assert bool((t8.quantize(x)[1] == 1.0).all())
    for scale in (1e30, 1.0000001e30, 2e30, 1.7e38, -3e38, 1e10):
        for mask in (-2e30, -1.0000001e30, -1e38, -1e30, float("-inf")):
            s, b = ws.clone(), bias.clone()
            s[700], b[700] = scale, mask
            t8.check_head(x, w, s, b, ids, 9)
    x = x * 1e12                                        # a scale of 10^12 for the tokens
    s, b = ws * 1e-12, bias.clone()
    s[700], b[700] = 1e18, -2e30                        # the product is 10^30 again
    t8.check_head(x, w, s, b, ids, 9)


def rows_of(o, at):
    return {n: v if v is None else v[at] for n, v in o.items()}


def check_rows(o, at, x, w, ws, bias, ids, k):
    """Rows `at` of the head's answers, as check_head does."""
    o, x, ids = rows_of(o, at), x[at], ids[at]
    q, xs = t8.sm.quantize(x.float().cpu().numpy())
    rows = torch.from_numpy(t8.sm.linear(q, xs, w[:, :x.shape[1]].cpu().numpy(), ws.cpu().numpy(), bias.cpu().numpy())).double()
    lps, orders = [t8.sm.log_probs(r, 1.0) for r in rows], [t8.sm.order(r)[:k] for r in rows]
    t8.near(o["entropy"], torch.stack([t8.sm.entropy(r, 1.0) for r in rows]))
    t8.near(o["logprob"], torch.stack([t8.sm.listed(lp, i) for lp, i in zip(lps, ids.cpu())]))
    assert torch.equal(o["idx"].cpu().long(), torch.stack(orders))
    t8.near(o["top"], torch.stack([lp[i] for lp, i in zip(lps, orders)]))


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_head_of_more_frames_than_a_part(gpu_lib, precision):
    """Two parts, the second one shorter: every frame has its own list and answers.  (A part holds at most
    180 * 2^20 / (32 + 16 * 4096 + 64) = 2875 frames of 262144 classes and 32 columns.)"""
    from paper_1907_05701_amd import binding as bd
    M, K, k = 5701, bd.SOFTMAX_MAX_CLASSES, 3
    x, w, ws, bias, ids = t8.head_case(M, 20, K, 2, precision)
    n = -(-M // 2)
    assert bd.int8_logprob_ws_bytes(M, K, 32) < M * K // 4
    wide = torch.full((M, 27), 1e9, dtype=x.dtype, device="cuda")
    wide[:, 4:24] = x
    o = t8.head(wide[:, 4:24], w, ws, bias, ids, k)
    for r0 in range(0, M, n):
        part = t8.head(x[r0:r0 + n], w, ws, bias, ids[r0:r0 + n], k)
        torch.cuda.synchronize()
        for name, v in part.items():
            assert torch.equal(v, o[name][r0:r0 + n]), (name, r0)
    check_rows(o, torch.tensor([0, n - 1, n, M - 1]), x, w, ws, bias, ids, k)


def test_a_product_needs_its_output(gpu_lib):
    from paper_1907_05701_amd import binding as bd
    q, s = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    with pytest.raises(ValueError, match="y is required"):
        bd.int8_linear(q, s, q, s, None)


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
def test_head_of_long_tokens_in_parts(gpu_lib, precision):
    """More than 1024 columns, whose logits go through memory, 180 * 2^20 / 400000 = 471 frames of 100000 classes at a
    time: bit by bit what the product and the rows' operator give in turn."""
    from paper_1907_05701_amd import binding as bd
    M, K, k = 500, 100000, 4
    x, w, ws, bias, ids = t8.head_case(M, 1030, K, 2, precision)
    o = t8.head(x, w, ws, bias, ids, k)
    logits = t8.linear_rows(x.float(), w, ws, bias)
    want = {n: torch.empty_like(v) for n, v in o.items()}
    bd.softmax_logprob_rows(logits, ids=ids, **want)
    torch.cuda.synchronize()
    for name, v in want.items():
        assert torch.equal(v, o[name]), name
    check_rows(o, torch.tensor([0, 470, 471, M - 1]), x, w, ws, bias, ids, k)


@pytest.mark.parametrize("M,P", [(17, 512), (40, 300), (64, 512)])
def test_head_of_some_frames_and_many_classes(gpu_lib, M, P):
    x, w, ws, bias, ids = t8.head_case(M, P, 45000, 2, "bf16")
    o = t8.head(x, w, ws, bias, ids, 7)
    torch.cuda.synchronize()
    check_rows(o, torch.tensor([0, 15, 16, M - 1]), x, w, ws, bias, ids, 7)


@pytest.mark.parametrize("M", [1, 20, 40, 150])
def test_head_on_either_side_of_the_largest_reference(gpu_lib, M):
    """Largest exponents from 2^25 to 2^29, of one class, of many that tie, of all by their scales, and of ordinary logits at
    small temperatures."""
    x, w, ws, bias, ids = t8.head_case(M, 64, 900, 2, "fp32")
    for top in (2.5e7, 6e7, 1.2e8, 1.8e8, 1.9e8, 3e8, -1.2e8, -1.9e8):
        b = bias.clone()
        b[:] = top
        t8.check_head(x, w, ws, b, ids, 9)
        t8.check_head(x, w * 0, ws, b, ids, 9)
        if top > 0:
            b[:-2] = -top
            t8.check_head(x, w, ws, b, ids, 9)
    for size in (1e6, 4e6, 1e7, 3e7):
        t8.check_head(x, w, ws * size, bias, ids, 9)
    for tau in (2.0 ** -19, 2.0 ** -21, 2.0 ** -23, 2.0 ** -25):
        t8.check_head(x, w, ws, bias, ids, 9, tau)


@pytest.mark.parametrize("P,K", [(64, 900), (256, 9001), (500, 40000), (900, 700), (1100, 300)])
def test_one_workspace_for_batches_of_every_size(gpu_lib, P, K):
    """A workspace of the largest batch serves the smaller ones with the same bits, and no call writes behind its own size."""
    from paper_1907_05701_amd import binding as bd
    most = 150
    x, w, ws, bias, ids = t8.head_case(most, P, K, 2, "bf16")
    kept = torch.empty(bd.int8_logprob_ws_bytes(most, *w.shape), dtype=torch.uint8, device="cuda")
    for M in (most, 1, 16, 17, 32, 33, 64, 65, 129, 2):
        need = bd.int8_logprob_ws_bytes(M, *w.shape)
        own = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        a = t8.head(x[:M], w, ws, bias, ids[:M], 5, buf=own[:need])
        b = t8.head(x[:M], w, ws, bias, ids[:M], 5, buf=kept)
        torch.cuda.synchronize()
        assert all(torch.equal(a[n], b[n]) for n in a), M
        assert bool((own[need:] == 77).all()), M
