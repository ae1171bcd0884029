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
