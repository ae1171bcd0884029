"""CPU: the float64 forms that the GPU tests of scoring compare with, against
central differences and closed forms."""

import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import score_models as sm


@pytest.mark.parametrize("tau", [1.0, 0.5, 3.0])
def test_gradient_against_differences(tau):
    g = torch.Generator().manual_seed(3)
    s = torch.randn(17, generator=g, dtype=torch.float64) * 2
    ids = torch.tensor([4, 4, -1, 9, 40])            # a class twice, two that are no class
    w = torch.randn(5, generator=g, dtype=torch.float64)
    for h in (0.0, 0.7):
        got, size = sm.gradient(s, ids, w, h, tau)
        e = 1e-6
        for j in range(17):
            d = torch.zeros_like(s)
            d[j] = e
            want = float((sm.loss(s + d, ids, w, h, tau) - sm.loss(s - d, ids, w, h, tau)) / (2 * e))
            assert abs(float(got[j]) - want) <= 1e-8
        leaf = s.clone().requires_grad_()
        auto, = torch.autograd.grad(sm.loss(leaf, ids, w, h, tau), leaf)
        assert bool(((got - auto).abs() <= 1e-13 * (1 + size)).all())


def test_closed_forms():
    s = torch.zeros(8, dtype=torch.float64)
    assert math.isclose(float(sm.entropy(s, 2.0)), math.log(8)) and math.isclose(float(sm.log_probs(s, 1.0)[3]), -math.log(8))
    s[3:] = -math.inf
    assert math.isclose(float(sm.entropy(s, 1.0)), math.log(3)) and float(sm.log_probs(s, 1.0)[5]) == -math.inf
    none = torch.full((4,), -math.inf, dtype=torch.float64)
    assert float(sm.entropy(none, 1.0)) == 0.0 and bool(torch.isneginf(sm.log_probs(none, 1.0)).all())
    assert sm.order(torch.tensor([1.0, math.nan, 1.0, 2.0])).tolist() == [1, 3, 0, 2]
    assert float(sm.gradient(none, torch.tensor([1]), torch.ones(1, dtype=torch.float64), 0.5, 1.0)[0].abs().sum()) == 0.0


def test_integers_are_the_nearest():
    x = np.random.default_rng(0).normal(size=(6, 40)).astype(np.float32)
    x[2] = 0
    x[3, 7] = np.inf
    x[4] = np.arange(40) * 0.5       # 127 / 19.5 of a half: near and on borders
    x[5, 0], x[5, 1:] = 127.0, np.arange(39) + 0.5   # ties
    q, scale = sm.quantize(x)
    assert (q[2] == 0).all() and scale[2] == 0 and (q[3] == 0).all() and np.isnan(scale[3])
    assert q[5, 1:5].tolist() == [0, 2, 2, 4]
    for m in (0, 1, 4, 5):
        top = Fraction(float(np.abs(x[m]).max()))
        for v, k in zip(x[m], q[m]):
            assert abs(Fraction(float(v)) * 127 / top - int(k)) <= Fraction(1, 2)
    y = sm.linear(q[:2], scale[:2], q[:2], scale[:2])
    assert np.allclose(y, x[:2] @ x[:2].T, atol=0.2)
