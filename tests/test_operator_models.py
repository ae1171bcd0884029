"""CPU: the float64 forms that the GPU tests compare with, against central
differences and against what they have to be in closed form."""

import math

import pytest
import torch

import operator_models as om

torch.manual_seed(0)


def _rand(*shape):
    return torch.randn(shape, dtype=torch.float64)


def _check_differences(f, args, seed):
    """d f / d (a direction in all arguments): autograd against a central difference."""
    g = torch.Generator().manual_seed(seed)
    leaves = [a.clone().requires_grad_() for a in args]
    grads = torch.autograd.grad(f(*leaves), leaves)
    way = [torch.randn(a.shape, generator=g, dtype=torch.float64) for a in args]
    e = 1e-5
    up = f(*[a + e * w for a, w in zip(args, way)])
    down = f(*[a - e * w for a, w in zip(args, way)])
    want = float((up - down) / (2 * e))
    got = float(sum((a * w).sum() for a, w in zip(grads, way)))
    assert abs(got - want) <= 1e-7 * max(1.0, abs(want))


def test_scan_gradients_against_differences():
    T, B, D, N, G = 6, 2, 4, 3, 2
    args = [_rand(T, B, D), _rand(T, B, D), -torch.rand(D, N, dtype=torch.float64), _rand(T, B, G * N),
            _rand(T, B, G * N), _rand(D), _rand(T, B, D), _rand(D), _rand(B, D, N)]
    c, e = _rand(T, B, D), _rand(B, D, N)

    def f(*a):
        y, h = om.scan(*a, lens=[6, 3])
        return (y * c).sum() + (h * e).sum()

    _check_differences(f, args, 1)


def test_scan_of_constant_inputs_is_a_geometric_series():
    T, s, A = 9, 0.3, -0.7
    one = torch.ones(T, 1, 1, dtype=torch.float64)
    y, h = om.scan(one, one * s, torch.full((1, 1), A, dtype=torch.float64), one, one, softplus_on=False)
    a = math.exp(s * A)
    want = [s * (1 - a ** (t + 1)) / (1 - a) for t in range(T)]
    assert torch.allclose(y[:, 0, 0], torch.tensor(want, dtype=torch.float64), atol=1e-14)
    assert abs(float(h) - want[-1]) < 1e-14


def test_conv_gradients_against_differences_and_torch():
    T, B, D, W = 7, 3, 4, 4
    args = [_rand(T, B, D), _rand(D, W), _rand(D), _rand(B, W - 1, D)]
    c, e = _rand(T, B, D), _rand(B, W - 1, D)

    def f(*a):
        y, s = om.conv(*a, lens=[7, 2, 0])
        return (y * c).sum() + (s * e).sum()

    _check_differences(f, args, 2)
    y, _ = om.conv(args[0], args[1], args[2], act=False)
    x = torch.nn.functional.pad(args[0].permute(1, 2, 0), (W - 1, 0))
    want = torch.nn.functional.conv1d(x, args[1][:, None], args[2], groups=D).permute(2, 0, 1)
    assert torch.allclose(y, want, atol=1e-13)


def test_distill_gradient_against_differences():
    K = 9
    top, idx, rest = _rand(4), torch.tensor([3, 7, 3, -1]), _rand(1)[0]
    _check_differences(lambda s: om.distill_row(s, top, idx, rest, 5, 1.7, 0.8, 0.4), [_rand(K)], 3)


def test_distill_of_every_class_is_the_divergence():
    K = 11
    s, t = _rand(K), _rand(K)
    got = om.distill_row(s, t, torch.arange(K), torch.tensor(-math.inf, dtype=torch.float64), -1, 2.0, 1.0, 0.0)
    p = torch.softmax(t / 2, 0)
    want = 4 * (p * (torch.log(p) - torch.log_softmax(s / 2, 0))).sum()
    assert abs(float(got - want)) < 1e-13


def test_distill_from_itself_is_zero_with_zero_gradient():
    K, k, tau = 20, 5, 1.5
    s = _rand(K).requires_grad_()
    top, at, rest = om.topk(s.detach(), k, tau)
    loss = om.distill_row(s, top, at, rest, -1, tau, 1.0, 0.0)
    (g,) = torch.autograd.grad(loss, s)
    assert abs(float(loss.detach())) < 1e-14 and float(g.abs().max()) < 1e-14


@pytest.mark.parametrize("k", [1, 3, 6])
def test_topk_orders_ties_by_class(k):
    s = torch.tensor([1.0, 3.0, 3.0, -0.0, 0.0, float("nan")], dtype=torch.float64)
    v, at, rest = om.topk(s, k, 1.0)
    assert at.tolist() == [5, 1, 2, 0, 3, 4][:k]
    if k == 6:
        assert float(rest) == -math.inf
