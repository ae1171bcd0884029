"""Plain float64 forms (torch, CPU, one row after the other) of the scoring
operators and exact ones of the 8-bit products."""

from fractions import Fraction

import numpy as np
import torch


def log_probs(s, tau):
    """Log probabilities of a row of logits: all -inf where no class is above that, NaN where one is NaN or +inf."""
    if bool(torch.isnan(s).any()) or bool(torch.isposinf(s).any()):
        return torch.full_like(s, torch.nan)
    if bool(torch.isneginf(s).all()):
        return s.clone()
    return torch.log_softmax(s / tau, 0)


def entropy(s, tau):
    lp = log_probs(s, tau)
    if bool(torch.isnan(lp).any()):
        return s.new_tensor(torch.nan)
    keep = lp > -torch.inf
    return -(torch.exp(lp[keep]) * lp[keep]).sum()


def listed(lp, ids):
    """The listed classes' log probabilities, 0 for an id that is no class."""
    ok = (ids >= 0) & (ids < lp.shape[0])
    return torch.where(ok, lp[torch.where(ok, ids, 0).long()], lp.new_zeros(()))


def order(s):
    """Classes by descending logit, the lower class first among equals, a NaN above all."""
    f = s.double()
    return torch.tensor(sorted(range(f.shape[0]),
                               key=lambda c: (0 if torch.isnan(f[c]) else 1, -float(f[c]) if f[c] == f[c] else 0, c)))


def loss(s, ids, g, h, tau):
    """What the gradients g of the listed log probabilities and h of the entropy belong to."""
    lp = torch.log_softmax(s / tau, 0)
    ok = (ids >= 0) & (ids < s.shape[0])
    e = -(torch.exp(lp) * torch.where(lp > -torch.inf, lp, 0.0)).sum()
    return (g[ok] * lp[ids[ok].long()]).sum() + h * e


def gradient(s, ids, g, h, tau):
    """(d loss / d s by the formula, the size of the terms that add up to it)."""
    lp = log_probs(s, tau)
    ok = (ids >= 0) & (ids < s.shape[0])
    own, size = torch.zeros_like(s), torch.zeros_like(s)
    own.scatter_add_(0, ids[ok].long(), g[ok])
    size.scatter_add_(0, ids[ok].long(), g[ok].abs())
    if not bool((g[ok] != 0).any()) and float(h) == 0.0 or bool(torch.isneginf(s).all()):
        return torch.zeros_like(s), torch.zeros_like(s)
    p, H = torch.exp(lp), entropy(s, tau)
    ev = torch.where(lp > -torch.inf, lp, 0.0)
    d = own - p * (g[ok].sum() + h * (ev + H))
    return d / tau, (size + p * (g[ok].abs().sum() + abs(h) * (ev.abs() + H))) / tau


def quantize(x):
    """(integers, scales) of rows of numbers: the nearest integer to 127 x / max |x| in exact arithmetic, ties to
    the even one.  Rows with a NaN or an infinite value: zeros and a NaN."""
    x = np.asarray(x, dtype=np.float32)
    q = np.zeros(x.shape, dtype=np.int8)
    scale = np.zeros(x.shape[0], dtype=np.float32)
    for m, row in enumerate(x):
        if not np.isfinite(row).all():
            scale[m] = np.nan
            continue
        top = np.abs(row).max() if row.size else np.float32(0)
        scale[m] = top / np.float32(127)
        if top > 0:
            q[m] = [round(Fraction(float(v)) * 127 / Fraction(float(top))) for v in row]   # round() goes to the even one
    return q, scale


def linear(q, x_scale, w, w_scale, bias=None):
    """float32 results, every step rounded as the operator says."""
    s = q.astype(np.int64) @ w.astype(np.int64).T
    with np.errstate(all="ignore"):
        y = s.astype(np.float32) * (x_scale[:, None] * w_scale[None, :])
        return y if bias is None else y + bias[None, :]
