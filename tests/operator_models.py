"""Plain float64 forms (torch, CPU, one frame after the other) of the state
space operators and of distillation, the gradients by autograd, and the
measure that the GPU tests compare with."""

import torch


def softplus(v):
    return torch.logaddexp(v, torch.zeros_like(v))


def silu(v):
    return v * torch.sigmoid(v)


def lengths(lens, T, B):
    return [T] * B if lens is None else [min(T, max(0, int(n))) for n in lens]


def conv(x, w, bias, state=None, lens=None, act=True):
    """(y [T, B, D], the last W - 1 inputs of each sequence [B, W - 1, D])."""
    T, B, D = x.shape
    W = w.shape[1]
    ys, ends = [], []
    for b, n in enumerate(lengths(lens, T, B)):
        past = torch.zeros(W - 1, D, dtype=x.dtype) if state is None else state[b]
        seq = torch.cat((past, x[:n, b]))
        rows = []
        for t in range(n):
            pre = (seq[t:t + W] * w.t()).sum(0) + (0 if bias is None else bias)
            rows.append(silu(pre) if act else pre)
        rows += [torch.zeros(D, dtype=x.dtype)] * (T - n)
        ys.append(torch.stack(rows))
        ends.append(seq[n:])
    return torch.stack(ys, 1), torch.stack(ends)


def scan(x, dt, A, Bm, Cm, Dskip=None, z=None, dt_bias=None, h0=None, lens=None, softplus_on=True):
    """(y [T, B, D], the state behind each sequence [B, D, N])."""
    T, B, D = x.shape
    N = A.shape[1]
    G = Bm.shape[2] // N
    ys, ends = [], []
    for b, n in enumerate(lengths(lens, T, B)):
        h = torch.zeros(D, N, dtype=x.dtype) if h0 is None else h0[b]
        rows = []
        for t in range(n):
            s = dt[t, b] if dt_bias is None else dt[t, b] + dt_bias
            s = softplus(s) if softplus_on else s
            Bv = Bm[t, b].view(G, N).repeat_interleave(D // G, 0)
            Cv = Cm[t, b].view(G, N).repeat_interleave(D // G, 0)
            h = torch.exp(s[:, None] * A) * h + (s * x[t, b])[:, None] * Bv
            o = (h * Cv).sum(1)
            if Dskip is not None:
                o = o + Dskip * x[t, b]
            rows.append(o if z is None else o * silu(z[t, b]))
        rows += [torch.zeros(D, dtype=x.dtype)] * (T - n)
        ys.append(torch.stack(rows))
        ends.append(h)
    return torch.stack(ys, 1), torch.stack(ends)


def topk(logits, k, tau):
    """Descending, the lower class first among equals, a NaN above all."""
    f = logits.double()
    order = sorted(range(f.shape[0]), key=lambda c: (0 if torch.isnan(f[c]) else 1, -float(f[c]) if f[c] == f[c] else 0, c))
    at = torch.tensor(order[:k])
    others = torch.tensor(order[k:], dtype=torch.long)
    rest = torch.logsumexp(f[others] / tau, 0) if len(others) else torch.tensor(-torch.inf, dtype=torch.float64)
    return f[at], at, rest


def distill_row(s, top, idx, rest, label, tau, soft, hard):
    """Loss of one row; s requires grad where its gradient is wanted.  The others
    are one bucket; a class listed twice has both probabilities."""
    K = s.shape[0]
    ok = [i for i, c in enumerate(idx) if 0 <= c < K]
    loss = s.new_zeros(())
    v = torch.cat((top[ok] / tau, rest.view(1)))
    if soft and not torch.isneginf(v.max()):   # a loss that is not asked for may be infinite
        p = torch.softmax(v, 0)
        lq = torch.log_softmax(s / tau, 0)
        per = {}
        for i, c in enumerate(ok):
            per[int(idx[c])] = per.get(int(idx[c]), 0) + p[i]
        kl = s.new_zeros(())
        for c, pc in per.items():
            if pc > 0:
                kl = kl + pc * (torch.log(pc) - lq[c])
        if p[-1] > 0:
            others = torch.tensor([c for c in range(K) if c not in per], dtype=torch.long)
            kl = kl + p[-1] * (torch.log(p[-1]) - torch.logsumexp(lq[others], 0))
        loss = loss + soft * tau * tau * kl
    if 0 <= label < K and hard:
        loss = loss - hard * torch.log_softmax(s, 0)[label]
    return loss


def half_step(dtype):
    """Half a step of rounding, relative to the value."""
    return torch.finfo(dtype).eps / 2


def far(got, want, tol):
    """How many times |got - want| is over its bound: half a step of got's type at
    the value, and `tol` of the values' root mean square beside it (sums over
    many terms are as exact as their terms' size, not as their own)."""
    g, w = got.detach().double().cpu(), want.detach().double()
    assert g.shape == w.shape, (g.shape, w.shape)
    assert torch.equal(torch.isfinite(g), torch.isfinite(w))
    fine = torch.isfinite(w)
    if not fine.any():
        return 0.0
    g, w = g[fine], w[fine]
    rms = float(w.square().mean().sqrt())
    bound = half_step(got.dtype) * w.abs() + tol * (w.abs() + rms) + 1e-30
    return float(((g - w).abs() / bound).max())
