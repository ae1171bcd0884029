"""The measured cases of the operators for a causal student of the acoustic
model: its recurrence (a selective state space scan with a short causal
convolution) and its training targets (a teacher's top logits, and the loss
and gradient against them).

A case is a dict of plain values.  ``kind`` says which calls one pass makes:

  conv_frame   the convolution of one frame of every stream, its state updated
  conv_train   the convolution of a batch of chunks, and its backward
  scan_frame   the scan's single step of every stream, its state updated
  scan_prompt  the scan over whole sequences, from a state to a state
  scan_train   the scan over a batch of chunks, and its backward
  top          the top logits of every frame and the log-sum-exp of the others
  distill      loss and logit gradients against a teacher's top logits

``run`` computes them in plain torch operations in 32 bits, or, where ``own``
is set, by the library's calls."""

import math

import torch

own = False


def listed():
    return [
        # one stream's next frame: two words of state a channel, launch latency
        dict(name="conv_frame_b1", kind="conv_frame", B=1, D=1024, W=4, bias=True, precision="bf16"),
        # a training batch of the paper's 128 chunks of 21 frames, both directions' width
        dict(name="conv_train_b128", kind="conv_train", T=21, B=128, D=1024, W=4, bias=True, ragged=False, state=False,
             precision="bf16"),
        # one stream's next frame
        dict(name="scan_frame_b1", kind="scan_frame", B=1, D=1024, N=16, G=1, gate=True, precision="bf16"),
        # a server's 512 streams: the states themselves are most of the bytes
        dict(name="scan_frame_b512", kind="scan_frame", B=512, D=1024, N=16, G=1, gate=True, precision="bf16"),
        # a minute of one recording at 100 frames a second: one row, a long axis
        dict(name="scan_prompt_t6000", kind="scan_prompt", T=6000, B=1, D=1024, N=16, G=1, gate=True, ragged=False,
             state=True, precision="bf16"),
        # the training batch of 128 chunks
        dict(name="scan_train_b128", kind="scan_train", T=21, B=128, D=1024, N=16, G=1, gate=True, ragged=False,
             state=False, precision="bf16"),
        # whole utterances of up to 15 s, padded to the longest
        dict(name="scan_train_t1500", kind="scan_train", T=1500, B=4, D=1024, N=16, G=1, gate=True, ragged=True,
             state=False, precision="bf16"),
        # float32, two groups, no gate, a batch and a length that are no round numbers
        dict(name="scan_train_fp32", kind="scan_train", T=37, B=50, D=640, N=10, G=2, gate=False, ragged=True,
             state=True, precision="fp32"),
        # the teacher's 32 top states of 32000, at the paper's batch
        dict(name="top_b128", kind="top", M=2688, K=32000, k=32, tau=1.0, precision="bf16"),
        # the small float32 model's frames
        dict(name="top_tiny_fp32", kind="top", M=168, K=100, k=8, tau=2.0, precision="fp32"),
        # the student's loss at the paper's batch, mixed with the labels' cross-entropy
        dict(name="distill_b128", kind="distill", M=2688, K=32000, k=32, tau=2.0, soft=0.7, hard=0.3, rest=True,
             masked=False, precision="bf16"),
        # float32, odd sizes, no mass beside the listed classes, some frames masked
        dict(name="distill_ragged_fp32", kind="distill", M=777, K=9001, k=21, tau=1.0, soft=1.0, hard=0.0, rest=False,
             masked=True, precision="fp32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ones' ranges, at most as costly as the largest."""
    kind = rng.choice(["conv_frame", "conv_train", "scan_frame", "scan_prompt", "scan_prompt", "scan_train",
                       "scan_train", "scan_train", "top", "top", "distill", "distill"])
    precision = "bf16" if rng.random() < 0.7 else "fp32"
    if kind in ("top", "distill"):
        K = 32000 if rng.random() < 0.3 else _log_int(rng, 60, 131072)
        M = _log_int(rng, 1, min(20000, (86_000_000 if precision == "bf16" else 43_000_000) // K))
        c = dict(kind=kind, M=M, K=K, k=_log_int(rng, 1, min(128, K // 2)), tau=rng.choice([1.0, 1.0, 2.0, 3.5]))
        if kind == "distill":
            soft = rng.choice([1.0, 0.5, 0.9])
            c.update(soft=soft, hard=rng.choice([0.0, 1.0 - soft, 0.1]), rest=rng.random() < 0.7,
                     masked=rng.random() < 0.5)
        return dict(c, precision=precision)
    G = rng.choice([1, 1, 1, 2, 3])
    D = rng.choice([512, 640, 1024, 1024]) // G * G if rng.random() < 0.6 else G * _log_int(rng, 8, 2048 // G)
    if kind == "conv_frame":
        return dict(kind=kind, B=_log_int(rng, 1, 1024), D=D, W=rng.randint(2, 4), bias=rng.random() < 0.7,
                    precision=precision)
    N = rng.choice([16, 16, 16, 8, 32, rng.randint(1, 24)])
    if kind == "scan_frame":
        B = _log_int(rng, 1, max(1, min(1024, 512 * 1024 * 16 // (D * N))))
        return dict(kind=kind, B=B, D=D, N=N, G=G, gate=rng.random() < 0.7, precision=precision)
    if kind == "conv_train":
        T = _log_int(rng, 1, 4000)
        B = _log_int(rng, 1, max(1, min(1024, 8_000_000 // (T * D))))
        return dict(kind=kind, T=T, B=B, D=D, W=rng.randint(2, 4), bias=rng.random() < 0.7, ragged=rng.random() < 0.4,
                    state=rng.random() < 0.4, precision=precision)
    T = _log_int(rng, 1, 8000 if kind == "scan_prompt" else 2000)
    B = _log_int(rng, 1, max(1, min(1024, 98_000_000 // (T * D * N))))
    T = max(1, min(T, 98_000_000 // (B * D * N)))
    return dict(kind=kind, T=T, B=B, D=D, N=N, G=G, gate=rng.random() < 0.7, ragged=rng.random() < 0.4,
                state=rng.random() < 0.5, precision=precision)


# ------------------------------------------------------------------ inputs ---
def _type(case):
    return torch.bfloat16 if case["precision"] == "bf16" else torch.float32


def _lens(case, g):
    """Lengths of a padded batch: the longest sequence fills it, one may be empty and one a single frame."""
    T, B = case["T"], case["B"]
    n = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    n[0] = T
    n[1:2] = 1 if T > 1 else 0
    n[2:3] = 0
    return n


def _inputs(case, seed):
    """Device tensors made from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 29)
    t = _type(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    kind = case["kind"]
    s = {"case": case}
    if kind in ("top", "distill"):
        M, K, k = case["M"], case["K"], case["k"]
        logits = normal(M, K) * 2
        # distinct classes a frame: an odd step that does not divide K
        step = 2 * torch.randint(0, max(1, K // 2), (M, 1), generator=g, device="cuda") + 1
        step = torch.where(torch.gcd(step, torch.full_like(step, K)) == 1, step, torch.ones_like(step))
        at = torch.randint(0, K, (M, 1), generator=g, device="cuda")
        idx = (at + step * torch.arange(k, device="cuda")) % K
        # a few likely states a frame, as a trained model has them
        top = torch.sort(normal(M, k) * 2 + 8, dim=1, descending=True).values
        logits.scatter_add_(1, idx, top * 0.8 + normal(M, k))
        s["logits"] = logits.to(t)
        if kind == "distill":
            s.update(top=top, idx=idx.to(torch.int32))
            s["rest"] = normal(M) * 0.5 + 6 / case["tau"] if case["rest"] else None
            hit = uniform(M) < 0.8
            other = torch.randint(0, K, (M,), generator=g, device="cuda")
            s["labels"] = torch.where(hit, idx[:, 0], other).to(torch.int32) if case["hard"] else None
            s["weights"] = (uniform(M) < 0.8).float() if case["masked"] else None
        return s
    B, D = case["B"], case["D"]
    T = case.get("T", 1)
    if kind.startswith("conv"):
        W = case["W"]
        # the convolution reads one half of the input projection
        s["x"] = normal(T, B, 2 * D).to(t)[..., :D]
        s["w"] = (uniform(D, W) * 2 - 1) / math.sqrt(W)
        s["bias"] = (uniform(D) * 2 - 1) * 0.1 if case["bias"] else None
        if kind == "conv_frame":
            s["x"] = s["x"][0]
            s["state"] = normal(B, W - 1, D).to(t)
            return s
        s["state"] = normal(B, W - 1, D).to(t) if case["state"] else None
        s["lens"] = _lens(case, g) if case["ragged"] else None
        s["dy"] = normal(T, B, D).to(t)
        return s
    N, G = case["N"], case["G"]
    xz = normal(T, B, 2 * D).to(t)                        # the two halves of the input projection
    bc = normal(T, B, 2 * G * N).to(t)
    s.update(x=xz[..., :D], z=xz[..., D:] if case["gate"] else None, dt=(normal(T, B, D) * 0.5).to(t),
             Bm=bc[..., :G * N], Cm=bc[..., G * N:])
    s["A"] = -torch.exp(torch.log(torch.arange(1, N + 1, device="cuda").float()) + 0.1 * normal(D, N))
    step = torch.exp(uniform(D) * math.log(100.0) + math.log(1e-3))       # 1e-3 .. 1e-1
    s["dt_bias"] = step + torch.log(-torch.expm1(-step))                  # softplus of it is the step
    s["Dskip"] = 1 + 0.1 * normal(D)
    if kind == "scan_frame":
        for name in ("x", "z", "dt", "Bm", "Cm"):
            s[name] = s[name][0] if s[name] is not None else None
        s["state"] = normal(B, D, N)
        return s
    s["h0"] = normal(B, D, N) if case["state"] else None
    s["lens"] = _lens(case, g) if case["ragged"] else None
    if kind == "scan_train":
        s["dy"] = normal(T, B, D).to(t)
    return s


def prepare(case, seed):
    """The inputs and the output buffers that a program keeps between passes."""
    s = _inputs(case, seed)
    t, kind = _type(case), case["kind"]

    def out(*shape, dtype=t):
        return torch.empty(shape, dtype=dtype, device="cuda")

    f32 = torch.float32
    if kind == "top":
        M, k = case["M"], case["k"]
        s["out"] = {"top": out(M, k, dtype=f32), "idx": out(M, k, dtype=torch.int32), "rest": out(M, dtype=f32)}
        return s
    if kind == "distill":
        s["out"] = {"row_loss": out(case["M"], dtype=f32), "dlogits": out(case["M"], case["K"])}
        return s
    B, D = case["B"], case["D"]
    if kind == "conv_frame":
        s["out"] = {"y": out(B, D)}
    elif kind == "conv_train":
        T, W = case["T"], case["W"]
        s["out"] = {"y": out(T, B, D), "state": out(B, W - 1, D), "dx": out(T, B, D), "dw": out(D, W, dtype=f32)}
        if case["bias"]:
            s["out"]["dbias"] = out(D, dtype=f32)
    elif kind == "scan_frame":
        s["out"] = {"y": out(B, D)}
    else:
        T, N, G = case["T"], case["N"], case["G"]
        s["out"] = {"y": out(T, B, D), "h_last": out(B, D, N, dtype=f32)}
        if kind == "scan_train":
            s["out"].update(dx=out(T, B, D), ddt=out(T, B, D), dBm=out(T, B, G * N), dCm=out(T, B, G * N),
                            dA=out(D, N, dtype=f32), dDskip=out(D, dtype=f32), ddt_bias=out(D, dtype=f32))
            if case["gate"]:
                s["out"]["dz"] = out(T, B, D)
            if case["state"]:
                s["out"]["dh0"] = out(B, D, N, dtype=f32)
    return s


# ------------------------------------------------------------- plain forms ---
def _silu(v):
    return v / (1 + torch.exp(-v))


def _dsilu(v):
    p = 1 / (1 + torch.exp(-v))
    return p * (1 + v * (1 - p))


def _softplus(v):
    return torch.where(v > 20, v, torch.log1p(torch.exp(torch.clamp(v, max=20.0))))


def _inside(s, T, B):
    """[T, B, 1] truth values: whether a frame lies within its sequence."""
    at = torch.arange(T, device="cuda").view(T, 1, 1)
    if s["lens"] is None:
        return (at >= 0).expand(T, B, 1)
    return at < s["lens"].view(1, B, 1)


def _plain_conv_frame(s):
    x, w = s["x"].float(), s["w"]
    window = torch.cat((s["state"].float(), x[:, None]), 1)              # [B, W, D]
    pre = (window * w.t()).sum(1)
    if s["bias"] is not None:
        pre = pre + s["bias"]
    s["state"].copy_(window[:, 1:])
    return {"y": _silu(pre).to(s["x"].dtype), "state": s["state"]}


def _plain_conv_train(s):
    c, t = s["case"], s["x"].dtype
    T, B, D, W = (c[k] for k in ("T", "B", "D", "W"))
    inside = _inside(s, T, B)
    x = torch.where(inside, s["x"].float(), 0.0)
    first = torch.zeros(W - 1, B, D, device="cuda") if s["state"] is None else s["state"].float().transpose(0, 1)
    xs = torch.cat((first, x))                                           # [T + W - 1, B, D]
    at = torch.arange(T, device="cuda").view(T, 1) + torch.arange(W, device="cuda")
    windows = xs[at]                                                     # [T, W, B, D]
    pre = (windows * s["w"].t()[None, :, None]).sum(1)
    if s["bias"] is not None:
        pre = pre + s["bias"]
    y = torch.where(inside, _silu(pre), 0.0)
    n = torch.full((B,), T, device="cuda") if s["lens"] is None else s["lens"].long()
    last = n.view(B, 1) + torch.arange(W - 1, device="cuda")             # the last W - 1 inputs of each sequence
    state = xs[last, torch.arange(B, device="cuda").view(B, 1)]
    dpre = torch.where(inside, s["dy"].float() * _dsilu(pre), 0.0)
    dp = torch.cat((dpre, torch.zeros(W - 1, B, D, device="cuda")))
    dx = torch.where(inside, (dp[at] * s["w"].flip(1).t()[None, :, None]).sum(1), 0.0)
    dw = (dpre[:, None] * windows).sum((0, 2)).t()
    out = {"y": y.to(t), "state": state.to(t), "dx": dx.to(t), "dw": dw}
    if s["bias"] is not None:
        out["dbias"] = dpre.sum((0, 1))
    return out


def _recur(a, b):
    """h[t] = a[t] h[t-1] + b[t] along the first axis, in log2 T steps that each join spans twice as long."""
    n = 1
    while n < a.shape[0]:
        b = torch.cat((b[:n], b[n:] + a[n:] * b[:-n]))
        a = torch.cat((a[:n], a[n:] * a[:-n]))
        n *= 2
    return b


def _plain_scan_frame(s):
    c, t = s["case"], s["x"].dtype
    B, D, N, G = (c[k] for k in ("B", "D", "N", "G"))
    x, d = s["x"].float(), _softplus(s["dt"].float() + s["dt_bias"])
    Bm = s["Bm"].float().view(B, G, 1, N).expand(B, G, D // G, N).reshape(B, D, N)
    Cm = s["Cm"].float().view(B, G, 1, N).expand(B, G, D // G, N).reshape(B, D, N)
    s["state"].copy_(torch.exp(d[..., None] * s["A"]) * s["state"] + (d * x)[..., None] * Bm)
    o = (s["state"] * Cm).sum(-1) + s["Dskip"] * x
    if s["z"] is not None:
        o = o * _silu(s["z"].float())
    return {"y": o.to(t), "state": s["state"]}


def _plain_scan(s, train):
    c, t = s["case"], s["x"].dtype
    T, B, D, N, G = (c[k] for k in ("T", "B", "D", "N", "G"))
    inside = _inside(s, T, B)
    x, v = s["x"].float(), s["dt"].float() + s["dt_bias"]
    d = torch.where(inside, _softplus(v), 0.0)                           # behind the end the state stays
    Bm = s["Bm"].float().view(T, B, G, 1, N).expand(T, B, G, D // G, N).reshape(T, B, D, N)
    Cm = s["Cm"].float().view(T, B, G, 1, N).expand(T, B, G, D // G, N).reshape(T, B, D, N)
    a = torch.exp(d[..., None] * s["A"])
    b = (d * x)[..., None] * Bm
    h0 = torch.zeros(B, D, N, device="cuda") if s["h0"] is None else s["h0"]
    b[0] += a[0] * h0
    h = _recur(a, b)
    o = (h * Cm).sum(-1) + s["Dskip"] * x
    z = s["z"].float() if s["z"] is not None else None
    y = o * _silu(z) if z is not None else o
    out = {"y": torch.where(inside, y, 0.0).to(t), "h_last": h[-1].clone()}
    if not train:
        return out
    dy = torch.where(inside, s["dy"].float(), 0.0)
    g = dy * _silu(z) if z is not None else dy
    later = torch.cat((a[1:], torch.zeros_like(a[:1]))).flip(0)
    dh = _recur(later, (g[..., None] * Cm).flip(0)).flip(0)
    q = dh * a * torch.cat((h0[None], h[:-1]))
    db = (dh * Bm).sum(-1)
    dd = x * db + (q * s["A"]).sum(-1)
    ddt = torch.where(inside, dd / (1 + torch.exp(-v)), 0.0)
    per = (T, B, G, D // G, N)
    out.update(dx=torch.where(inside, d * db + s["Dskip"] * g, 0.0).to(t), ddt=ddt.to(t),
               dBm=(dh * (d * x)[..., None]).view(per).sum(3).reshape(T, B, G * N).to(t),
               dCm=torch.where(inside, (h * g[..., None]).view(per).sum(3).reshape(T, B, G * N), 0.0).to(t),
               dA=(q * d[..., None]).sum((0, 1)), dDskip=(g * x).sum((0, 1)), ddt_bias=ddt.sum((0, 1)))
    if z is not None:
        out["dz"] = torch.where(inside, dy * o * _dsilu(z), 0.0).to(t)
    if s["h0"] is not None:
        out["dh0"] = a[0] * dh[0]
    return out


def _plain_top(s):
    c = s["case"]
    f = s["logits"].float()
    v, i = torch.sort(f, dim=1, descending=True, stable=True)            # equal logits: the lower class first
    k = c["k"]
    u = v[:, k:] / c["tau"]
    m = u[:, :1]
    rest = m[:, 0] + torch.log(torch.exp(u - m).sum(1))
    return {"top": v[:, :k].contiguous(), "idx": i[:, :k].to(torch.int32), "rest": rest}


def _plain_distill(s):
    c = s["case"]
    M, K, tau, soft, hard = (c[k] for k in ("M", "K", "tau", "soft", "hard"))
    f, idx = s["logits"].float(), s["idx"].long()
    w = torch.ones(M, device="cuda") if s["weights"] is None else s["weights"]
    # the teacher's probabilities of its listed classes, and of all the others together
    v = s["top"] / tau
    if s["rest"] is not None:
        v = torch.cat((v, s["rest"][:, None]), 1)
    e = torch.exp(v - v.max(1, keepdim=True).values)
    lp = torch.log(e / e.sum(1, keepdim=True))
    # the student's: of every class, and of the same buckets
    u = f / tau
    m = u.max(1, keepdim=True).values
    e = torch.exp(u - m)
    z = e.sum(1, keepdim=True)
    listed_u = torch.gather(u, 1, idx)
    lq = listed_u - m - torch.log(z)
    q = e / z
    dense = q
    if s["rest"] is not None:
        others = e.scatter(1, idx, 0.0)
        zr = others.sum(1, keepdim=True)
        lq = torch.cat((lq, torch.log(zr / z)), 1)
        dense = q - others * (torch.exp(lp[:, -1:]) / zr)
    p = torch.exp(lp)
    kl = (p * (lp - lq)).sum(1)
    dense = dense.scatter_add(1, idx, -p[:, :c["k"]])
    loss, grad = soft * tau * tau * kl, (soft * tau) * dense
    if s["labels"] is not None:
        lab = s["labels"].long()[:, None]
        m = f.max(1, keepdim=True).values
        e = torch.exp(f - m)
        z = e.sum(1, keepdim=True)
        loss = loss + hard * (m + torch.log(z) - torch.gather(f, 1, lab))[:, 0]
        grad = grad + hard * (e / z).scatter_add(1, lab, -torch.ones_like(z))
    return {"row_loss": w * loss, "dlogits": (grad * (w / M)[:, None]).to(s["logits"].dtype)}


# ------------------------------------------------------ the library's calls ---
def _ssm(s, bd):
    """The dims and workspaces that a program keeps, made on the first pass."""
    if "dims" not in s:
        c = s["case"]
        s["dims"] = bd.make_ssm_dims(T=c.get("T", 1), B=c["B"], D=c["D"], N=c.get("N", 1), G=c.get("G", 1),
                                     W=c.get("W", 1), precision=c["precision"])
        s["ws"] = {name: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
                   for name, n in bd.ssm_workspace_bytes(s["dims"]).items()}
    return s["dims"], s["ws"]


def _own(s):
    from paper_1907_05701_amd import binding as bd
    c, o = s["case"], s["out"]
    kind = c["kind"]
    if kind == "top":
        bd.softmax_topk_rows(s["logits"], o["top"], o["idx"], o["rest"], temperature=c["tau"])
        return o
    if kind == "distill":
        bd.softmax_distill_rows(s["logits"], s["top"], s["idx"], o["row_loss"], o["dlogits"], rest=s["rest"],
                                labels=s["labels"], weights=s["weights"], temperature=c["tau"], soft=c["soft"],
                                hard=c["hard"], loss_scale=1.0 / c["M"])
        return o
    dims, ws = _ssm(s, bd)
    if kind == "conv_frame":
        bd.ssm_conv_step(dims, s["x"], s["w"], s["bias"], s["state"], o["y"])
        return {"y": o["y"], "state": s["state"]}
    if kind == "conv_train":
        bd.ssm_conv_fwd(dims, s["x"], s["w"], s["bias"], o["y"], lens=s["lens"], state=s["state"], state_out=o["state"])
        bd.ssm_conv_bwd(dims, s["x"], s["w"], s["bias"], s["dy"], o["dx"], o["dw"], o.get("dbias"), ws["conv_bwd"],
                        lens=s["lens"], state=s["state"])
        return o
    if kind == "scan_frame":
        bd.ssm_scan_step(dims, s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["state"], o["y"], Dskip=s["Dskip"],
                         z=s["z"], dt_bias=s["dt_bias"])
        return {"y": o["y"], "state": s["state"]}
    train = kind == "scan_train"
    bd.ssm_scan_fwd(dims, s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], o["y"], ws["fwd"], Dskip=s["Dskip"], z=s["z"],
                    dt_bias=s["dt_bias"], h0=s["h0"], h_last=o["h_last"], lens=s["lens"],
                    saved=ws["saved"] if train else None)
    if train:
        bd.ssm_scan_bwd(dims, s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["dy"], ws["saved"], ws["bwd"], o["dx"],
                        o["ddt"], o["dA"], o["dBm"], o["dCm"], Dskip=s["Dskip"], dDskip=o["dDskip"], z=s["z"],
                        dz=o.get("dz"), dt_bias=s["dt_bias"], ddt_bias=o["ddt_bias"], dh0=o.get("dh0"),
                        lens=s["lens"])
    return o


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    if kind == "conv_frame":
        return _plain_conv_frame(s)
    if kind == "conv_train":
        return _plain_conv_train(s)
    if kind == "scan_frame":
        return _plain_scan_frame(s)
    if kind == "top":
        return _plain_top(s)
    if kind == "distill":
        return _plain_distill(s)
    return _plain_scan(s, kind == "scan_train")


# ------------------------------------------------------------------- work ----
def work(case):
    es, kind = 2 if case["precision"] == "bf16" else 4, case["kind"]
    if kind in ("top", "distill"):
        M, K, k = case["M"], case["K"], case["k"]
        if kind == "top":   # a comparison, and a difference, an exponential and a sum
            return {"bytes": M * K * es + M * (8 * k + 4), "flops": 4 * M * K}
        n = M * (8 * k + 4 + 4 * case["rest"] + 4 * (case["hard"] > 0) + 4 * case["masked"])
        return {"bytes": 2 * M * K * es + n, "flops": (6 + 5 * (case["hard"] > 0)) * M * K}
    B, D = case["B"], case["D"]
    T = case.get("T", 1)
    M = T * B
    lens = 4 * B if case.get("ragged") else 0
    if kind.startswith("conv"):
        W, par = case["W"], D * (case["W"] + case["bias"])
        st = B * (W - 1) * D * es
        if kind == "conv_frame":
            return {"bytes": 2 * M * D * es + 2 * st + 4 * par, "flops": M * D * (2 * W + 4)}
        # x is read and y written; x and dy are read and dx written
        return {"bytes": 5 * M * D * es + st * (1 + 2 * case["state"]) + 4 * par * 3 + 2 * lens,
                "flops": M * D * (8 * W + 14)}
    N, G = case["N"], case["G"]
    par = 4 * D * (N + 2)
    io = (3 + case["gate"]) * M * D * es + 2 * M * G * N * es
    st = 4 * B * D * N
    per = M * D * N
    if kind == "scan_frame":
        return {"bytes": io + par + 2 * st, "flops": 7 * per + 10 * M * D}
    fwd = {"bytes": io + par + st * (1 + case["state"]) + lens, "flops": 7 * per + 10 * M * D}
    if kind == "scan_prompt":
        return fwd
    # back: x, dt, dy, B, C (and z) are read, their gradients written
    back = (5 + 2 * case["gate"]) * M * D * es + 4 * M * G * N * es + 2 * par + 2 * st * case["state"] + lens
    return {"bytes": fwd["bytes"] + back, "flops": fwd["flops"] + 18 * per + 25 * M * D}


# ----------------------------------------------------------- in 64 bits ------
def _double(s):
    return {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}


def _exact_conv(s, c):
    """The convolution and its gradients, one tap and one frame's window at a time."""
    T, B, D, W = c.get("T", 1), c["B"], c["D"], c["W"]
    frame = c["kind"] == "conv_frame"
    x = s["x"][None] if frame else s["x"]
    lens = None if frame else s["lens"]
    n = torch.full((B,), T, device="cuda") if lens is None else lens.long()
    live = (torch.arange(T, device="cuda")[:, None] < n)[..., None].double()
    x = x * live
    past = x.new_zeros(W - 1, B, D) if s["state"] is None else s["state"].transpose(0, 1)
    xs = torch.cat((past, x), 0)
    bias = 0.0 if s["bias"] is None else s["bias"]
    pre = x.new_zeros(T, B, D) + bias
    for j in range(W):
        pre += xs[j:j + T] * s["w"][:, j]
    sig = torch.sigmoid(pre)
    state = torch.stack([xs[n + j, torch.arange(B, device="cuda")] for j in range(W - 1)], 1)
    if frame:
        return {"y": (pre * sig)[0], "state": state}
    dpre = s["dy"] * (sig + pre * sig * (1 - sig)) * live
    dxs = torch.zeros_like(xs)
    dw = torch.zeros_like(s["w"])
    for j in range(W):
        dxs[j:j + T] += dpre * s["w"][:, j]
        dw[:, j] = (dpre * xs[j:j + T]).sum((0, 1))
    out = {"y": pre * sig * live, "state": state, "dx": dxs[W - 1:] * live, "dw": dw}
    if s["bias"] is not None:
        out["dbias"] = dpre.sum((0, 1))
    return out


def _exact_scan(s, c):
    """The scan frame by frame, and its adjoint frame by frame from the end."""
    B, D, N, G = (c[k] for k in ("B", "D", "N", "G"))
    T = c.get("T", 1)
    frame, train = c["kind"] == "scan_frame", c["kind"] == "scan_train"
    if frame:
        s = dict(s, h0=s["state"], lens=None)
        for name in ("x", "z", "dt", "Bm", "Cm"):
            s[name] = s[name][None] if s[name] is not None else None
    x = s["x"]
    v = s["dt"] + s["dt_bias"]
    d = torch.logaddexp(v, torch.zeros_like(v))
    n = torch.full((B,), T, device="cuda") if s["lens"] is None else s["lens"].long()
    live = (torch.arange(T, device="cuda")[:, None] < n)[..., None]      # [T, B, 1]

    def wide(v):   # a group's values for each of its channels
        return v.reshape(B, G, N).repeat_interleave(D // G, 1)

    h = x.new_zeros(B, D, N) if s["h0"] is None else s["h0"].clone()
    o, hs = torch.empty_like(x), []
    for t in range(T):
        if train:
            hs.append(h)
        new = torch.exp(d[t][..., None] * s["A"]) * h + (d[t] * x[t])[..., None] * wide(s["Bm"][t])
        h = torch.where(live[t][..., None], new, h)
        o[t] = (h * wide(s["Cm"][t])).sum(-1)
    o = o + s["Dskip"] * x
    if s["z"] is not None:
        sig = torch.sigmoid(s["z"])
        gate, slope = s["z"] * sig, sig * (1 + s["z"] * (1 - sig))
        y = o * gate
    else:
        gate, y = torch.ones_like(o), o
    y = torch.where(live, y, torch.zeros_like(y))
    if frame:
        return {"y": y[0], "state": h}
    out = {"y": y, "h_last": h}
    if not train:
        return out
    zero = x.new_zeros(())
    g = torch.where(live, s["dy"] * gate, zero)
    dx, ddt = torch.empty_like(x), torch.empty_like(x)
    dB, dC = x.new_empty(T, B, G * N), x.new_empty(T, B, G * N)
    dA, dh = torch.zeros_like(s["A"]), x.new_zeros(B, D, N)
    hn = h
    for t in range(T - 1, -1, -1):
        Bt = wide(s["Bm"][t])
        dh = dh + g[t][..., None] * wide(s["Cm"][t])
        a = torch.exp(d[t][..., None] * s["A"])
        into, q = (dh * Bt).sum(-1), dh * a * hs[t]
        dx[t] = d[t] * into + s["Dskip"] * g[t]
        ddt[t] = (x[t] * into + (q * s["A"]).sum(-1)) * torch.sigmoid(v[t])
        on = live[t][..., None]
        dA += torch.where(on, q * d[t][..., None], zero).sum(0)
        dB[t] = torch.where(on, dh * (d[t] * x[t])[..., None], zero).reshape(B, G, D // G, N).sum(2).reshape(B, G * N)
        dC[t] = (hn * g[t][..., None]).reshape(B, G, D // G, N).sum(2).reshape(B, G * N)
        dh = torch.where(on, a * dh, dh)
        hn = hs[t]
    dx, ddt = torch.where(live, dx, zero), torch.where(live, ddt, zero)
    out.update(dx=dx, ddt=ddt, dBm=dB, dCm=dC, dA=dA, dDskip=(g * x).sum((0, 1)), ddt_bias=ddt.sum((0, 1)))
    if s["z"] is not None:
        out["dz"] = torch.where(live, s["dy"] * o * slope, zero)
    if s["h0"] is not None:
        out["dh0"] = dh
    return out


def _exact_top(s, c):
    f, k = s["logits"], c["k"]
    # the class's place breaks ties: ranks of (-logit, class)
    order = torch.argsort(-f, dim=1, stable=True)
    idx = order[:, :k]
    rest = torch.logsumexp(f.scatter(1, idx, -math.inf) / c["tau"], 1)
    return {"top": torch.gather(f, 1, idx), "idx": idx.to(torch.int32), "rest": rest}


def _exact_distill(s, c):
    f, tau = s["logits"], c["tau"]
    M, K = f.shape
    idx = s["idx"].long()
    rest = torch.full((M, 1), -math.inf, dtype=f.dtype, device=f.device) if s["rest"] is None else s["rest"][:, None]
    p = torch.softmax(torch.cat((s["top"] / tau, rest), 1), 1)
    r, p = p[:, -1:], p[:, :-1]
    q = torch.softmax(f / tau, 1)
    target = torch.zeros_like(f).scatter_(1, idx, p)
    at = torch.zeros_like(f).scatter_(1, idx, 1.0)
    qr = (q * (1 - at)).sum(1, keepdim=True)
    kl = torch.xlogy(p, p).sum(1) - (p * torch.log(torch.gather(q, 1, idx))).sum(1)
    kl = kl + (torch.xlogy(r, r) - torch.xlogy(r, qr))[:, 0]
    ds = q - target - (1 - at) * q * (r / qr)
    loss, ds = c["soft"] * tau ** 2 * kl, c["soft"] * tau * ds
    if s["labels"] is not None:
        ls = torch.log_softmax(f, 1)
        hot = torch.zeros_like(f).scatter_(1, s["labels"].long()[:, None], 1.0)
        loss = loss - c["hard"] * (ls * hot).sum(1)
        ds = ds + c["hard"] * (torch.exp(ls) - hot)
    w = torch.ones(M, dtype=f.dtype, device=f.device) if s["weights"] is None else s["weights"]
    return {"row_loss": w * loss, "dlogits": ds * (w / M)[:, None]}


def exact(case, seed):
    s = _double(_inputs(case, seed))
    kind = case["kind"]
    if kind == "top":
        return _exact_top(s, case)
    if kind == "distill":
        return _exact_distill(s, case)
    return _exact_conv(s, case) if kind.startswith("conv") else _exact_scan(s, case)
