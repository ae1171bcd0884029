"""The measured cases of the operators that score frames: log probabilities of
given states with entropy and the most likely alternatives (with gradients, for
sequence training), and products in 8-bit integers, with the head that answers
with log probabilities without its logits in memory.

A case is a dict of plain values.  ``kind`` says which call one pass makes:

  linear   tokens quantised one by one, times weights of 8 bits
  score    log probabilities of given classes, entropy and top classes of rows of logits
  grad     the gradient of the logits, given those of log probabilities and entropy
  head     tokens quantised one by one, the 8-bit head's logits, and what score gives of them

``run`` computes them in plain torch operations in 32 bits, or, where ``own``
is set, by the library's calls."""

import math

import torch

own = False


def listed():
    return [
        # one stream's next frame through the gate projection of both directions: latency
        dict(name="linear_b1", kind="linear", M=1, N=4096, K=1024, bias=True, precision="bf16"),
        # a server's 64 streams
        dict(name="linear_b64", kind="linear", M=64, N=4096, K=1024, bias=True, precision="bf16"),
        # the paper's batch of 128 chunks of 21 frames
        dict(name="linear_b128", kind="linear", M=2688, N=4096, K=1024, bias=True, precision="bf16"),
        # a large product of long recordings at once
        dict(name="linear_large", kind="linear", M=16384, N=4096, K=4096, bias=False, precision="bf16"),
        # float32 features of 260 columns, sizes that no tile divides
        dict(name="linear_odd_fp32", kind="linear", M=777, N=1003, K=260, bias=True, precision="fp32"),
        # one stream's next frame: its state's score and five alternatives
        dict(name="score_b1_fp32", kind="score", M=1, K=32000, n=1, k=5, entropy=True, tau=1.0, masked=False,
             precision="fp32"),
        # forced alignment with confidences, the paper's batch
        dict(name="score_b128", kind="score", M=2688, K=32000, n=1, k=8, entropy=True, tau=1.0, masked=False,
             precision="bf16"),
        # lists of a lattice's states, ragged, some classes masked
        dict(name="score_lists_fp32", kind="score", M=1500, K=9001, n=33, k=0, entropy=False, tau=2.0, masked=True,
             precision="fp32"),
        # a step of sequence training with an entropy term, the paper's batch
        dict(name="grad_b128", kind="grad", M=2688, K=32000, n=1, entropy=True, tau=1.0, masked=False,
             precision="bf16"),
        # occupancies of a lattice's states in float32, odd sizes, some frames without a gradient
        dict(name="grad_lists_fp32", kind="grad", M=777, K=9001, n=21, entropy=False, tau=1.0, masked=True,
             precision="fp32"),
        # the paper's head for a server's 16 streams
        dict(name="head_b16", kind="head", M=16, P=256, K=32000, n=1, k=8, entropy=True, masked=False,
             precision="bf16"),
        # and for its batch
        dict(name="head_b128", kind="head", M=2688, P=256, K=32000, n=1, k=8, entropy=True, masked=False,
             precision="bf16"),
    ]


def _log_int(rng, lo, hi):
    hi = max(lo, hi)
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ones' ranges, at most as costly as the largest."""
    kind = rng.choice(["linear", "linear", "linear", "score", "score", "grad", "grad", "head", "head"])
    precision = "bf16" if rng.random() < 0.7 else "fp32"
    if kind == "linear":
        K = rng.choice([256, 260, 512, 1024, 2048, 4096]) if rng.random() < 0.5 else _log_int(rng, 16, 8192)
        N = rng.choice([256, 1024, 2048, 4096]) if rng.random() < 0.5 else _log_int(rng, 16, 16384)
        M = _log_int(rng, 1, min(16384, 270_000_000_000 // (N * K), 67_000_000 // N))
        return dict(kind=kind, M=M, N=N, K=K, bias=rng.random() < 0.6, precision=precision)
    K = 32000 if rng.random() < 0.3 else _log_int(rng, 60, 131072)
    n = rng.choice([0, 1, 1, _log_int(rng, 2, min(64, K // 2))])
    k = rng.choice([0, 1, _log_int(rng, 2, min(32, K // 2))])
    entropy = rng.random() < 0.6 or n + k == 0
    masked = rng.random() < 0.5
    if kind == "head":
        P = rng.choice([128, 256, 256, 512]) if rng.random() < 0.6 else _log_int(rng, 16, 512)
        M = _log_int(rng, 1, min(4096, 86_000_000 // K, 22_000_000_000 // (K * P)))
        return dict(kind=kind, M=M, P=P, K=K, n=n, k=k, entropy=entropy, masked=masked, precision=precision)
    M = _log_int(rng, 1, min(20000, (86_000_000 if precision == "bf16" else 43_000_000) // K))
    tau = rng.choice([1.0, 1.0, 2.0, 0.7])
    if kind == "score":
        return dict(kind=kind, M=M, K=K, n=n, k=k, entropy=entropy, tau=tau, masked=masked, precision=precision)
    n, entropy = max(n, 1), rng.random() < 0.5
    return dict(kind=kind, M=M, K=K, n=n, entropy=entropy, tau=tau, masked=masked, precision=precision)


# ------------------------------------------------------------------ inputs ---
def _type(case):
    return torch.bfloat16 if case["precision"] == "bf16" else torch.float32


def _distinct(M, K, n, g):
    """n classes a row, no class twice: an odd step that does not divide K."""
    step = 2 * torch.randint(0, max(1, K // 2), (M, 1), generator=g, device="cuda") + 1
    step = torch.where(torch.gcd(step, torch.full_like(step, K)) == 1, step, torch.ones_like(step))
    at = torch.randint(0, K, (M, 1), generator=g, device="cuda")
    return (at + step * torch.arange(n, device="cuda")) % K


def _ids(M, K, n, likely, g):
    """n classes a row: the first mostly one of the likely ones, the others any; lists end early (-1) in some rows."""
    if n == 0:
        return None
    ids = _distinct(M, K, n, g)
    hit = torch.rand(M, generator=g, device="cuda") < 0.8
    if likely is not None:
        hit = hit & ~(ids[:, 1:] == likely[:, None]).any(1)
        ids[:, 0] = torch.where(hit, likely, ids[:, 0])
    ends = torch.randint(1, n + 1, (M, 1), generator=g, device="cuda")
    short = torch.rand((M, 1), generator=g, device="cuda") < 0.3
    ids = torch.where(short & (torch.arange(n, device="cuda") >= ends), -1, ids)
    return ids.to(torch.int32)


def _int8(w):
    """Weights as a program keeps them: rows of 8-bit integers, a scale a row, columns padded with zeros to a
    multiple of 16."""
    amax = w.double().abs().amax(1)
    q = torch.round(w.double() * (127 / amax)[:, None]).to(torch.int8)
    return torch.nn.functional.pad(q, (0, -w.shape[1] % 16)), (amax / 127).float()


def _inputs(case, seed):
    """Device tensors made from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 71)
    t, kind, M, K = _type(case), case["kind"], case["M"], case["K"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = {"case": case}
    if kind == "linear":
        N = case["N"]
        s["x"] = (normal(M, K) * (0.5 + uniform(M, 1))).to(t)          # frames of different level
        s["w"], s["w_scale"] = _int8(normal(N, K) / math.sqrt(K) * (0.5 + uniform(N, 1)))
        s["bias"] = (uniform(N) * 2 - 1) * 0.1 if case["bias"] else None
        return s
    n = case["n"]
    if kind == "head":
        P = case["P"]
        w = normal(K, P) / math.sqrt(P)
        # a frame leans to one class, as a trained model's does
        likely = torch.randint(0, K, (M,), generator=g, device="cuda")
        s["x"] = (normal(M, P) + w[likely] * (uniform(M, 1) * 12)).to(t)
        s["w"], s["w_scale"] = _int8(w * 2)
        s["bias"] = normal(K) * 0.5
        if case["masked"]:                                             # states outside the inventory in use
            s["bias"][uniform(K) < 0.3] = -math.inf
        s["ids"] = _ids(M, K, n, likely, g)
        return s
    logits = normal(M, K) * 2
    m = max(1, min(16, K // 4))
    at = _distinct(M, K, m, g)
    logits.scatter_(1, at, torch.sort(normal(M, m) * 2 + 8, dim=1, descending=True).values)
    if case["masked"]:
        logits[uniform(M, K) < 0.2] = -math.inf
        if M > 2:
            logits[2] = -math.inf                                      # a row whose mask leaves nothing
    s["logits"] = logits.to(t)
    s["ids"] = _ids(M, K, n, at[:, 0], g)
    if kind == "grad":
        s["dlogprob"] = normal(M, n) / M
        if case["masked"]:
            s["dlogprob"][uniform(M) < 0.2] = 0.0                      # frames that are not trained on
        s["dentropy"] = normal(M) * 0.01 / M if case["entropy"] else None
    return s


def prepare(case, seed):
    """The inputs and the output buffers that a program keeps between passes."""
    s = _inputs(case, seed)
    t, kind, M = _type(case), case["kind"], case["M"]
    f32 = torch.float32

    def out(*shape, dtype=f32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if kind == "linear":
        s["out"] = {"y": out(M, case["N"], dtype=t)}
    elif kind == "grad":
        s["out"] = {"dlogits": out(M, case["K"], dtype=t)}
    else:
        s["out"] = {}
        if case["n"]:
            s["out"]["logprob"] = out(M, case["n"])
        if case["entropy"]:
            s["out"]["entropy"] = out(M)
        if case["k"]:
            s["out"].update(top=out(M, case["k"]), idx=out(M, case["k"], dtype=torch.int32))
    return s


# ------------------------------------------------------------- plain forms ---
def _plain_quantize(x):
    """Rows of integers (in float32) and their scales; the nearest integer is decided in 64 bits."""
    amax = x.float().abs().amax(1)
    scale = amax / torch.full_like(amax, 127.0)
    q = torch.round(x.double() * 127 / amax.double()[:, None])
    return torch.where(amax[:, None] > 0, q, 0.0).float(), scale


def _plain_product(s):
    """The product of whole numbers (their float32 sums are whole too: below 2^24), scaled."""
    q, scale = _plain_quantize(s["x"])
    y = (q @ s["w"][:, :q.shape[1]].float().t()) * (scale[:, None] * s["w_scale"])
    return y if s["bias"] is None else y + s["bias"]


def _plain_score(f, s, tau):
    c, out = s["case"], {}
    u = f / tau
    m = u.amax(1, keepdim=True)
    some = m > -math.inf                                               # not every class is masked
    v = torch.where(some, u - torch.where(some, m, 0.0), -math.inf)
    e = torch.exp(v)
    lz = torch.log(e.sum(1, keepdim=True))
    lp = torch.where(some, v - lz, -math.inf)
    if c["n"]:
        ids = s["ids"].long()
        out["logprob"] = torch.where(ids < 0, 0.0, torch.gather(lp, 1, ids.clamp(min=0)))
    if c["entropy"]:
        h = lz[:, 0] - torch.where(e > 0, e * v, 0.0).sum(1) / e.sum(1)
        out["entropy"] = torch.where(some[:, 0], h, 0.0)
    if c["k"]:
        i = torch.sort(f, dim=1, descending=True, stable=True).indices[:, :c["k"]]   # equal logits: the lower class first
        out.update(top=torch.gather(lp, 1, i), idx=i.to(torch.int32))
    return out


def _plain_grad(s):
    c = s["case"]
    u = s["logits"].float() / c["tau"]
    m = u.amax(1, keepdim=True)
    some = m > -math.inf
    v = torch.where(some, u - torch.where(some, m, 0.0), -math.inf)
    e = torch.exp(v)
    z = e.sum(1, keepdim=True)
    p = torch.where(some, e / z, 0.0)
    ids = s["ids"].long()
    g = torch.where(ids < 0, 0.0, s["dlogprob"])
    d = -p * g.sum(1, keepdim=True)
    if s["dentropy"] is not None:
        ev = torch.where(e > 0, v, 0.0)
        h = torch.log(z) - (e * ev).sum(1, keepdim=True) / z
        d = d - s["dentropy"][:, None] * p * (ev - torch.log(z) + h)
    d = d.scatter_add(1, ids.clamp(min=0), g)
    return {"dlogits": (torch.where(some, d, 0.0) / c["tau"]).to(s["logits"].dtype)}


# ------------------------------------------------------ the library's calls ---
def _ws(s, size):
    """The workspace that a program keeps, made on the first pass."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(size(), 1), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own(s):
    from paper_1907_05701_amd import binding as bd
    c, o = s["case"], s["out"]
    kind = c["kind"]
    if kind == "linear":
        ws = _ws(s, lambda: bd.int8_linear_ws_bytes(c["M"], s["w"].shape[1]))
        bd.int8_linear_rows(s["x"], s["w"], s["w_scale"], o["y"], ws, bias=s["bias"])
        return o
    if kind == "grad":
        bd.softmax_logprob_bwd_rows(s["logits"], o["dlogits"], ids=s["ids"], dlogprob=s["dlogprob"],
                                    dentropy=s["dentropy"], temperature=c["tau"])
        return o
    wanted = dict(ids=s["ids"], logprob=o.get("logprob"), entropy=o.get("entropy"), top=o.get("top"), idx=o.get("idx"))
    if kind == "score":
        bd.softmax_logprob_rows(s["logits"], temperature=c["tau"], **wanted)
        return o
    ws = _ws(s, lambda: bd.int8_logprob_ws_bytes(c["M"], c["K"], s["w"].shape[1]))
    bd.int8_logprob_rows(s["x"], s["w"], s["w_scale"], ws, bias=s["bias"], **wanted)
    return o


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    if kind == "linear":
        return {"y": _plain_product(s).to(s["x"].dtype)}
    if kind == "grad":
        return _plain_grad(s)
    if kind == "head":
        return _plain_score(_plain_product(s), s, 1.0)
    return _plain_score(s["logits"].float(), s, s["case"]["tau"])


# ------------------------------------------------------------------- work ----
def work(case):
    es, kind, M, K = (2 if case["precision"] == "bf16" else 4), case["kind"], case["M"], case["K"]
    if kind == "linear":
        N = case["N"]
        return {"bytes": M * K * es + N * K + 4 * N * (1 + case["bias"]) + M * N * es, "flops": 2 * M * N * K}
    n = case["n"]
    if kind == "grad":   # a maximum, a difference, an exponential and a sum; a difference, an exponential and a product
        return {"bytes": 2 * M * K * es + 8 * M * n + 4 * M * case["entropy"],
                "flops": (7 + 4 * case["entropy"]) * M * K}
    out = M * (8 * n + 8 * case["k"] + 4 * case["entropy"])
    per = 4 + 2 * case["entropy"]
    if kind == "score":
        return {"bytes": M * K * es + out, "flops": per * M * K}
    P = case["P"]
    return {"bytes": M * P * es + K * (P + 8) + out, "flops": (2 * P + per) * M * K}


# ----------------------------------------------------------- in 64 bits ------
def _exact_linear(s):
    x = s["x"].double()
    amax = x.abs().max(1, keepdim=True).values
    q = torch.zeros_like(x)
    live = amax[:, 0] > 0
    q[live] = torch.round(x[live] * 127 / amax[live])
    y = torch.matmul(q, s["w"].double()[:, :x.shape[1]].t().contiguous())
    y = y * (amax / 127) * s["w_scale"].double()
    return y if s["bias"] is None else y + s["bias"].double()


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "linear":
        return {"y": _exact_linear(s)}
    f = _exact_linear(s) if kind == "head" else s["logits"].double() / case["tau"]
    nothing = torch.isneginf(f).all(1)
    lp = torch.log_softmax(torch.where(nothing[:, None], 0.0, f), 1)   # rows with nothing left are put right below
    plogp = torch.xlogy(torch.exp(lp), torch.exp(lp))
    ids = None if s["ids"] is None else s["ids"].long()
    out = {}
    if kind == "grad":
        p = torch.exp(lp)
        g = s["dlogprob"].double() * (ids >= 0)
        d = torch.zeros_like(f).scatter_add_(1, ids.clamp(min=0), g) - p * g.sum(1, keepdim=True)
        if s["dentropy"] is not None:
            h = -plogp.sum(1, keepdim=True)
            d = d - s["dentropy"].double()[:, None] * (plogp + p * h)
        d[nothing] = 0.0
        return {"dlogits": d / case["tau"]}
    lp[nothing] = -math.inf
    if case["n"]:
        out["logprob"] = torch.gather(lp, 1, ids.clamp(min=0)).masked_fill(ids < 0, 0.0)
    if case["entropy"]:
        out["entropy"] = (-plogp.sum(1)).masked_fill(nothing, 0.0)
    if case["k"]:
        out["top"] = torch.topk(lp, case["k"], dim=1).values
        out["idx"] = None   # whole numbers
    return out
