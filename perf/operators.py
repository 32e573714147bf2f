"""The operators of training on aggregated node features, as cases that can be timed and compared.

A graph model on top of the aggregation product normalises its features, scores
them against classes or against the rows of a node table, and updates a table
that is far larger than its other weights.  Kinds of work:

  norm       Y = layer norm of X with the row's mean and 1/deviation kept
  norm_back  dX, dgamma, dbeta of it
  xent       softmax cross entropy of the scores H W^T against labels; "train"
             returns the loss and both gradients, "eval" the loss
  adamw      one AdamW step over all tensors of a model, states in 32 bits, or
             in 8 bits with a scale for each 256 values

A label outside [0, V) marks a row that is not trained on.  States in 8 bits
are float8 tensors (e4m3 first moments, e5m2 second moments) with their
scales, rounded at random in proportion to the distance, from a counter hash
of the element's index and a seed that is an input.
"""
from __future__ import annotations

import math

import torch

own = False  # False: the plain forms; True: the framework's operators

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
BLOCK = 256
LR, BETA1, BETA2, AEPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 10
TINY = 2.0 ** -110  # a block with no larger value is held as zeros


def listed():
    return [
        # a sampled mini-batch of nodes with narrow features: launches and latency
        dict(name="norm-batch", kind="norm", m=128, n=64, x="f32", y="f32"),
        # aggregated features of the mid-sized graph, handed on in bfloat16
        dict(name="norm-features", kind="norm", m=262144, n=512, x="f32", y="bf16"),
        # backward pass over a graph of a million nodes: the weights' gradients sum over all rows
        dict(name="norm-back-nodes", kind="norm_back", m=1048576, n=256, x="f32", y="bf16"),
        # wide rows of an odd length (bag-of-words features)
        dict(name="norm-back-words", kind="norm_back", m=4001, n=6001, x="f16", y="f16"),
        # node classification over a whole graph: few classes, many rows
        dict(name="xent-classes", kind="xent", t=150001, d=256, v=41, x="f32", mode="train"),
        # one query node scored against every node of the mid-sized graph
        dict(name="xent-query", kind="xent", t=1, d=512, v=262144, x="bf16", mode="eval"),
        # a small batch of queries trained against a table: bound by the table's bytes
        dict(name="xent-batch", kind="xent", t=100, d=200, v=60013, x="f16", mode="train"),
        # single-precision scores against a mid-sized table
        dict(name="xent-single", kind="xent", t=4099, d=256, v=30011, x="f32", mode="train"),
        # a large batch against a large table: three matrix products
        dict(name="xent-table", kind="xent", t=8192, d=512, v=100003, x="bf16", mode="train"),
        # every weight of six layers at once: many small tensors
        dict(name="adamw-layers", kind="adamw", rows=4096, f=256, layers=6, bits=32, g="f32", copy=False),
        # a node table with states in 32 bits and a bfloat16 copy for the products
        dict(name="adamw-table", kind="adamw", rows=262144, f=512, layers=0, bits=32, g="bf16", copy=True),
        # a node table whose states are held in 8 bits, so that they fit next to the graph
        dict(name="adamw-table-8", kind="adamw", rows=1048576, f=256, layers=0, bits=8, g="bf16", copy=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_back", "xent", "xent", "adamw"])
    if kind in ("norm", "norm_back"):
        n = _log(rng, 16, 12000)
        m = _log(rng, 1, min(1048576, 2.0e8 / n))
        return dict(kind=kind, m=m, n=n, x=rng.choice(["f32", "bf16", "f16"]), y=rng.choice(["f32", "bf16", "f16"]))
    if kind == "xent":
        d, v = _log(rng, 8, 1024), _log(rng, 2, 262144)
        t = _log(rng, 1, max(2, min(200000, 4.0e11 / (d * v), 8.0e8 / v)))
        return dict(kind=kind, t=t, d=d, v=v, x=rng.choice(["f32", "bf16", "f16"]),
                    mode=rng.choice(["train", "train", "eval"]))
    f, bits = _log(rng, 8, 512), rng.choice([8, 32])
    return dict(kind=kind, rows=_log(rng, 10, 2.0e8 / f), f=f, layers=rng.choice([0, 1, 3] if bits == 8 else [0, 2, 5]),
                bits=bits, g=rng.choice(["f32", "bf16", "f16"]), copy=rng.random() < 0.3)


# ----------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _shapes(case):
    f = case["f"]
    return [(case["rows"], f)] + [s for _ in range(case["layers"]) for s in ((f, f), (f,), (f,))]


def _features(m, n, g):
    """Rows of different size and offset, as sums over neighbourhoods have."""
    x = torch.randn((m, n), generator=g, device=DEV)
    x *= torch.exp(0.7 * torch.randn((m, 1), generator=g, device=DEV))
    return x.add_(torch.randn((m, 1), generator=g, device=DEV))


def _hold(x, kind, top):
    """x (flat, float32) in 8 bits: codes, and the scale of each block (nearest codes)."""
    n = x.numel()
    b = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = b.abs().amax(1, keepdim=True) / top
    code = torch.where(scale > 0, b / scale, 0 * b).clamp(-top, top).to(kind)
    return code.view(-1)[:n].clone(), scale.view(-1).contiguous()


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    state = dict(case)
    if kind in ("norm", "norm_back"):
        m, n = case["m"], case["n"]
        x = _features(m, n, g)
        state["X"] = x.to(TYPES[case["x"]])
        state["gamma"] = 1 + 0.2 * torch.randn(n, generator=g, device=DEV)
        state["beta"] = 0.1 * torch.randn(n, generator=g, device=DEV)
        if kind == "norm_back":
            x = state["X"].float()
            state["mean"] = x.mean(1)
            state["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt()
            state["dY"] = torch.randn((m, n), generator=g, device=DEV).to(TYPES[case["y"]])
        return state
    if kind == "xent":
        t, d, v = case["t"], case["d"], case["v"]
        H = torch.randn((t, d), generator=g, device=DEV)
        # classes of different frequency: their rows have different lengths; scores have a deviation of about 2
        W = torch.randn((v, d), generator=g, device=DEV) * (2.0 / math.sqrt(d))
        W *= 0.5 + torch.rand((v, 1), generator=g, device=DEV)
        labels = (v * torch.rand(t, generator=g, device=DEV) ** 2).long().clamp_(max=v - 1)
        off = torch.rand(t, generator=g, device=DEV) < 0.1  # nodes without a label, or held out
        off[0] = False
        state["labels"] = torch.where(off, torch.full_like(labels, -1), labels)
        state["H"], state["W"] = H.to(TYPES[case["x"]]), W.to(TYPES[case["x"]])
        return state
    state["params"], state["grads"], state["m"], state["v"] = [], [], [], []
    for shape in _shapes(case):
        rows = shape[:1] + (1,) * (len(shape) - 1)
        size = 1e-3 * torch.exp(torch.randn(rows, generator=g, device=DEV))  # rarely and often visited rows
        state["params"].append(0.05 * torch.randn(shape, generator=g, device=DEV))
        state["grads"].append((size * torch.randn(shape, generator=g, device=DEV)).to(TYPES[case["g"]]))
        m = 0.3 * size * torch.randn(shape, generator=g, device=DEV)
        v = 0.01 * (size * torch.randn(shape, generator=g, device=DEV)).square() + 0.003 * size.square()
        if case["bits"] == 8:
            cm, sm = _hold(m.view(-1), torch.float8_e4m3fn, 448.0)
            cv, sv = _hold(v.view(-1), torch.float8_e5m2, 57344.0)
            m, v = (cm.view(shape), sm), (cv.view(shape), sv)
        state["m"].append(m)
        state["v"].append(v)
    state["copies"] = [torch.empty_like(p, dtype=torch.bfloat16) for p in state["params"]] if case["copy"] else None
    state["seed"] = int(seed) & 0x7FFFFFFF
    return state


# ------------------------------------------------------------ plain forms

def _plain_norm(s):
    x = s["X"].float()
    n = s["n"]
    mean = x.sum(1) / n
    x = x - mean[:, None]
    rstd = 1 / torch.sqrt((x * x).sum(1) / n + EPS)
    y = x * rstd[:, None] * s["gamma"] + s["beta"]
    return {"Y": y.to(TYPES[s["y"]]), "mean": mean, "rstd": rstd}


def _plain_norm_back(s):
    n, rstd = s["n"], s["rstd"][:, None]
    xhat = (s["X"].float() - s["mean"][:, None]) * rstd
    dy = s["dY"].float()
    dgamma, dbeta = (dy * xhat).sum(0), dy.sum(0)
    dy = dy * s["gamma"]
    dx = rstd * (dy - dy.sum(1, keepdim=True) / n - xhat * ((dy * xhat).sum(1, keepdim=True) / n))
    return {"dX": dx.to(TYPES[s["x"]]), "dgamma": dgamma, "dbeta": dbeta}


def _plain_xent(s):
    H, W, labels = s["H"].float(), s["W"].float(), s["labels"]
    rows = torch.arange(s["t"], device=H.device)
    there = (labels >= 0) & (labels < s["v"])
    at = torch.where(there, labels, 0)
    z = H @ W.t()
    target = z[rows, at]
    top = z.amax(1)
    z.sub_(top[:, None]).exp_()
    total = z.sum(1)
    row_loss = torch.where(there, torch.log(total) + top - target, 0.0)
    count = there.sum().clamp(min=1)
    out = {"loss": row_loss.sum() / count, "row_loss": row_loss}
    if s["mode"] == "train":
        z.mul_((1 / total)[:, None])
        z[rows, at] -= 1
        z.mul_((there / count)[:, None])
        out["dH"], out["dW"] = (z @ W).to(s["H"].dtype), (z.t() @ H).to(s["W"].dtype)
    return out


def _flat(tensors):
    return tensors[0].reshape(-1).float() if len(tensors) == 1 else torch.cat([t.reshape(-1) for t in tensors]).float()


def _blocks(tensors):
    """All tensors as one sequence of blocks, the last block of each filled up with zeros."""
    return torch.cat([torch.nn.functional.pad(t.reshape(-1).float(), (0, -t.numel() % BLOCK)) for t in tensors]).view(-1, BLOCK)


def _unblock(x, tensors):
    """The tensors' own values of such blocks."""
    parts = x.view(-1).split([t.numel() + -t.numel() % BLOCK for t in tensors])
    return [p[:t.numel()].view(t.shape) for p, t in zip(parts, tensors)]


def _noise(tensors, seed):
    """32 random bits for each element: a hash of its index and of its tensor's number and the seed."""
    low = 0xFFFFFFFF
    lens = [t.numel() + -t.numel() % BLOCK for t in tensors]
    x = torch.cat([torch.arange(n, device=DEV) * 0x9E3779B1 + (((seed + k * 0x632BE5AB) * 0x85157AF5) & low) for k, n in enumerate(lens)])
    x = x & low
    x = ((x ^ (x >> 16)) * 0x7C2E9D35) & low
    x = ((x ^ (x >> 15)) * 0x6A8F3B47) & low
    return (x ^ (x >> 16)).view(-1, BLOCK)


def _scale(x, top):
    """Scale of each block, and what a value is multiplied with; values that are not finite do not count."""
    big = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(1, keepdim=True)
    used = big >= TINY
    return torch.where(used, big / top, 0.0), torch.where(used, top / torch.where(used, big, 1.0), 0.0)


def _round(x, r, drop, least, top):
    """|x| to a code above or below it, in proportion to the distance: r are 16 random bits, `drop` the
    bits of the mantissa that go, `least` the smallest normal number (below it codes are evenly spaced)."""
    a = x.abs().clamp(max=top)
    off = torch.where(a < least, least, 0.0)
    bits = (a + off).view(torch.int32) + ((r << (drop - 16)) | (1 << (drop - 17))).to(torch.int32)
    q = ((bits >> drop) << drop).view(torch.float32) - off
    return torch.where(torch.isfinite(x), torch.copysign(q.clamp(max=top), x), math.nan)


def _plain_adamw(s):
    params, eight = s["params"], s["bits"] == 8
    pick = _blocks if eight else _flat
    p, g = pick(params), pick(s["grads"])
    if eight:
        m = pick([c for c, _ in s["m"]]) * torch.cat([x for _, x in s["m"]])[:, None]
        v = pick([c for c, _ in s["v"]]) * torch.cat([x for _, x in s["v"]])[:, None]
    else:
        m, v = pick(s["m"]), pick(s["v"])
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    den = torch.sqrt(v) / math.sqrt(1 - BETA2 ** STEP) + AEPS
    p = p * (1 - LR * DECAY) - (LR / (1 - BETA1 ** STEP)) * (m / den)
    back = (lambda x, like: _unblock(x, like)) if eight else \
        (lambda x, like: [a.view(t.shape) for a, t in zip(x.view(-1).split([t.numel() for t in like]), like)])
    torch._foreach_copy_(params, back(p, params))
    if eight:
        noise = _noise(params, s["seed"])
        (sm, im), (sv, iv) = _scale(m, 448.0), _scale(v, 57344.0)
        cm = _round(m * im, noise & 0xFFFF, 20, 2.0 ** -6, 448.0)
        cv = _round(v * iv, noise >> 16, 21, 2.0 ** -14, 57344.0)
        cv = torch.where((v * iv > 0) & (cv == 0), 2.0 ** -16, cv)
        counts = [x.numel() for _, x in s["m"]]
        for new, scale, old, kind in ((cm, sm, s["m"], torch.float8_e4m3fn), (cv, sv, s["v"], torch.float8_e5m2)):
            torch._foreach_copy_([c for c, _ in old], back(new.to(kind), params))
            torch._foreach_copy_([x for _, x in old], list(scale.view(-1).split(counts)))
    else:
        torch._foreach_copy_(s["m"], back(m, params))
        torch._foreach_copy_(s["v"], back(v, params))
    if s["copies"]:
        torch._foreach_copy_(s["copies"], params)
    return _updated(s)


def _updated(s):
    return {"params": s["params"], "m": s["m"], "v": s["v"], "copies": s["copies"] or []}


# -------------------------------------------------------------------- run

def run(state):
    kind = state["kind"]
    if not own:
        return {"norm": _plain_norm, "norm_back": _plain_norm_back, "xent": _plain_xent, "adamw": _plain_adamw}[kind](state)
    import paper_2507_02006_amd as aires
    if kind == "norm":
        Y, mean, rstd = aires.layer_norm(state["X"], state["gamma"], state["beta"], eps=EPS, out_dtype=TYPES[state["y"]])
        return {"Y": Y, "mean": mean, "rstd": rstd}
    if kind == "norm_back":
        dX, dgamma, dbeta = aires.layer_norm_backward(state["dY"], state["X"], state["mean"], state["rstd"], state["gamma"])
        return {"dX": dX, "dgamma": dgamma, "dbeta": dbeta}
    if kind == "xent":
        r = aires.linear_xent(state["H"], state["W"], state["labels"], grads=state["mode"] == "train")
        out = {"loss": r.loss, "row_loss": r.row_loss}
        if state["mode"] == "train":
            out["dH"], out["dW"] = r.dH, r.dW
        return out
    aires.adamw(state["params"], state["grads"], state["m"], state["v"], step=STEP, lr=LR, betas=(BETA1, BETA2),
                eps=AEPS, weight_decay=DECAY, seed=state["seed"], copies=state["copies"])
    return _updated(state)


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_back"):
        m, n, sx, sy = case["m"], case["n"], SIZE[case["x"]], SIZE[case["y"]]
        if kind == "norm":
            return {"bytes": m * n * (sx + sy) + 8 * m + 8 * n, "flops": 8.0 * m * n}
        return {"bytes": m * n * (2 * sx + sy) + 8 * m + 12 * n, "flops": 14.0 * m * n}
    if kind == "xent":
        t, d, v, size = case["t"], case["d"], case["v"], SIZE[case["x"]]
        both = case["mode"] == "train"
        return {"bytes": (2 if both else 1) * size * (t + v) * d + 12 * t + 4, "flops": (6.0 if both else 2.0) * t * v * d + 4.0 * t * v}
    n = sum(math.prod(s) for s in _shapes(case))
    states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (8 + SIZE[case["g"]] + states + (2 if case["copy"] else 0)), "flops": 15.0 * n}


# ------------------------------------------------------ results in 64 bits

def _exact_xent(case, s):
    H, W = s["H"].double(), s["W"].double()
    t, v = case["t"], case["v"]
    labels = s["labels"]
    there = (labels >= 0) & (labels < v)
    count = max(1, int(there.sum()))
    row_loss = torch.zeros(t, dtype=torch.float64, device=DEV)
    dH, dW = torch.zeros_like(H), torch.zeros_like(W)
    step = max(1, (1 << 28) // v)
    for r0 in range(0, t, step):
        h, l, ok = H[r0:r0 + step], labels[r0:r0 + step], there[r0:r0 + step]
        z = h @ W.t()
        lse = torch.logsumexp(z, 1)
        hot = ok.nonzero().squeeze(1)
        row_loss[r0 + hot] = (lse[hot] - z[hot, l[hot]])
        if case["mode"] == "train":
            z = torch.exp(z - lse[:, None])
            z[hot, l[hot]] -= 1.0
            z = z * (ok.double()[:, None] / count)
            dH[r0:r0 + step] = z @ W
            dW += z.t() @ h
    out = {"loss": row_loss.sum() / count, "row_loss": row_loss}
    return {**out, "dH": dH, "dW": dW} if case["mode"] == "train" else out


def _exact_code(x, u, bits, low, top):
    """Random rounding from its definition: neighbours of |x| are multiples of 2^(e - bits)."""
    a = x.abs()
    e = torch.frexp(a)[1] - 1  # a in [2^e, 2^(e + 1))
    unit = torch.ldexp(torch.ones_like(a), e.clamp(min=low) - bits)
    q = (torch.floor(a / unit + u) * unit).clamp(max=top)
    return torch.where(x < 0, -q, q)


def _exact_adamw(case, s):
    out = {"params": [], "m": [], "v": [], "copies": []}
    for k, (p, g) in enumerate(zip(s["params"], s["grads"])):
        n, g = p.numel(), g.double().view(-1)
        if case["bits"] == 8:
            (cm, sm), (cv, sv) = s["m"][k], s["v"][k]
            m = cm.double().view(-1) * sm.double().repeat_interleave(BLOCK)[:n]
            v = cv.double().view(-1) * sv.double().repeat_interleave(BLOCK)[:n]
        else:
            m, v = s["m"][k].double().view(-1), s["v"][k].double().view(-1)
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
        new = p.double().view(-1) * (1 - LR * DECAY)
        new -= LR * (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + AEPS)
        out["params"].append(new.view(p.shape))
        if case["copy"]:
            out["copies"].append(new.view(p.shape))
        if case["bits"] == 32:
            out["m"].append(m.view(p.shape))
            out["v"].append(v.view(p.shape))
            continue
        low = 0xFFFFFFFF
        h = (torch.arange(n, device=DEV) * 0x9E3779B1 + (s["seed"] + k * 0x632BE5AB) * 0x85157AF5 % (1 << 32)) & low
        h = ((h ^ (h >> 16)) * 0x7C2E9D35) & low
        h = ((h ^ (h >> 15)) * 0x6A8F3B47) & low
        h = h ^ (h >> 16)
        for name, x, r, bits, least, top in (("m", m, h % 65536, 3, -6, 448.0), ("v", v, h // 65536, 2, -14, 57344.0)):
            blocks = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
            scale = blocks.abs().amax(1) / top
            scale = torch.where(scale * top >= TINY, scale, torch.zeros_like(scale))
            each = scale.repeat_interleave(BLOCK)[:n]
            y = torch.where(each > 0, x / torch.where(each > 0, each, torch.ones_like(each)), torch.zeros_like(x))
            q = _exact_code(y, (r.double() + 0.5) / 65536, bits, least, top)
            if name == "v":
                q = torch.where((y > 0) & (q == 0), torch.full_like(q, 2.0 ** -16), q)
            out[name].append((q.view(p.shape), scale))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "xent":
        return _exact_xent(case, s)
    if kind == "adamw":
        return _exact_adamw(case, s)
    x, gamma, beta = s["X"].double(), s["gamma"].double(), s["beta"].double()
    if kind == "norm":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        return {"Y": (x - mean[:, None]) * rstd[:, None] * gamma + beta, "mean": mean, "rstd": rstd}
    dy, rstd = s["dY"].double(), s["rstd"].double()
    x.sub_(s["mean"].double()[:, None]).mul_(rstd[:, None])
    dgamma, dbeta = (dy * x).sum(0), dy.sum(0)
    dy.mul_(gamma)
    along, mean = (dy * x).mean(1), dy.mean(1)
    dy.sub_(mean[:, None]).sub_(x.mul_(along[:, None])).mul_(rstd[:, None])
    return {"dX": dy, "dgamma": dgamma, "dbeta": dbeta}
