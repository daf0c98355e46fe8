"""The operators around a scorer that is trained, as cases to be timed.

A training step normalises the rows that the scorer reads (``layer_norm``),
adds a learned bias by a span's width to its scores (``width_bias``), goes back
through both, and moves each weight matrix by its orthogonalised momentum
(``muon_step``; ``orthogonalize`` alone for a program with its own update).

``run`` computes a case by elementary torch operations, or, where ``own`` is
true, by the calls of the public binding on the same inputs.  Lengths come from
the lognormal laws of the benchmark batches (treebank-like).
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
NORM_EPS = 1e-7
STEPS = ((3.4445, -4.7750, 2.0315),) * 5
MU, RATE, DECAY = 0.95, 0.02, 0.01

# treebank-like length laws (mean, sd, shortest, longest)
TREEBANK = dict(mean=25.0, std=12.0, lo=2, hi=140)


def _rows(op, B, mean=0.0, std=0.0, lo=1, hi=1, d=0, wide=False, labels=1, buckets=0, reach=0, scores=False, pad=0, lseed=0,
          name=None):
    """op: the call; B sentences with lognormal lengths of (mean, std) within
    [lo, hi] (uniform where mean is 0) at seed lseed; pad: fence posts past the
    longest one.  d, wide: entries of a row, and whether they are float32;
    labels, buckets, reach: of the bias (the last bucket starts by that width);
    scores: its scores' gradient too, which a scorer that adds the bias itself
    has no use for."""
    c = dict(op=op, B=B, mean=mean, std=std, lo=lo, hi=hi, d=d, wide=wide, labels=labels, buckets=buckets, reach=reach,
             scores=scores, pad=pad, lseed=lseed)
    if name is not None:
        c["name"] = name
    return c


def _matrices(op, count, rows, cols, ld, nesterov=True, name=None):
    """count matrices of rows x cols at a row stride of ld."""
    c = dict(op=op, count=count, rows=rows, cols=cols, ld=ld, nesterov=nesterov)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the rows of one sentence of an interactive parser, the paper's d = 500: latency only
        _rows("norm", 1, lo=23, hi=23, d=500, name="norm_one"),
        # the rows of the benchmark batch (`mixed`)
        _rows("norm", 5000, **TREEBANK, d=500, name="norm_mixed"),
        # back through the rows of a training minibatch of about 5,000 words
        _rows("norm_bwd", 200, **TREEBANK, d=500, name="norm_bwd_batch"),
        # and of the benchmark batch
        _rows("norm_bwd", 5000, **TREEBANK, d=500, name="norm_bwd_mixed"),
        # a wide encoder's float32 states over paragraphs
        _rows("norm_bwd", 24, lo=200, hi=300, d=4096, wide=True, lseed=2, name="norm_bwd_wide"),
        # span scores of the benchmark batch
        _rows("bias", 5000, **TREEBANK, buckets=16, reach=64, name="bias_mixed"),
        # label scores of a full treebank label set
        _rows("bias", 100, **TREEBANK, labels=138, buckets=16, reach=64, lseed=3, name="bias_labels"),
        # their gradients: of a call of its own, and of the table alone
        _rows("bias_bwd", 5000, **TREEBANK, buckets=16, reach=64, scores=True, name="bias_bwd_mixed"),
        _rows("bias_bwd", 100, **TREEBANK, labels=138, buckets=16, reach=64, lseed=3, name="bias_bwd_labels"),
        # one update of the span scorer's W, d = 500 with its bias row
        _matrices("muon", 1, 500, 501, 504, name="muon_span"),
        # of the label scorer's, d = 100
        _matrices("muon", 138, 100, 101, 104, name="muon_labels"),
        # a wide layer's update direction
        _matrices("ortho", 1, 2048, 2048, 2048, name="ortho_wide"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """One more case: any call above on one sentence of a word up to the
    largest batch listed, odd padding, rows of 4 to 8,192 entries, 1 to 160
    labels, 1 to 64 buckets; one to 160 matrices of 1 to 2,048 rows and
    columns, odd strides."""
    op = rng.choice(["norm", "norm_bwd", "norm_bwd", "bias", "bias_bwd", "muon", "muon", "ortho"])
    if op in ("muon", "ortho"):
        rows, cols = _log_uniform(rng, 1, 2048), _log_uniform(rng, 1, 2048)
        p, q = min(rows, cols), max(rows, cols)
        room = int(2048 ** 3 / (p * p * q))
        count = 1 if rng.random() < 0.4 else _log_uniform(rng, 1, max(1, min(160, room, 2 ** 22 // (p * q))))
        return _matrices(op, count, rows, cols, cols + rng.choice([0, 0, 1, 3, 8]), nesterov=rng.random() < 0.7)
    lseed, pad = rng.randrange(1 << 30), rng.choice([0, 0, 1, 6])
    if rng.random() < 0.25:
        hi = rng.randrange(144, 400)
        law = dict(lo=rng.choice([1, hi // 2, hi]), hi=hi)
    else:
        mean = rng.uniform(6.0, 32.0)
        law = dict(mean=round(mean, 2), std=round(mean * rng.uniform(0.3, 0.6), 2), lo=rng.choice([1, 2]),
                   hi=rng.choice([60, 100, 140]))
    n1 = law["hi"] + 1 + pad
    if op in ("norm", "norm_bwd"):
        d = 4 * _log_uniform(rng, 1, 2048)
        B = _log_uniform(rng, 1, max(1, min(5000, int(1.5e8 / (n1 * d)))))
        return _rows(op, B, **law, d=d, wide=rng.random() < 0.3, pad=pad, lseed=lseed)
    labels = _log_uniform(rng, 2, 160) if rng.random() < 0.5 else 1
    B = _log_uniform(rng, 1, max(1, min(5000, int(4.5e7 / (n1 * n1 * labels)))))
    return _rows(op, B, **law, labels=labels, buckets=_log_uniform(rng, 1, 64), reach=_log_uniform(rng, 4, 400),
                 scores=op == "bias_bwd" and rng.random() < 0.5, pad=pad, lseed=lseed)


# --------------------------------------------------------------------------
# Inputs.

def _lengths(case):
    rng = np.random.default_rng(case["lseed"])
    if case["mean"] <= 0:
        return rng.integers(case["lo"], case["hi"] + 1, size=case["B"]).astype(np.int32)
    var_ln = math.log1p((case["std"] / case["mean"]) ** 2)
    x = rng.lognormal(math.log(case["mean"]) - var_ln / 2, math.sqrt(var_ln), size=case["B"])
    return np.clip(np.rint(x), case["lo"], case["hi"]).astype(np.int32)


def _buckets(n1, buckets, reach):
    """The bucket of each width: one for each of the first half, the others by
    the width's logarithm up to the one from which on all share the last."""
    w = np.arange(n1)
    single = (buckets + 1) // 2
    far = single + (buckets - single) * np.log(np.maximum(w, 1) / single) / math.log(max(reach, single + 1) / single)
    return np.clip(np.where(w <= single, w - 1, far), 0, buckets - 1).astype(np.int32)


def prepare(case, seed):
    op = case["op"]
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)

    if op in ("muon", "ortho"):
        n, r, c, ld = case["count"], case["rows"], case["cols"], case["ld"]
        x = dict(op=op, cols=c, nesterov=case["nesterov"])

        # a gradient: a few strong directions and a floor of noise
        def gradient():
            k = min(16, r, c)
            strong = (normal(n, r, k) * torch.exp(-0.2 * torch.arange(k, device=DEVICE))) @ normal(n, k, ld)
            return (1e-3 * (strong + normal(n, r, ld))).contiguous()

        x["grad"] = gradient()
        if op == "muon":
            x["momentum"] = 5.0 * (x["grad"] + gradient())
            x["w"] = normal(n, r, ld) * (1.0 / math.sqrt(c))
            x["out"] = dict(w_out=torch.zeros_like(x["w"]), momentum_out=torch.zeros_like(x["w"]))
        else:
            x["out"] = dict(out=torch.zeros_like(x["grad"]))
        return x

    host = _lengths(case)
    B, n1, d, L = case["B"], int(host.max()) + 1 + case["pad"], case["d"], case["labels"]
    x = dict(op=op, lengths=torch.from_numpy(host).to(DEVICE))
    if op in ("norm", "norm_bwd"):
        kind = torch.float32 if case["wide"] else torch.bfloat16
        # states: a size and an offset a row, a few entries that are large in every row
        v = normal(B, n1, d) * torch.exp(0.5 * normal(B, n1, 1)) + 0.3 * normal(B, n1, 1)
        x["x"] = (v * torch.where(torch.rand(d, generator=g, device=DEVICE) < 0.01, 8.0, 1.0)).to(kind)
        x["gamma"] = 1.0 + 0.2 * normal(d)
        if op == "norm":
            x["beta"] = 0.1 * normal(d)
            x["out"] = dict(out=torch.zeros((B, n1, d), dtype=torch.bfloat16, device=DEVICE))
        else:
            x["grad"] = (0.1 * normal(B, n1, d)).bfloat16()
            x["out"] = dict(grad_x=torch.zeros_like(x["x"]), grad_gamma=torch.zeros(d, device=DEVICE),
                            grad_beta=torch.zeros(d, device=DEVICE))
    else:
        shape = (B, n1, n1) if L == 1 else (B, n1, n1, L)
        x["buckets"] = torch.from_numpy(_buckets(n1, case["buckets"], case["reach"])).to(DEVICE)
        x["count"] = case["buckets"]
        x["need"] = (case["scores"], True)
        if op == "bias":
            x["scores"] = 2.0 * normal(*shape)
            x["table"] = 0.5 * normal(case["buckets"], L)
            x["out"] = dict(out=torch.zeros(shape, device=DEVICE))
        else:
            # a CRF loss's gradient: a probability, less one on a few spans
            p = torch.sigmoid(2.0 * normal(*shape) - 4.0)
            p -= (torch.rand(shape, generator=g, device=DEVICE) < 0.1 / L).float()
            x["grad"] = p
            x["out"] = dict(grad_table=torch.zeros((case["buckets"], L), device=DEVICE))
            if case["scores"]:
                x["out"]["grad_scores"] = torch.zeros(shape, device=DEVICE)
    if own:   # the batch's plan, which a program keeps (the plain forms have no use for one)
        from paper_2008_03736_amd import binding
        x["plan"] = binding.Plan(host, n1=n1, device=DEVICE)
    return x


# --------------------------------------------------------------------------
# One pass.

def run(x):
    op = x["op"]
    if own:
        if op == "norm":
            return x["plan"].layer_norm(x["x"], x["gamma"], x["beta"], eps=EPS, **x["out"])
        if op == "norm_bwd":
            return x["plan"].layer_norm_bwd(x["x"], x["gamma"], x["grad"], eps=EPS, **x["out"])
        if op == "bias":
            return x["plan"].width_bias(x["scores"], x["table"], x["buckets"], **x["out"])
        if op == "bias_bwd":
            return x["plan"].width_bias_bwd(x["grad"], x["buckets"], x["count"], need=x["need"], **x["out"])
        from paper_2008_03736_amd import binding
        if op == "muon":
            return binding.muon_step(x["w"], x["grad"], x["momentum"], cols=x["cols"], lr=RATE, weight_decay=DECAY, mu=MU,
                                     nesterov=x["nesterov"], scale=1.0, coefficients=STEPS, eps=NORM_EPS, **x["out"])
        return binding.orthogonalize(x["grad"], cols=x["cols"], coefficients=STEPS, eps=NORM_EPS, **x["out"])
    if op == "norm":
        _, hat, _ = _normalised(x)
        return torch.where(_there(x), hat * x["gamma"] + x["beta"], 0.0).bfloat16()
    if op == "norm_bwd":
        return _plain_norm_bwd(x)
    if op == "bias":
        n1 = x["scores"].shape[1]
        at = torch.arange(n1, device=DEVICE)
        bias = x["table"][x["buckets"][(at - at[:, None]).clamp(min=0)].long()]     # [i, j, l]
        s = x["scores"].view(*x["scores"].shape[:3], -1)
        return torch.where(_valid(x, n1)[..., None], s + bias, 0.0).view_as(x["scores"])
    if op == "bias_bwd":
        return _plain_bias_bwd(x)
    return _plain_update(x)


def _there(x):
    return (torch.arange(x["x"].shape[1], device=DEVICE) <= x["lengths"][:, None])[..., None]


def _valid(x, n1):
    at = torch.arange(n1, device=DEVICE)
    return (at[:, None] < at)[None] & (at <= x["lengths"][:, None])[:, None, :]


def _normalised(x):
    v = x["x"].float()
    v = v - v.mean(2, keepdim=True)
    r = (v.square().mean(2, keepdim=True) + EPS).rsqrt()
    return v, v * r, r


def _plain_norm_bwd(x):
    _, hat, r = _normalised(x)
    there = _there(x)
    dy = torch.where(there, x["grad"].float(), 0.0)
    u = dy * x["gamma"]
    grad_x = r * (u - u.mean(2, keepdim=True) - hat * (u * hat).mean(2, keepdim=True))
    hat = torch.where(there, hat, 0.0)
    # (64 bits: sums over every post of the batch)
    return (torch.where(there, grad_x, 0.0).to(x["x"].dtype), (dy * hat).sum((0, 1), dtype=torch.float64).float(),
            dy.sum((0, 1), dtype=torch.float64).float())


def _plain_bias_bwd(x):
    grad = x["grad"]
    n1 = grad.shape[1]
    g = torch.where(_valid(x, n1)[..., None], grad.view(*grad.shape[:3], -1), 0.0)
    at = torch.arange(n1, device=DEVICE)
    bucket = x["buckets"][(at - at[:, None]).clamp(min=0)].view(-1)
    member = (bucket == torch.arange(x["count"], device=DEVICE)[:, None]).double()      # [k, i j]
    # (64 bits: a sum over the batch)
    table = (member @ g.sum(0, dtype=torch.float64).view(n1 * n1, -1)).float()
    return (g.view_as(grad) if x["need"][0] else None), table


def _plain_update(x):
    c = x["cols"]
    grad = x["grad"][:, :, :c]
    u = grad
    if x["op"] == "muon":
        momentum = MU * x["momentum"][:, :, :c] + grad
        u = grad + MU * momentum if x["nesterov"] else momentum
    y = (u.double() / (u.double().square().sum((1, 2), keepdim=True).sqrt() + NORM_EPS)).float()
    tall = y.shape[1] > y.shape[2]
    y = y.transpose(1, 2).contiguous() if tall else y
    for a, b, e in STEPS:
        gram = torch.matmul(y, y.transpose(1, 2).contiguous())
        y = a * y + torch.matmul(b * gram + e * torch.matmul(gram, gram), y)
    y = y.transpose(1, 2) if tall else y
    if x["op"] == "ortho":
        x["out"]["out"][:, :, :c] = y
        return x["out"]["out"]
    x["out"]["w_out"][:, :, :c] = (1.0 - RATE * DECAY) * x["w"][:, :, :c] - RATE * y
    x["out"]["momentum_out"][:, :, :c] = momentum
    return x["out"]["w_out"], x["out"]["momentum_out"]


# --------------------------------------------------------------------------
# What a pass cannot do without.

def work(case):
    """Bytes: each valid row, score, gradient and weight read once, each valid
    output written once.  Operations: a few per entry; for the update the
    products of each step, the symmetric ones by half."""
    op = case["op"]
    if op in ("muon", "ortho"):
        p, q = sorted((case["rows"], case["cols"]))
        flops = case["count"] * len(STEPS) * (p * (p + 1) * q + p * p * (p + 1) + 2 * p * p * q)
        return {"bytes": case["count"] * p * q * (20 if op == "muon" else 8), "flops": flops}
    n = _lengths(case).astype(np.float64)
    d, L = case["d"], case["labels"]
    cells, posts = float((n * (n + 1) / 2).sum()), float((n + 1).sum())
    held = 4 if case["wide"] else 2
    if op == "norm":
        return {"bytes": posts * d * (held + 2) + 8 * d, "flops": 8 * posts * d}
    if op == "norm_bwd":
        return {"bytes": posts * d * (2 * held + 2) + 12 * d, "flops": 16 * posts * d}
    moved = 8 if op == "bias" or case["scores"] else 4
    return {"bytes": cells * L * moved + 4 * case["buckets"] * L, "flops": cells * L}


# --------------------------------------------------------------------------
# The definitions in 64 bits.

def exact(case, seed):
    x = prepare(case, seed)
    op = case["op"]
    if op in ("muon", "ortho"):
        c = case["cols"]
        grad = x["grad"].double()[..., :c]
        u = grad
        if op == "muon":
            momentum = grad + MU * x["momentum"].double()[..., :c]
            u = MU * momentum + grad if case["nesterov"] else momentum
        y = u / (torch.linalg.matrix_norm(u, keepdim=True) + NORM_EPS)
        # X (a + b X^T X + e (X^T X)^2), from the side with fewer entries in the product
        left = case["rows"] < c
        y = y.transpose(1, 2).contiguous() if left else y.contiguous()
        one = torch.eye(y.shape[2], dtype=torch.float64, device=DEVICE)
        for a, b, e in STEPS:
            inner = y.transpose(1, 2).contiguous() @ y
            y = y @ (a * one + inner @ (b * one + e * inner))
        y = y.transpose(1, 2) if left else y
        full = torch.zeros(x["grad"].shape, dtype=torch.float64, device=DEVICE)
        full[..., :c] = y
        if op == "ortho":
            return full
        second = torch.zeros_like(full)
        second[..., :c] = momentum
        full[..., :c] = x["w"].double()[..., :c] * (1.0 - RATE * DECAY) - RATE * y
        return full, second
    sizes = x["lengths"].tolist()
    if op in ("norm", "norm_bwd"):
        d = case["d"]
        at = torch.cat([torch.arange(n + 1) + b * x["x"].shape[1] for b, n in enumerate(sizes)]).to(DEVICE)
        out = torch.zeros((x["x"].shape[0] * x["x"].shape[1], d), dtype=torch.float64, device=DEVICE)
        gamma = x["gamma"].double()
        grad_gamma, grad_beta = torch.zeros_like(gamma), torch.zeros_like(gamma)
        for part in at.split(max(1, int(3e7 / d))):      # posts, some at a time
            v = x["x"].view(-1, d)[part].double()
            sd = torch.sqrt(torch.var(v, 1, correction=0, keepdim=True) + EPS)
            hat = (v - v.mean(1, keepdim=True)) / sd
            if op == "norm":
                out[part] = hat * gamma + x["beta"].double()
                continue
            dy = x["grad"].view(-1, d)[part].double()
            grad_gamma += torch.einsum("rd,rd->d", dy, hat)
            grad_beta += dy.sum(0)
            # the projection of dy gamma off the constant row and off hat
            t = dy * gamma
            t = t - t.mean(1, keepdim=True)
            out[part] = (t - hat * ((t * hat).sum(1, keepdim=True) / d)) / sd
        out = out.view(x["x"].shape)
        return out if op == "norm" else (out, grad_gamma, grad_beta)
    L = case["labels"]
    of_width = x["buckets"].tolist()
    if op == "bias":
        out = torch.zeros(x["scores"].shape, dtype=torch.float64, device=DEVICE)
        for w in range(1, max(sizes) + 1):     # a width's spans are a diagonal
            ends = torch.arange(w, x["scores"].shape[1], device=DEVICE) <= x["lengths"][:, None]
            ends = ends if L == 1 else ends[:, None]
            row = x["table"][of_width[w]].double()
            v = x["scores"].diagonal(w, 1, 2).double() + (row[0] if L == 1 else row[:, None])
            out.diagonal(w, 1, 2).copy_(torch.where(ends, v, 0.0))
        return out
    table = torch.zeros((case["buckets"], L), dtype=torch.float64, device=DEVICE)
    for w in range(1, max(sizes) + 1):
        ends = torch.arange(w, x["grad"].shape[1], device=DEVICE) <= x["lengths"][:, None]
        v = x["grad"].diagonal(w, 1, 2).double()
        v = torch.where(ends, v, 0.0).sum() if L == 1 else torch.where(ends[:, None], v, 0.0).sum((0, 2))
        table[of_width[w]] += v
    return (torch.where(_valid(x, x["grad"].shape[1]).view(x["grad"].shape[:3] + (1,) * (L > 1)), x["grad"].double(), 0.0)
            if case["scores"] else None), table
