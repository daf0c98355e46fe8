"""The operators that train a parser past its gold trees, as cases to be timed.

A fine-tuning step scores a batch's spans, takes the log-probabilities of a
few candidate trees a sentence (``tree_logprobs``), their clipped policy loss
with a KL term and its gradient with respect to the scores (``policy_loss``),
and goes back through the biaffine scorer to the boundary representations and
the weights (``biaffine_bwd``), which between the two passes may be held in 8
bits (``pack_rows``, ``unpack_rows``).

``run`` computes a case by elementary torch operations, or, where ``own`` is
true, by the calls of the public binding on the same inputs.  Lengths come
from the lognormal laws of the benchmark batches (treebank-like), scores from
N(0, sd^2), candidate trees from the CRF itself.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
FORBIDDEN = -1.0e4
CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.28, 0.05
BLOCK = 32          # entries that share a scale in the 8-bit form
E4M3_MAX = 448.0

# treebank-like length laws (mean, sd, shortest, longest)
TREEBANK = dict(mean=25.0, std=12.0, lo=2, hi=140)


def _case(op, B, mean=0.0, std=0.0, lo=1, hi=1, sd=2.0, trees=0, ragged=False, forbid=0.0, labels=1, d=0, held="bf16",
          pad=0, lseed=0, name=None):
    """op: the call; B sentences with lognormal lengths of (mean, std) within
    [lo, hi] (uniform where mean is 0) at seed lseed; sd, forbid: of the
    scores (share of spans at -1e4); trees: candidates a sentence, ragged: not
    all sentences have them all, some have none; labels, d: of the scorer;
    held: what its representations are held in; pad: fence posts past the
    longest sentence."""
    c = dict(op=op, B=B, mean=mean, std=std, lo=lo, hi=hi, sd=sd, trees=trees, ragged=ragged, forbid=forbid,
             labels=labels, d=d, held=held, pad=pad, lseed=lseed)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the candidates of one sentence of an interactive parser rescored: launches and latency only
        _case("logp", 1, lo=23, hi=23, trees=4, name="logp_one"),
        # old and reference log-probabilities of a development set's candidates
        _case("logp", 1700, **TREEBANK, trees=8, lseed=1, name="logp_dev"),
        # a fine-tuning minibatch of about 5,000 words, eight candidates each, some dropped
        _case("policy", 200, **TREEBANK, trees=8, ragged=True, name="policy_batch"),
        # the benchmark batch's lengths (`mixed`)
        _case("policy", 5000, **TREEBANK, trees=4, lseed=0, name="policy_mixed"),
        # paragraphs, past what one CU's LDS holds
        _case("policy", 24, lo=200, hi=300, sd=2.0, trees=16, forbid=0.05, lseed=2, name="policy_long"),
        # a label scorer's representations of a small batch: latency
        _case("pack", 32, lo=5, hi=40, d=100, name="pack_tiny"),
        # a span scorer's of the benchmark batch
        _case("pack", 5000, **TREEBANK, d=500, name="pack_mixed"),
        # the span scorer's backward pass, the paper's d = 500: one sentence
        _case("bwd", 1, lo=23, hi=23, d=500, name="bwd_one"),
        # a training minibatch of about 5,000 words
        _case("bwd", 200, **TREEBANK, d=500, name="bwd_batch"),
        # the benchmark batch, the representations in 16 bits and from their 8-bit form
        _case("bwd", 5000, **TREEBANK, d=500, name="bwd_mixed"),
        _case("bwd", 5000, **TREEBANK, d=500, held="8bit", name="bwd_mixed_8bit"),
        # the label scorer of a full treebank label set (d = 100)
        _case("bwd", 100, **TREEBANK, labels=138, d=100, lseed=3, name="bwd_labels"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """One more case: any call above on one sentence up to the largest batch
    listed, sentences of one word to paragraphs, 1 to 64 candidates, odd
    padding, d of 4 to 508, 1 to 160 labels."""
    op = rng.choice(["logp", "policy", "policy", "pack", "bwd", "bwd", "bwd"])
    lseed, pad = rng.randrange(1 << 30), rng.choice([0, 0, 1, 6])
    long = rng.random() < 0.25
    if long:
        hi = rng.randrange(144, 400)
        law = dict(lo=rng.choice([1, hi // 2, hi]), hi=hi)
        most = max(1, min(48, int(24 * (300.0 / hi) ** 3)))
    else:
        mean = rng.uniform(6.0, 32.0)
        law = dict(mean=round(mean, 2), std=round(mean * rng.uniform(0.3, 0.6), 2), lo=rng.choice([1, 2]),
                   hi=rng.choice([60, 100, 140]))
        most = 5000
    if op in ("logp", "policy"):
        trees = _log_uniform(rng, 1, 64)
        B = _log_uniform(rng, 1, max(1, min(most, 20000 // trees)))
        return _case(op, B, **law, sd=rng.choice([1.0, 2.0]), trees=trees, ragged=rng.random() < 0.5,
                     forbid=rng.choice([0.0, 0.0, 0.05]), pad=pad, lseed=lseed)
    d = 4 * rng.randrange(1, 128)
    held = rng.choice(["bf16", "bf16", "8bit"]) if op == "bwd" else "bf16"
    labels = _log_uniform(rng, 2, 160) if op == "bwd" and rng.random() < 0.4 else 1
    # padded gradients and label-wise products of bounded size
    room = 2.0e8 / (labels * (law["hi"] + 1) * (max(d, law["hi"]) if labels > 1 else 64))
    B = _log_uniform(rng, 1, max(1, min(most, int(room) if labels > 1 else 5000)))
    return _case(op, B, **law, labels=labels, d=d, held=held, pad=pad, lseed=lseed)


# --------------------------------------------------------------------------
# Inputs.

def _lengths(case):
    rng = np.random.default_rng(case["lseed"])
    if case["mean"] <= 0:
        return rng.integers(case["lo"], case["hi"] + 1, size=case["B"]).astype(np.int32)
    var_ln = math.log1p((case["std"] / case["mean"]) ** 2)
    x = rng.lognormal(math.log(case["mean"]) - var_ln / 2, math.sqrt(var_ln), size=case["B"])
    return np.clip(np.rint(x), case["lo"], case["hi"]).astype(np.int32)


def _n1(case, lengths):
    return int(lengths.max()) + 1 + case["pad"]


def _valid(lengths, n1):
    at = torch.arange(n1, device=DEVICE)
    return (at[:, None] < at)[None] & (at <= lengths[:, None])[:, None, :]


def _charts(scores, lengths):
    """Inside charts in 64 bits, by width: at_start[b, w, i] = alpha(i, i+w),
    at_end[b, w, j] = alpha(j-w, j), and log Z.  (64 bits: sums over hundreds
    of spans whose difference decides on which side of a clip border a ratio
    falls.)"""
    B, n1 = scores.shape[:2]
    s = torch.where(_valid(lengths, n1), scores, 0.0).double()
    at_start = torch.zeros((B, n1, n1), dtype=torch.float64, device=scores.device)
    at_end = torch.zeros_like(at_start)
    at_start[:, 1, :n1 - 1] = at_end[:, 1, 1:] = s.diagonal(1, 1, 2)
    for w in range(2, n1):
        pairs = at_start[:, 1:w, :n1 - w] + at_end[:, 1:w, w:].flip(1)
        top = pairs.amax(1, keepdim=True)
        at_start[:, w, :n1 - w] = at_end[:, w, w:] = \
            (top + (pairs - top).exp().sum(1, keepdim=True).log())[:, 0] + s.diagonal(w, 1, 2)
    b = torch.arange(B, device=scores.device)
    return s, at_start, at_end, at_start[b, lengths, 0]


def _marginals(s, at_start, at_end, lengths):
    """Span marginals from the charts: a span's probability is shared out over
    its splits, widest spans first."""
    B, n1 = s.shape[:2]
    by_start, by_end = torch.zeros_like(at_start), torch.zeros_like(at_end)
    mu = torch.zeros_like(s)
    for w in range(n1 - 1, 0, -1):
        m = by_start[:, w, :n1 - w] + by_end[:, w, w:]
        m[:, 0] += (lengths == w).double()
        mu.diagonal(w, 1, 2).copy_(m)
        if w > 1:
            inner = at_start[:, w, :n1 - w] - s.diagonal(w, 1, 2)
            share = (at_start[:, 1:w, :n1 - w] + at_end[:, 1:w, w:].flip(1) - inner[:, None]).exp() * m[:, None]
            by_start[:, 1:w, :n1 - w] += share
            by_end[:, 1:w, w:] += share.flip(1)
    return mu


def _sampled_trees(charts, lengths, trees, g):
    """Trees drawn from the CRF, [B, trees, 2 (N1 - 1) - 1, 2] in preorder,
    then rows of -1: every span's split by its probability given the span."""
    s, at_start, at_end, _ = charts
    B, n1 = s.shape[:2]
    T, R = B * trees, 2 * (n1 - 1) - 1
    b = torch.arange(B, device=DEVICE).repeat_interleave(trees)
    t = torch.arange(T, device=DEVICE)
    rows = torch.full((T, R, 2), -1, dtype=torch.int32, device=DEVICE)
    stack = torch.zeros((T, n1 + 1, 2), dtype=torch.long, device=DEVICE)
    stack[:, 0, 1] = lengths.long()[b]
    size = torch.ones(T, dtype=torch.long, device=DEVICE)
    split = torch.arange(1, max(2, int(lengths.max())), device=DEVICE)
    u = torch.rand((T, R), generator=g, device=DEVICE, dtype=torch.float64)
    for r in range(R):
        live = size > 0
        at = (size - 1).clamp(min=0)
        i, j = stack[t, at].unbind(1)
        w = j - i
        rows[:, r] = torch.where(live[:, None], torch.stack([i, j], 1).int(), rows[:, r])
        size = size - live.long()
        wide = live & (w >= 2)
        v = at_start[b[:, None], split, i[:, None]] + at_end[b[:, None], (w[:, None] - split).clamp(min=0), j[:, None]]
        v = torch.where(split < w[:, None], v, -math.inf)
        p = (v - v.amax(1, keepdim=True).clamp(min=-1e300)).exp().cumsum(1)
        cut = i + 1 + (p < u[:, r:r + 1] * p[:, -1:]).sum(1).clamp(max=n1).minimum((w - 2).clamp(min=0))
        at = size.clamp(max=n1 - 1)
        stack[t, at] = torch.where(wide[:, None], torch.stack([cut, j], 1), stack[t, at])
        at = (size + 1).clamp(max=n1)
        stack[t, at] = torch.where(wide[:, None], torch.stack([i, cut], 1), stack[t, at])
        size = size + 2 * wide.long()
    return rows.view(B, trees, R, 2)


def _tree_sums(s, trees):
    B, G, R = trees.shape[:3]
    n1 = s.shape[1]
    cell = trees[..., 0].long() * n1 + trees[..., 1]
    there = trees[..., 0] >= 0
    got = s.reshape(B, -1).gather(1, torch.where(there, cell, 0).view(B, -1)).view(B, G, R)
    return torch.where(there, got, 0.0).sum(2), torch.where(there, cell, 0), there


def _packed(x, lengths):
    """The 8-bit form of bf16 rows: e4m3 codes (a byte each, rows of a
    multiple of 32) and a power of two for each block of 32 (its exponent plus
    127).  Rows past a sentence's last post are left at zero."""
    B, n1, d = x.shape
    wide = (d + BLOCK - 1) // BLOCK * BLOCK
    there = (torch.arange(n1, device=x.device) <= lengths[:, None])[..., None]
    v = torch.zeros((B, n1, wide), device=x.device)
    v[..., :d] = torch.where(there, x.float(), 0.0)
    v = v.view(B, n1, -1, BLOCK)
    m, e = torch.frexp(v.abs().amax(3))                        # largest = m 2^e, m in [1/2, 1)
    e = torch.where(m > 0, e - 9 + (m > 0.875).int(), -127).clamp(min=-127)   # largest 2^-e <= 448
    codes = torch.ldexp(v, -e[..., None]).to(torch.float8_e4m3fn)
    scales = torch.where(there, e + 127, 0).to(torch.uint8)
    return codes.view(B, n1, wide).view(torch.uint8), scales


def _unpacked(codes, scales, d):
    """The values that an 8-bit form stands for, in 32 bits."""
    B, n1, wide = codes.shape
    v = codes.view(torch.float8_e4m3fn).float().view(B, n1, -1, BLOCK)
    return torch.ldexp(v, scales[..., None].int() - 127).view(B, n1, wide)[..., :d]


def prepare(case, seed):
    host = _lengths(case)
    lengths = torch.from_numpy(host).to(DEVICE)
    B, n1, d, L = case["B"], _n1(case, host), case["d"], case["labels"]
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)

    op = case["op"]
    x = dict(op=op, lengths=lengths, d=d)
    if op in ("logp", "policy"):
        G = case["trees"]
        x["scores"] = normal(B, n1, n1).mul_(case["sd"])
        if case["forbid"] > 0:
            hit = torch.rand((B, n1, n1), generator=g, device=DEVICE) < case["forbid"]
            x["scores"][hit] = FORBIDDEN
        charts = _charts(x["scores"], lengths)
        x["trees"] = _sampled_trees(charts, lengths, G, g)
        x["counts"] = None
        if case["ragged"]:
            x["counts"] = torch.randint(0, G + 1, (B,), generator=g, device=DEVICE, dtype=torch.int32)
        if op == "policy":
            logp = _tree_sums(charts[0], x["trees"])[0] - charts[3][:, None]
            # log ratios of a policy a few updates old; kept clear of the clip
            # borders, at which the last bit decides between two gradients
            ratio = normal(B, G).double() * 0.25
            for border in (math.log1p(-CLIP_LOW), math.log1p(CLIP_HIGH)):
                ratio = torch.where((ratio - border).abs() < 1e-3, border + 2e-3, ratio)
            x["old"] = (logp - ratio).float()
            x["ref"] = (logp + 0.4 * normal(B, G)).float()
            a = normal(B, G)
            x["adv"] = a - a.mean(1, keepdim=True) if G > 1 else a
            x["out"] = dict(loss=torch.zeros(B, device=DEVICE), logp=torch.zeros((B, G), device=DEVICE),
                            grad_scores=torch.zeros_like(x["scores"]))
        else:
            x["out"] = dict(logp=torch.zeros((B, G), device=DEVICE), logZ=torch.zeros(B, device=DEVICE))
    elif op == "pack":
        # activations: a common size a row, a few large entries
        v = normal(B, n1, d) * torch.exp(0.5 * normal(B, n1, 1))
        x["x"] = (v * torch.where(torch.rand((B, n1, d), generator=g, device=DEVICE) < 0.01, 8.0, 1.0)).bfloat16()
        wide = (d + BLOCK - 1) // BLOCK * BLOCK
        x["out"] = dict(codes=torch.zeros((B, n1, wide), dtype=torch.uint8, device=DEVICE),
                        scales=torch.zeros((B, n1, wide // BLOCK), dtype=torch.uint8, device=DEVICE))
        x["back"] = torch.zeros_like(x["x"])
    else:
        x["rl"], x["rr"] = normal(B, n1, d).bfloat16(), normal(B, n1, d).bfloat16()
        if case["held"] == "8bit":
            x["rl"], x["rr"] = _packed(x["rl"], lengths), _packed(x["rr"], lengths)
        ldw = (d + 1 + 7) // 8 * 8
        x["w"] = (normal(L, d, ldw) * (2.0 / d)).bfloat16()
        # a CRF loss's gradient: a probability, less one on a few spans
        shape = (B, n1, n1) if L == 1 else (B, n1, n1, L)
        p = torch.sigmoid(2.0 * normal(*shape) - 4.0)
        p -= (torch.rand(shape, generator=g, device=DEVICE) < 0.1 / L).float()
        valid = _valid(lengths, n1)
        x["grad"] = torch.where(valid if L == 1 else valid[..., None], p, 0.0)
        x["out"] = dict(grad_rl=torch.zeros((B, n1, d), dtype=torch.bfloat16, device=DEVICE),
                        grad_rr=torch.zeros((B, n1, d), dtype=torch.bfloat16, device=DEVICE),
                        grad_w=torch.zeros((L, d, ldw), device=DEVICE))
    if own:   # the batch's plan, which a program keeps (the plain forms have no use for one)
        from paper_2008_03736_amd import binding
        x["plan"] = binding.Plan(host, n1=n1, device=DEVICE)
    return x


# --------------------------------------------------------------------------
# One pass.

def run(x):
    op = x["op"]
    if own:
        plan = x["plan"]
        if op == "logp":
            return plan.tree_logprobs(x["scores"], x["trees"], counts=x["counts"], **x["out"])
        if op == "policy":
            return plan.policy_loss(x["scores"], x["trees"], x["adv"], x["old"], ref_logp=x["ref"], counts=x["counts"],
                                    clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL_COEF, **x["out"])
        if op == "pack":
            codes, scales = plan.pack_rows(x["x"], **x["out"])
            return plan.unpack_rows(codes, scales, x["d"], out=x["back"]), scales
        return plan.biaffine_bwd(x["rl"], x["rr"], x["w"], x["grad"], **x["out"])
    if op == "logp":
        return _plain_logp(x)
    if op == "policy":
        return _plain_policy(x)
    if op == "pack":
        codes, scales = _packed(x["x"], x["lengths"])
        return _unpacked(codes, scales, x["d"]).bfloat16(), scales
    return _plain_bwd(x)


def _counted(x, G):
    if x["counts"] is None:
        return torch.ones((x["scores"].shape[0], G), dtype=torch.bool, device=DEVICE)
    return torch.arange(G, device=DEVICE) < x["counts"][:, None]


def _plain_logp(x):
    s, _, _, logz = _charts(x["scores"], x["lengths"])
    sums, _, _ = _tree_sums(s, x["trees"])
    return torch.where(_counted(x, sums.shape[1]), sums - logz[:, None], 0.0).float(), logz.float()


def _plain_policy(x):
    s, at_start, at_end, logz = _charts(x["scores"], x["lengths"])
    mu = _marginals(s, at_start, at_end, x["lengths"])
    sums, cell, there = _tree_sums(s, x["trees"])
    B, G = sums.shape
    here = _counted(x, G)
    logp = sums - logz[:, None]
    each = here.sum(1, keepdim=True).clamp(min=1)
    adv, r = x["adv"].double(), (logp - x["old"]).exp()
    kept = r.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH)
    back = x["ref"] - logp
    kl = back.exp() - back - 1.0
    loss = torch.where(here, KL_COEF * kl - torch.minimum(r * adv, kept * adv), 0.0) / each
    c = KL_COEF * (1.0 - back.exp()) - torch.where(r * adv <= kept * adv, r * adv, 0.0)
    c = torch.where(here, c, 0.0) / each
    grad = -c.sum(1)[:, None, None] * mu
    grad.view(B, -1).scatter_add_(1, cell.view(B, -1), (c[..., None] * there).view(B, -1))
    return loss.sum(1).float(), torch.where(here, logp, 0.0).float(), grad.float()


def _rows(x):
    """[R^l ; 1] and R^r in 32 bits, zero past each sentence's last post."""
    n1 = x["grad"].shape[1]
    there = (torch.arange(n1, device=DEVICE) <= x["lengths"][:, None])[..., None]

    def whole(v):
        return torch.where(there, _unpacked(*v, x["d"]) if isinstance(v, tuple) else v.float(), 0.0)
    rl = whole(x["rl"])
    return torch.cat([rl, there.expand_as(rl[..., :1]).float()], 2), whole(x["rr"])


def _plain_bwd(x):
    one, rr = _rows(x)
    B, n1, d = rr.shape
    L, ldw = x["w"].shape[0], x["w"].shape[2]
    g = x["grad"].view(B, n1, n1, L).permute(0, 3, 1, 2).contiguous()
    w = x["w"][:, :, :d + 1].float()                              # [l, c, a]
    u = torch.matmul(g, rr[:, None])                              # U = G R^r: [b, l, i, c]
    u = u.permute(0, 2, 1, 3).reshape(B * n1, L * d)
    grad_rl = (u @ w[:, :, :d].reshape(L * d, d)).view(B, n1, d)
    grad_w = torch.zeros((L, d, ldw), device=DEVICE)
    # (64 bits: a sum over every post of the batch)
    grad_w[:, :, :d + 1] = (u.double().t().contiguous() @ one.double().view(B * n1, d + 1)).view(L, d, d + 1)
    v = torch.matmul(g.transpose(2, 3).contiguous(), one[:, None])   # G^T [R^l ; 1]: [b, l, j, a]
    v = v.permute(0, 2, 1, 3).reshape(B * n1, L * (d + 1))
    grad_rr = (v @ w.transpose(1, 2).reshape(L * (d + 1), d)).view(B, n1, d)
    return grad_rl.bfloat16(), grad_rr.bfloat16(), grad_w


# --------------------------------------------------------------------------
# What a pass cannot do without.

def work(case):
    """Bytes: each valid score, tree row, representation and weight read once,
    each valid output written once.  Operations: a multiply and an add per
    split of an inside sum (three times that with the marginals), the two
    triangular and the three dense products of the scorer's backward pass, a
    few per entry of the 8-bit form."""
    n = _lengths(case).astype(np.float64)
    d, L, G, op = case["d"], case["labels"], case["trees"], case["op"]
    cells, posts, splits = float((n * (n + 1) / 2).sum()), float((n + 1).sum()), float(((n ** 3 - n) / 6).sum())
    if op in ("logp", "policy"):
        kept = 0.5 if case["ragged"] else 1.0   # on average
        rows = kept * G * float((2 * n - 1).sum())
        if op == "logp":
            return {"bytes": 4 * cells + 8 * rows + 4 * (kept * G + 1) * len(n), "flops": 2 * splits + rows}
        return {"bytes": 8 * cells + 8 * rows + 4 * (4 * kept * G + 1) * len(n), "flops": 6 * splits + 2 * rows}
    if op == "pack":   # there and back
        return {"bytes": posts * 2 * (2 * d + d + math.ceil(d / BLOCK)), "flops": 4 * posts * d}
    held = 2 * d if case["held"] == "bf16" else d + math.ceil(d / BLOCK)
    return {"bytes": 2 * posts * (held + 2 * d) + 4 * cells * L + 6 * L * d * (d + 1),
            "flops": 2 * L * (3 * posts * d * (d + 1) + cells * (2 * d + 1))}


# --------------------------------------------------------------------------
# The definitions in 64 bits.

def _exact_policy(case, x):
    """Log Z by the recursion over spans kept as a list of diagonals, and its
    gradient by differentiation; the loss from its definition, differentiated
    through log p."""
    scores, lengths, trees = x["scores"], x["lengths"], x["trees"]
    B, n1 = scores.shape[:2]
    G = trees.shape[1]
    order = torch.argsort(lengths.long(), descending=True)
    logp = torch.zeros((B, G), dtype=torch.float64, device=DEVICE)
    logz = torch.zeros(B, dtype=torch.float64, device=DEVICE)
    loss, grad = torch.zeros_like(logz), torch.zeros(scores.shape, dtype=torch.float64, device=DEVICE)
    budget = 1.5e9
    at = 0
    while at < B:
        n = int(lengths[order[at]])
        take = max(1, min(B - at, int(budget / (n ** 3 / 6 + 1))))
        ids = order[at:at + take]
        at += take
        ln = lengths[ids].long()
        cells = _valid(ln, n1)[:, :n + 1, :n + 1]
        s = torch.where(cells, scores[ids][:, :n + 1, :n + 1], 0.0).double().requires_grad_(case["op"] == "policy")
        alpha = {1: s.diagonal(1, 1, 2)}
        for w in range(2, n + 1):
            m = n + 1 - w
            both = torch.stack([alpha[u][:, :m] + alpha[w - u][:, u:u + m] for u in range(1, w)])
            alpha[w] = torch.logsumexp(both, 0) + s.diagonal(w, 1, 2)
        z = torch.stack([alpha[w][:, 0] for w in range(1, n + 1)], 1).gather(1, ln[:, None] - 1)[:, 0]
        t = trees[ids].long()
        i, j = t.clamp(min=0).unbind(3)
        k = torch.arange(len(ids), device=DEVICE)[:, None, None]
        lp = (s[k, i, j] * (t[..., 0] >= 0)).sum(2) - z[:, None]
        logz[ids], logp[ids] = z.detach(), lp.detach()
        if case["op"] == "policy":
            left = None if x["counts"] is None else x["counts"][ids]
            keep = torch.ones_like(lp) if left is None else (torch.arange(G, device=DEVICE) < left[:, None]).double()
            a = x["adv"][ids].double()
            r = torch.exp(lp - x["old"][ids].double())
            first, second = r * a, torch.clip(r, 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * a
            gap = x["ref"][ids].double() - lp
            each = -torch.where(first <= second, first, second.detach()) + KL_COEF * (torch.expm1(gap) - gap)
            one = (each * keep).sum(1) / keep.sum(1).clamp(min=1.0)
            loss[ids] = one.detach()
            got, = torch.autograd.grad(one.sum(), s)
            full = torch.zeros((len(ids), n1, n1), dtype=torch.float64, device=DEVICE)
            full[:, :n + 1, :n + 1] = got
            grad[ids] = full
    if x["counts"] is not None:
        logp *= torch.arange(G, device=DEVICE) < x["counts"][:, None]
    return (loss, logp, grad) if case["op"] == "policy" else (logp, logz)


def exact(case, seed):
    x = prepare(case, seed)
    op = case["op"]
    if op in ("logp", "policy"):
        if int(x["lengths"].max()) > 420:
            return None
        return _exact_policy(case, x)
    if op == "pack":
        # the nearest value of the block's grid: spacing 2^-3 of the value's
        # own power of two, no finer than 2^-9, in units of the block's scale
        v = x["x"].double()
        B, n1, d = v.shape
        wide = -(-d // BLOCK) * BLOCK
        v = torch.nn.functional.pad(v, (0, wide - d)).view(B, n1, -1, BLOCK)
        v = v * (torch.arange(n1, device=DEVICE) <= x["lengths"][:, None])[..., None, None]
        top = v.abs().amax(3, keepdim=True)
        power = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / E4M3_MAX))
        power = torch.where(top > E4M3_MAX * torch.exp2(power), power + 1, power)
        power = torch.where(top <= E4M3_MAX * torch.exp2(power - 1), power - 1, power)
        step = torch.exp2(torch.frexp(v * torch.exp2(-power))[1].double().sub(1.0).clamp(min=-6.0) - 3.0 + power)
        return (torch.round(v / step) * step).view(B, n1, wide)[..., :d], None
    n1, d, L = x["grad"].shape[1], case["d"], case["labels"]
    if case["held"] == "8bit":
        rl, rr = (torch.exp2(s.double() - 127.0).repeat_interleave(BLOCK, 2) * c.view(torch.float8_e4m3fn).double()
                  for c, s in (x["rl"], x["rr"]))
        rl, rr = rl[..., :d], rr[..., :d]
    else:
        rl, rr = x["rl"].double(), x["rr"].double()
    w = x["w"].double()
    out = [torch.zeros(rl.shape, dtype=torch.float64, device=DEVICE) for _ in range(2)]
    grad_w = torch.zeros(w.shape, dtype=torch.float64, device=DEVICE)
    sizes = x["lengths"].tolist()
    # sentences of one length together, their posts as one long row of blocks
    for n in sorted(set(sizes)):
        ids = torch.tensor([b for b, m in enumerate(sizes) if m == n], device=DEVICE)
        a = torch.cat([rl[ids, :n + 1], torch.ones((len(ids), n + 1, 1), dtype=torch.float64, device=DEVICE)], 2)
        r = rr[ids, :n + 1]
        g = x["grad"][ids, :n + 1, :n + 1].double().view(len(ids), n + 1, n + 1, L)
        for q in range(L):
            gq = torch.triu(g[..., q], 1).contiguous()
            t = a @ w[q, :, :d + 1].t().contiguous()              # [R^l ; 1] W
            back = r @ w[q, :, :d]                                # R^r W^T, without the bias row
            out[0][ids, :n + 1] += gq @ back
            out[1][ids, :n + 1] += gq.transpose(1, 2).contiguous() @ t
            gr = gq @ r
            grad_w[q, :, :d + 1] += gr.reshape(-1, d).t().contiguous() @ a.reshape(-1, d + 1)
    return out[0], out[1], grad_w
