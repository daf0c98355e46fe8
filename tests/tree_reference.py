"""Plain float64 forms of the tree log-probabilities and the policy loss (the
oracle's log Z and marginals, numpy otherwise), and random trees."""
import numpy as np

from oracle import oracle as orc
from paper_2008_03736_amd import workloads as W


def random_trees(lengths, n1, G, seed):
    """int32 [B, G, 2(N1-1)-1, 2]: random binary trees in preorder, rows of -1."""
    rng = np.random.default_rng(seed)
    R = 2 * (n1 - 1) - 1
    out = np.full((len(lengths), G, R, 2), -1, np.int32)
    for b, n in enumerate(lengths):
        for g in range(G):
            rows, todo = [], [(0, int(n))]
            while todo:
                i, j = todo.pop()
                rows.append((i, j))
                if j - i >= 2:
                    k = int(rng.integers(i + 1, j))
                    todo += [(k, j), (i, k)]
            out[b, g, :len(rows)] = rows
    return out


def spans_of(tree, n):
    """The rows among a tree's first 2n-1 that are spans of the sentence."""
    rows = tree[:2 * n - 1]
    return [(int(i), int(j)) for i, j in rows if 0 <= i < j <= n]


def log_probs(scores, lengths, trees, logz=None):
    """float64 [B, G]."""
    lz = orc.logz(scores, lengths, threads=8) if logz is None else logz
    s = scores.astype(np.float64)
    return np.array([[sum(s[b, i, j] for i, j in spans_of(t, int(n))) - lz[b] for t in trees[b]]
                     for b, n in enumerate(lengths)])


def here(counts, B, G):
    n = np.full(B, G) if counts is None else np.clip(counts, 0, G)
    return np.arange(G)[None] < n[:, None]


def policy_terms(logp, there, adv, old, ref, lo, hi, kl):
    """(loss [B], coefficients [B, G], their error per unit error of log p)."""
    share = 1.0 / np.maximum(there.sum(1, keepdims=True), 1)
    r = np.exp(np.minimum(logp - old, 80.0))
    q = np.zeros_like(logp) if ref is None else np.minimum(ref - logp, 80.0)
    kept = np.clip(r, 1.0 - lo, 1.0 + hi)
    free = r * adv <= kept * adv
    term = -np.where(free, r, kept) * adv + kl * (np.exp(q) - q - 1.0)
    c = np.where(free, -r * adv, 0.0) + kl * (1.0 - np.exp(q))
    slope = np.where(free, np.abs(r * adv), 0.0) + kl * (np.exp(q) + 1.0)
    z = lambda x: np.where(there, x, 0.0) * share
    return z(term).sum(1), z(c), z(slope)


def spread(coef, trees, lengths, mu):
    """sum_g c_g (1[(i,j) in y_g] - p(i,j)) on valid cells, NaN elsewhere."""
    B, n1 = len(lengths), mu.shape[1]
    out = np.where(W.valid_mask(np.asarray(lengths), n1), -coef.sum(1)[:, None, None] * mu, np.nan)
    for b, n in enumerate(lengths):
        for g in range(coef.shape[1]):
            for i, j in set(spans_of(trees[b, g], int(n))):
                out[b, i, j] += coef[b, g]
    return out
