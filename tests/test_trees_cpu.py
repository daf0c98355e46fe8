"""The policy loss's formulas against differences (float64, no GPU): what the
GPU tests compare the kernels with."""
import numpy as np

import tree_reference as T
from oracle import bruteforce as bf
from oracle import oracle as orc
from paper_2008_03736_amd import workloads as W


def test_log_probs_of_all_trees_sum_to_one():
    b = W.custom([4], seed=3, sd=1.5)
    every = [spans for spans, _ in bf.trees(0, 4)]
    R = 2 * 4 - 1
    trees = np.array(every, np.int32).reshape(1, len(every), R, 2)
    lp = T.log_probs(b.scores, b.lengths, trees)
    assert abs(np.exp(lp).sum() - 1.0) < 1e-12


def test_policy_gradient_against_differences():
    b = W.custom([2, 5, 7, 6], seed=1, sd=1.0)
    G, rng = 4, np.random.default_rng(2)
    trees = T.random_trees(b.lengths, b.n1, G, 5)
    there = T.here(np.array([4, 3, 4, 0]), 4, G)
    lp = T.log_probs(b.scores, b.lengths, trees)
    adv = rng.standard_normal((4, G))
    old, ref = lp - 0.3 * rng.standard_normal((4, G)), lp + 0.4 * rng.standard_normal((4, G))

    def loss(scores):
        return T.policy_terms(T.log_probs(scores, b.lengths, trees), there, adv, old, ref, 0.2, 0.3, 0.1)[0]

    mu = orc.marginals(b.scores, b.lengths)[1]
    grad = T.spread(T.policy_terms(lp, there, adv, old, ref, 0.2, 0.3, 0.1)[1], trees, b.lengths, mu)
    h = 2.0 ** -10   # exact in float32 on scores of this size; central differences: h^2 L'''/6 < 1e-6 a term
    for k, n in enumerate(b.lengths):
        for i in range(int(n)):
            for j in range(i + 1, int(n) + 1):
                up, dn = b.scores.copy(), b.scores.copy()
                up[k, i, j] += h
                dn[k, i, j] -= h
                step = float(up[k, i, j]) - float(dn[k, i, j])
                diff = (loss(up) - loss(dn)) / step
                assert abs(diff[k] - grad[k, i, j]) < 1e-4, (k, i, j)
