"""Tree log-probabilities and the clipped policy loss on the GPU against their
plain float64 forms (tree_reference.py).

Tolerances.  log Z is off by at most e = 1e-5 max(1, |log Z|) and marginals by
1e-4, as for the other entry points.  log p = s(x,y) - log Z is a float64
difference rounded once: e + 2^-24 |log p|.  A coefficient c_g moves by its
slope (d c / d log p, |A| r + kl (e^q + 1), over the count) times e (1.1: the
second order of an e below 0.01), the loss by the coefficient's slope sum
likewise, and float32 roundings of c_g, of the at most 64 terms of a cell's
sum and of the products are below 2^-24 times 70 sums of |c_g|.  Ratios are
kept further from a clip border than e.
"""
import numpy as np
import pytest

import tree_reference as T
from oracle import oracle as orc
from paper_2008_03736_amd import binding as B
from paper_2008_03736_amd import workloads as W

pytestmark = pytest.mark.gpu

LO, HI, KL = 0.2, 0.3, 0.1


@pytest.fixture(scope="module")
def torch():
    import torch as _t

    if not _t.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load()
    return _t


def inputs(b, G, counts, seed):
    rng = np.random.default_rng(seed)
    trees = T.random_trees(b.lengths, b.n1, G, seed)
    lz, mu = orc.marginals(b.scores, b.lengths, threads=16)
    lp = T.log_probs(b.scores, b.lengths, trees, lz)
    ratio = 0.25 * rng.standard_normal(lp.shape)
    for border in (np.log1p(-LO), np.log1p(HI)):
        ratio = np.where(np.abs(ratio - border) < 0.02, border + 0.03, ratio)
    old, ref = (lp - ratio).astype(np.float32), (lp + 0.4 * rng.standard_normal(lp.shape)).astype(np.float32)
    adv = rng.standard_normal(lp.shape).astype(np.float32)
    return trees, lz, mu, lp, old, ref, adv


def check(torch, b, G, counts=None, flags=0, seed=0, ref=True, up=False, trees=None):
    t, lz, mu, lp, old, ref_lp, adv = inputs(b, G, counts, seed)
    if trees is not None:
        t = trees(t)
        lp = T.log_probs(b.scores, b.lengths, t, lz)
        old, ref_lp = (lp + 0.1).astype(np.float32), (lp - 0.2).astype(np.float32)
    Bn, dev = len(b.lengths), torch.device("cuda", 0)
    cu = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(dev)
    g = np.linspace(-1.5, 2.0, Bn).astype(np.float32) if up else None
    s, cn = cu(b.scores), cu(None if counts is None else np.asarray(counts, np.int32))
    with B.Plan(b.lengths, n1=b.n1, flags=flags, device=dev) as plan:
        lp1, lz1 = plan.tree_logprobs(s, cu(t), counts=cn, logp=torch.full((Bn, G), 7.5, device=dev))
        loss, lp2, grad = plan.policy_loss(s, cu(t), cu(adv), cu(old), ref_logp=cu(ref_lp) if ref else None, counts=cn,
                                           clip_low=LO, clip_high=HI, kl_coef=KL if ref else 0.0, grad_loss=cu(g),
                                           logp=torch.full((Bn, G), 7.5, device=dev),
                                           grad_scores=torch.full_like(s, 7.5))
        back = plan.tree_logprobs_bwd(s, cu(t), cu(adv), counts=cn, grad_scores=torch.full_like(s, 7.5))
        torch.cuda.synchronize()
    lp1, lz1, loss, lp2, grad, back = (x.cpu().numpy().astype(np.float64) for x in (lp1, lz1, loss, lp2, grad, back))
    there = T.here(counts, Bn, G)
    e = 1e-5 * np.maximum(1.0, np.abs(lz))
    assert np.all(np.abs(lz1 - lz) <= e)
    for x in (lp1, lp2):
        assert np.all(np.abs(x - lp)[there] <= (e[:, None] + 2.0 ** -24 * np.abs(lp))[there])
        assert np.all(x[~there] == 7.5)
    want, c, slope = T.policy_terms(lp, there, adv.astype(np.float64), old.astype(np.float64),
                                    ref_lp.astype(np.float64) if ref else None, LO, HI, KL if ref else 0.0)
    assert np.all(np.abs(loss - want) <= 1.1 * e * slope.sum(1) + 2.0 ** -24 * np.abs(want) + 1e-12)
    valid = W.valid_mask(np.asarray(b.lengths), b.n1)
    worst = 0.0
    for got, coef, move, scale in ((grad, c, slope, np.ones(Bn) if g is None else g),
                                   (back, np.where(there, adv, 0.0).astype(np.float64), 0.0 * slope, np.ones(Bn))):
        err = np.abs(got - scale[:, None, None] * T.spread(coef, t, b.lengths, mu))
        tol = 2.2 * e * move.sum(1) + 1e-4 * np.abs(coef.sum(1)) + 2.0 ** -24 * 70 * np.abs(coef).sum(1)
        tol = (np.abs(scale) * tol + 1e-12)[:, None, None]
        assert np.all((err <= tol)[valid]), float((err / tol)[valid].max())
        assert np.all(got[~valid] == 7.5)
        worst = max(worst, float((err / tol)[valid].max()))
    return grad, worst


@pytest.mark.parametrize("G", [1, 3, 8, 32, 33, 64])
def test_short_sentences(torch, G):
    b = W.custom([1, 2, 3, 4, 5, 9, 17, 40, 64, 65], seed=G, sd=1.5, n1=70)
    check(torch, b, G, seed=G)


@pytest.mark.parametrize("lengths,flags", [([90, 91, 127, 128, 139, 5], 0), ([140, 150, 200, 30], 0),
                                           ([20, 33, 60], B.CRF_FORCE_SPILL), ([460, 12], 0), ([460, 12], B.CRF_NO_TEAMS)])
def test_long_sentences(torch, lengths, flags):
    # stripes of rows (a mask word a cell past 90 words), workspace charts, teams
    check(torch, W.custom(lengths, seed=7, sd=1.0), 6, flags=flags, up=True)


def test_stripes_of_two_words(torch):
    check(torch, W.custom([64, 65, 90, 128], seed=4, sd=1.0), 40, counts=[40, 33, 1, 0])


def test_counts(torch):
    b = W.custom([6, 7, 8, 9, 30, 1], seed=2)
    check(torch, b, 5, counts=[5, 0, 1, -3, 9, 2], up=True)


def test_no_reference(torch):
    check(torch, W.custom([6, 30, 2], seed=5), 4, ref=False)


def test_rows_that_are_no_spans_and_repeated_spans(torch):
    b = W.custom([12, 5, 20], seed=6)

    def spoil(t):
        t = t.copy()
        t[:, 0, 2] = (4, 2)          # no span
        t[:, 0, 3] = (-1, 3)
        t[:, 1, 4] = (0, 1 << 20)
        t[:, 2, 3] = t[:, 2, 0]      # the root twice: its score again, one in the gradient
        t[:, 3] = t[:, 3, ::-1]      # some rows past the first 2n - 1
        return t
    check(torch, b, 4, trees=spoil)


def test_spans_of_every_tree_have_no_gradient(torch):
    b = W.custom([8, 23], seed=9)
    grad, _ = check(torch, b, 7, counts=[7, 6])
    for k, n in enumerate(b.lengths):
        assert grad[k, 0, n] == 0.0
        assert all(grad[k, i, i + 1] == 0.0 for i in range(n))


def test_forbidden_spans(torch):
    # near-forbidden spans, some of them in the trees: log p of -1e4 and less
    check(torch, W.custom([20, 40, 7], seed=3, sd=2.0, forbid=0.1), 6)


def test_huge_log_ratios_stay_finite(torch):
    dev = torch.device("cuda", 0)
    b = W.custom([5, 6], seed=1)
    t = T.random_trees(b.lengths, b.n1, 2, 1)
    one = torch.ones((2, 2), device=dev)
    with B.Plan(b.lengths, n1=b.n1, device=dev) as plan:
        s = torch.from_numpy(b.scores).to(dev)
        loss, lp, grad = plan.policy_loss(s, torch.from_numpy(t).to(dev), -one, -1e6 * one, ref_logp=-1e6 * one,
                                          kl_coef=0.1)
        assert torch.isfinite(loss).all() and torch.isfinite(grad[:, 0, 1]).all()
        # r = e^80: the loss is r (its KL term 0.1 (1e6 - 1) is nothing beside it)
        assert abs(float(loss[0]) / np.exp(80.0) - 1.0) < 1e-6


def test_differentiable_forms(torch):
    dev = torch.device("cuda", 0)
    b = W.custom([9, 14, 3], seed=8)
    G = 3
    trees, lz, mu, lp, old, ref, adv = inputs(b, G, None, 8)
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)
    with B.Plan(b.lengths, n1=b.n1, device=dev) as plan:
        s = cu(np.nan_to_num(b.scores)).requires_grad_(True)
        lpt = B.tree_log_prob(s, cu(trees), plan)
        (lpt * cu(adv)).sum().backward()
        want = plan.tree_logprobs_bwd(s.detach(), cu(trees), cu(adv))
        assert torch.equal(s.grad, want)
        s.grad = None
        loss = B.policy_loss(s, cu(trees), cu(adv), cu(old), plan, ref_logp=cu(ref), kl_coef=KL)
        loss.mean().backward()
        _, _, grad = plan.policy_loss(s.detach(), cu(trees), cu(adv), cu(old), ref_logp=cu(ref), kl_coef=KL)
        assert torch.allclose(s.grad, grad / 3, rtol=2.0 ** -22, atol=0)


def test_captured_and_other_stream(torch):
    dev = torch.device("cuda", 0)
    b = W.custom([9, 30, 50, 2], seed=11)
    G = 4
    trees, lz, mu, lp, old, ref, adv = inputs(b, G, None, 11)
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)
    s, tr, ad, ol, rf = (cu(x) for x in (b.scores, trees, adv, old, ref))
    with B.Plan(b.lengths, n1=b.n1, device=dev) as plan:
        call = lambda x: plan.policy_loss(x, tr, ad, ol, ref_logp=rf, kl_coef=KL)
        want = [call(s), call(s * 0.5)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = call(s)
        torch.cuda.current_stream().wait_stream(side)
        for x, y in zip(other, want[0]):
            assert torch.equal(x, y)
        held = s.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call(held)
        for k in (0, 1, 0, 1):
            held.copy_(s if k == 0 else s * 0.5)
            graph.replay()
            torch.cuda.synchronize()
            call(s)   # eager work between the replays
            for x, y in zip(out, want[k]):
                assert torch.equal(x, y)


def test_refusals(torch):
    dev = torch.device("cuda", 0)
    b = W.custom([4, 6], seed=0)
    s = torch.from_numpy(b.scores).to(dev)
    t = torch.from_numpy(T.random_trees(b.lengths, b.n1, 2, 0)).to(dev)
    f = torch.zeros((2, 2), device=dev)
    with B.Plan(b.lengths, n1=b.n1, device=dev) as plan:
        for bad, what in ((dict(clip_low=-0.1), "clip_low"), (dict(clip_low=1.5), "clip_low"),
                          (dict(clip_high=-1.0), "clip_high"), (dict(clip_high=float("nan")), "clip_high"), (dict(clip_low=float("nan")), "clip_low"),
                          (dict(clip_high=float("inf")), "clip_high"), (dict(kl_coef=float("nan"), ref_logp=f), "kl_coef"),
                          (dict(kl_coef=-1.0, ref_logp=f), "kl_coef"), (dict(kl_coef=0.1), "ref_logp"),
                          (dict(grad_scores=s), "alias")):
            with pytest.raises(B.CrfError, match=what):
                plan.policy_loss(s, t, f, f, **bad)
        with pytest.raises(ValueError):
            plan.policy_loss(s, t, f[:1], f)
        with pytest.raises(ValueError):
            plan.policy_loss(s, t.long(), f, f)
        with pytest.raises(ValueError):
            plan.tree_logprobs(s, t[:, :, :-1])
        with pytest.raises(B.CrfError, match="num_trees"):
            plan.tree_logprobs(s, t.repeat(1, 40, 1, 1))
        ws = plan._workspace(256)
        with pytest.raises(B.CrfError, match="workspace"):
            B.crf_tree_logprobs(plan._handle, s.data_ptr(), t.data_ptr(), 2, None, f.data_ptr(), None, ws.data_ptr(), 255,
                                None)
        with pytest.raises(B.CrfError, match="8-byte"):
            B.crf_tree_logprobs(plan._handle, s.data_ptr(), t.data_ptr() + 4, 2, None, f.data_ptr(), None, ws.data_ptr(),
                                256, None)
    with B.Plan(b.lengths, n1=b.n1, num_labels=3, device=dev) as plan:
        s3 = torch.zeros((2, b.n1, b.n1, 3), device=dev)
        with pytest.raises(B.CrfError, match="labelled"):
            plan.tree_logprobs(s3, t)


def test_refused_aliases(torch):
    # the stripes of a long sentence each read what one of them would overwrite
    dev = torch.device("cuda", 0)
    b = W.custom([4, 120], seed=0)
    s = torch.from_numpy(b.scores).to(dev)
    t = torch.from_numpy(T.random_trees(b.lengths, b.n1, 2, 0)).to(dev)
    f, g, up = torch.zeros((2, 2), device=dev), torch.zeros((2, 2), device=dev), torch.ones(2, device=dev)
    with B.Plan(b.lengths, n1=b.n1, device=dev) as plan:
        for bad in (dict(logp=f), dict(logp=g), dict(ref_logp=up.repeat(2, 1), loss=up, grad_loss=up)):
            with pytest.raises(B.CrfError, match="alias"):
                plan.policy_loss(s, t, f, g, **bad)
        with pytest.raises(TypeError):   # would scale the gradient but not the loss that it is the gradient of
            B.policy_loss(s, t, f, g, plan, grad_loss=up)


@pytest.mark.parametrize("where", ["advantages", "old_logp", "ref_logp", "log Z"])
def test_nan_reaches_the_loss_and_its_gradient(torch, where):
    # sentence 1's tree 2 (absent in sentence 3, whose counts leave it out)
    dev = torch.device("cuda", 0)
    b = W.custom([6, 100, 9, 5], seed=12)
    G, counts = 3, [3, 3, 0, 2]
    trees, lz, mu, lp, old, ref, adv = inputs(b, G, counts, 12)
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)
    s = cu(b.scores)
    given = dict(advantages=cu(np.abs(adv)), old_logp=cu(old), ref_logp=cu(ref))
    with B.Plan(b.lengths, n1=b.n1, device=dev) as plan:
        call = lambda x: plan.policy_loss(x, cu(trees), **given, counts=cu(np.asarray(counts, np.int32)), kl_coef=KL,
                                          logp=torch.full((4, G), 7.5, device=dev), grad_scores=torch.full_like(s, 7.5))
        want = call(s)
        if where == "log Z":
            s = s.clone()
            s[1, 4, 5] = float("nan")   # a word: in log Z and in every tree
        else:
            given[where][1, 2] = given[where][3, 2] = float("nan")
        loss, logp, grad = call(s)
    there, valid = T.here(counts, 4, G), W.valid_mask(np.asarray(b.lengths), b.n1)
    assert np.array_equal(np.isnan(loss.cpu().numpy()), [False, True, False, False])
    nan_logp = there & (np.arange(4) == 1)[:, None] if where == "log Z" else np.zeros_like(there)
    assert np.array_equal(np.isnan(logp.cpu().numpy()), nan_logp)
    assert np.array_equal(np.isnan(grad.cpu().numpy()), valid & (np.arange(4) == 1)[:, None, None])
    others = [0, 2, 3]
    for x, y in zip((loss, logp, grad), want):
        assert torch.equal(x[others], y[others])


def test_reference_without_a_kl_term(torch):
    # kl_coef = 0: the reference is not part of the loss, also a tree it rules out
    dev = torch.device("cuda", 0)
    b = W.custom([6, 80], seed=13)
    trees, lz, mu, lp, old, ref, adv = inputs(b, 2, None, 13)
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)
    ref[0, 1], ref[1, 0] = -np.inf, np.nan
    with B.Plan(b.lengths, n1=b.n1, device=dev) as plan:
        call = lambda r: plan.policy_loss(cu(b.scores), cu(trees), cu(adv), cu(old), ref_logp=r)
        for x, y in zip(call(cu(ref)), call(None)):
            assert torch.equal(x, y)


# log2(e) as the charts hold it, relative to itself: every score that a tree is
# free to have is scaled by it, in the tree's score as in log Z.
CHART_SCORE = float(np.float32(np.log2(np.e))) / np.log2(np.e)


@pytest.mark.parametrize("lengths,flags", [([139, 120, 130, 138], 0), ([300, 250, 300, 300], 0),
                                           ([300, 250, 300], B.CRF_FORCE_SPILL), ([500, 460, 600, 480], 0),
                                           ([500, 460, 600], B.CRF_NO_TEAMS), ([1000, 700], 0)])
def test_log_probs_of_long_sentences_are_exact(torch, lengths, flags):
    """An absolute bound, which log Z in float32, a shift of float32's own steps
    and a tree's score without the charts' factor would each miss.  A chart's
    value is off by rounding its sum, its score factor and their product: taken
    as independent errors of at most 2^-23 of it (root mean square), the n - 2
    free nodes of a tree come to sqrt(n) 2^-23, and five times that is allowed.
    Ratios exp(log p - old) have float32's relative steps, 2^-24, on top."""
    dev = torch.device("cuda", 0)
    b = W.custom(lengths, seed=21, sd=2.0)
    Bn, G = len(lengths), 4
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)
    s = cu(b.scores)
    trees = T.random_trees(b.lengths, b.n1, G, 5)
    with B.Plan(b.lengths, n1=b.n1, flags=flags, device=dev) as plan:
        trees[:, 3] = plan.cky_decode(s)[0].cpu().numpy()   # one of many times a tree's mean score
        lz, mu = orc.marginals(b.scores, b.lengths, threads=16)
        lp = T.log_probs(b.scores, b.lengths, trees, lz)
        free = W.valid_mask(np.asarray(lengths), b.n1)
        for k, n in enumerate(lengths):
            free[k, np.arange(n), np.arange(n) + 1] = free[k, 0, n] = False
        own = np.where(free, b.scores.astype(np.float64), 0.0)
        tree_free = np.array([[sum(own[k, i, j] for i, j in T.spans_of(t, n)) for t in trees[k]] for k, n in enumerate(lengths)])
        lp = lp + (CHART_SCORE - 1.0) * (tree_free - (np.where(free, mu, 0.0) * own).sum((1, 2))[:, None])
        old = lp.astype(np.float32)
        tol = (5.0 * np.sqrt(np.asarray(lengths)) * 2.0 ** -23)[:, None]
        got = plan.tree_logprobs(s, cu(trees))[0].cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - lp) <= tol + 2.0 ** -24 * np.abs(lp)), np.abs(got - lp).max(1)
        for g in range(G):   # (one tree at a time: its ratio is the loss)
            loss, _, _ = plan.policy_loss(s, cu(trees[:, g:g + 1]), -torch.ones((Bn, 1), device=dev), cu(old[:, g:g + 1]),
                                          clip_low=1.0, clip_high=1e6)
            err = np.log(loss.cpu().numpy().astype(np.float64)) - (lp[:, g] - old[:, g])
            assert np.all(np.abs(err) <= tol[:, 0] + 1.01 * 2.0 ** -24), (g, err, tol[:, 0])
