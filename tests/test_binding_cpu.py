"""The differentiable forms around a stand-in plan, on the CPU: what they keep
for the backward pass and what they refuse.  (The stand-in computes nothing;
what it is handed is what is checked.)"""
import pytest
import torch

from paper_2008_03736_amd import binding as B


class StandIn:
    """The Plan methods that the differentiable forms call, on CPU tensors."""
    B, n1 = 2, 4

    def tree_logprobs(self, scores, trees, counts=None):
        return torch.zeros(trees.shape[:2]), None

    def tree_logprobs_bwd(self, scores, trees, grad_logp, counts=None):
        self.seen = trees.clone(), None if counts is None else counts.clone()
        return torch.zeros_like(scores)


def bare_plan(monkeypatch, *raw):
    """A Plan without a library handle whose raw entry points `raw` do nothing."""
    plan = object.__new__(B.Plan)
    plan._torch, plan.device, plan._handle = torch, torch.device("cpu"), None
    plan.B, plan.n1, plan.L = 2, 4, 1
    monkeypatch.setattr(B, "_stream_ptr", lambda *a: 0)
    for name in raw:
        monkeypatch.setattr(B, name, lambda *a: None)
    return plan


@pytest.mark.parametrize("which", ["trees", "counts"])
def test_trees_rewritten_before_the_backward_pass(which):
    # the gradient is that of the trees of the forward pass, or it is refused
    scores = torch.zeros((2, 4, 4), requires_grad=True)
    kept = dict(trees=torch.zeros((2, 3, 5, 2), dtype=torch.int32), counts=torch.tensor([3, 2], dtype=torch.int32))
    plan = StandIn()
    B.tree_log_prob(scores, kept["trees"], plan, counts=kept["counts"]).sum().backward()
    assert torch.equal(plan.seen[0], kept["trees"]) and torch.equal(plan.seen[1], kept["counts"])
    logp = B.tree_log_prob(scores, kept["trees"], plan, counts=kept["counts"])
    kept[which].add_(1)
    with pytest.raises(RuntimeError, match="inplace"):
        logp.sum().backward()


@pytest.mark.parametrize("call", ["cky_decode", "parse", "mbr_decode"])
def test_library_calls_count_as_rewriting(monkeypatch, call):
    # a buffer of trees that a later decode fills again
    plan = bare_plan(monkeypatch, "crf_cky_decode", "crf_inside_fwd_bwd_cky", "crf_mbr_decode")
    scores = torch.zeros((2, 4, 4), requires_grad=True)
    buf = torch.zeros((2, 5, 2), dtype=torch.int32)
    logp = B.tree_log_prob(scores, buf[:, None], StandIn())
    getattr(plan, call)(scores.detach(), spans=buf)
    with pytest.raises(RuntimeError, match="inplace"):
        logp.sum().backward()


def test_scores_that_the_scorer_fills_again(monkeypatch):
    plan = bare_plan(monkeypatch, "crf_biaffine_scores")
    scores = torch.zeros((2, 4, 4), requires_grad=True)
    logp = B.tree_log_prob(scores, torch.zeros((2, 1, 5, 2), dtype=torch.int32), StandIn())
    x, w = torch.zeros((2, 4, 8), dtype=torch.int16), torch.zeros((1, 8, 12), dtype=torch.int16)
    plan.biaffine_scores(x, x, w, scores=scores.detach())
    with pytest.raises(RuntimeError, match="inplace"):
        logp.sum().backward()


def test_inference_buffers_are_taken(monkeypatch):
    plan = bare_plan(monkeypatch, "crf_cky_decode")
    with torch.inference_mode():
        buf = torch.zeros((2, 5, 2), dtype=torch.int32)
        assert plan.cky_decode(torch.zeros((2, 4, 4)), spans=buf)[0] is buf
    assert plan.cky_decode(torch.zeros((2, 4, 4)), spans=buf)[0] is buf


class Scorer:
    """A plan that only counts what biaffine hands it."""
    B, n1 = 2, 4

    def __init__(self):
        self.packed = self.scored = 0

    def biaffine_scores(self, rl, rr, w, scores=None):
        self.scored += 1

    def pack_rows(self, x):
        self.packed += 1
        return x.clone(), x.clone()

    def biaffine_bwd(self, rl, rr, w, g, need=None):
        return torch.zeros((2, 4, 8)), torch.zeros((2, 4, 8)), torch.zeros(w.shape)


def rows_and_w(dtype=torch.bfloat16):
    return (torch.zeros((2, 4, 8), dtype=dtype), torch.zeros((2, 4, 8), dtype=dtype),
            torch.zeros((1, 8, 12), dtype=torch.bfloat16))


@pytest.mark.parametrize("held", ["bf16", "8bit"])
@pytest.mark.parametrize("at", [0, 1, 2])
def test_representations_of_another_type(held, at):
    # 16 bits of another kind would be read as bf16 (its bit patterns are taken)
    args = list(rows_and_w())
    plan = Scorer()
    B.biaffine(*args, plan, held=held)
    args[at] = args[at].view(torch.int16)
    B.biaffine(*args, plan, held=held)
    assert plan.scored == 2
    args[at] = args[at].view(torch.float16)
    with torch.no_grad(), pytest.raises(ValueError, match="bfloat16"):
        B.biaffine(*args, plan, held=held)
    assert plan.scored == 2


def test_rows_are_packed_only_for_a_backward_pass():
    plan = Scorer()
    rl, rr, w = rows_and_w()
    B.biaffine(rl, rr, w, plan, held="8bit")                       # nothing needs a gradient
    with torch.no_grad():
        B.biaffine(rl.clone().requires_grad_(True), rr, w, plan, held="8bit")
    assert plan.packed == 0 and plan.scored == 2
    for args in ((rl.clone().requires_grad_(True), rr, w), (rl, rr, w.clone().requires_grad_(True))):
        B.biaffine(*args, plan, held="8bit").sum().backward()
    assert plan.packed == 4


class Loss:
    """A plan whose log Z and losses are functions of the scores' sums."""
    B, n1 = 2, 4

    def inside_fwd(self, s):
        return s.sum((1, 2)) ** 3

    def inside_bwd(self, s, grad_logZ=None):
        return (3 * s.sum((1, 2)) ** 2 * grad_logZ)[:, None, None].expand_as(s).contiguous()

    def tree_logprobs(self, s, trees, counts=None):
        return (s.sum((1, 2)) ** 3)[:, None].expand(trees.shape[:2]).contiguous(), None

    def tree_logprobs_bwd(self, s, trees, g, counts=None):
        return self.inside_bwd(s, grad_logZ=g.sum(1))

    def policy_loss(self, s, trees, *args, **kw):
        return s.sum((1, 2)) ** 3, None, self.inside_bwd(s, grad_logZ=torch.ones(2))


@pytest.mark.parametrize("form", ["log_partition", "tree_log_prob", "policy_loss", "biaffine"])
def test_second_derivatives_are_refused(form):
    # (silently left out of them else: the gradients are no functions of the
    # scores to autograd)
    s = torch.ones((2, 4, 4), requires_grad=True)
    trees = torch.zeros((2, 1, 5, 2), dtype=torch.int32)
    if form == "biaffine":
        x = rows_and_w()
        leaf = x[0].clone().requires_grad_(True)
        out = B.biaffine(leaf, *x[1:], Scorer())
    else:
        leaf = s
        out = {"log_partition": lambda: B.log_partition(s, Loss()),
               "tree_log_prob": lambda: B.tree_log_prob(s, trees, Loss()),
               "policy_loss": lambda: B.policy_loss(s, trees, None, None, Loss())}[form]()
    (g,) = torch.autograd.grad(out.sum() ** 2, leaf, create_graph=True)   # the gradient itself is there
    with pytest.raises(RuntimeError, match="differentiate twice"):
        (g.sum() + leaf.sum()).backward()


def test_float32_w_gets_the_float32_gradient():
    third = torch.full((1, 8, 12), 1.0 / 3.0)

    class Thirds(Scorer):
        def biaffine_scores(self, rl, rr, w, scores=None):
            self.w = w.view(torch.bfloat16)

        def biaffine_bwd(self, rl, rr, w, g, need=None):
            assert w.dtype == torch.bfloat16
            return None, None, third

    rl, rr, _ = rows_and_w()
    for held in ("bf16", "8bit"):
        plan, w = Thirds(), (third + 1.0).requires_grad_(True)
        B.biaffine(rl, rr, w, plan, held=held).sum().backward()
        assert torch.equal(plan.w, w.detach().to(torch.bfloat16))   # the products' operand
        assert w.grad.dtype == torch.float32 and torch.equal(w.grad, third)
        w = third.to(torch.bfloat16).requires_grad_(True)
        B.biaffine(rl, rr, w, plan, held=held).sum().backward()
        assert w.grad.dtype == torch.bfloat16 and torch.equal(w.grad, third.to(torch.bfloat16))
