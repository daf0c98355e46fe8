"""Layer norm, the scorer with its width bias, the CRF's loss and the weights'
update as a training step runs them, on the GPU: the scorer with the bias equals
the scorer and then the bias bit for bit, a step through autograd equals the
calls one by one bit for bit (each of them is held to float64 by its own tests),
the loss' gradient by the table is that of the oracle's marginals, and the whole
step is captured and replayed."""
import numpy as np
import pytest

from oracle import oracle as orc
from paper_2008_03736_amd import binding as B
from paper_2008_03736_amd import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as _t

    if not _t.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load()
    return _t


def bf16(torch, *shape, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(shape, generator=g)).bfloat16().to("cuda:0")


@pytest.mark.parametrize("lengths,n1", [([1], 2), ([62, 63, 64, 65, 1, 5, 30], 70), ([200, 3, 130], 203), ([20] * 90, 21)])
@pytest.mark.parametrize("d,L", [(4, 1), (100, 1), (100, 3), (124, 40), (128, 1), (252, 5), (500, 1), (500, 9)])
def test_scorer_with_a_bias(torch, lengths, n1, d, L):
    ldw = (d + 8) // 8 * 8
    rl, rr, w = bf16(torch, len(lengths), n1, d), bf16(torch, len(lengths), n1, d, seed=1), bf16(torch, L, d, ldw, seed=2)
    v = lambda x: x.view(torch.int16)
    rng = np.random.default_rng(d + L)
    K = 7
    table = torch.from_numpy(rng.standard_normal((K, L)).astype(np.float32)).to("cuda:0")
    buckets = torch.from_numpy(rng.integers(-2, K + 2, n1).astype(np.int32)).to("cuda:0")
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        plain = plan.biaffine_scores(v(rl), v(rr), v(w))
        want = plan.width_bias(plain, table, buckets, out=torch.full_like(plain, 5.0))
        got = plan.biaffine_scores(v(rl), v(rr), v(w), scores=torch.full_like(plain, 5.0), table=table, buckets=buckets)
    assert torch.equal(got, want)
    valid = W.valid_mask(np.asarray(lengths), n1)
    assert (got.cpu().numpy()[~valid] == 5.0).all() and np.isfinite(got.cpu().numpy()).all()


def gold_trees(lengths, n1, seed):
    """Random binary trees, rows of (i, j) and then -1."""
    rng = np.random.default_rng(seed)
    out = np.full((len(lengths), 2 * (n1 - 1) - 1, 2), -1, np.int32)
    for b, n in enumerate(lengths):
        stack, r = [(0, n)], 0
        while stack:
            i, j = stack.pop()
            out[b, r] = i, j
            r += 1
            if j - i > 1:
                k = int(rng.integers(i + 1, j))
                stack += [(k, j), (i, k)]
    return out


LENGTHS, N1, D, K = [5, 1, 23, 40, 64, 70, 9], 72, 100, 8


class Step:
    """The parameters of a scorer and one training step on a batch."""

    def __init__(self, torch, plan, seed=0):
        self.torch, self.plan = torch, plan
        self.x = torch.randn((plan.B, N1, D), generator=torch.Generator().manual_seed(seed)).to("cuda:0")
        self.gamma = torch.ones(D, device="cuda:0")
        self.beta = torch.zeros(D, device="cuda:0")
        self.w = 0.1 * torch.randn((1, D, 104), generator=torch.Generator().manual_seed(seed + 1)).to("cuda:0")
        self.table = torch.zeros((K, 1), device="cuda:0")
        self.buckets = torch.from_numpy(B.width_buckets(N1, K, 32)).to("cuda:0")
        self.gold = torch.from_numpy(gold_trees(LENGTHS, N1, seed)).to("cuda:0")
        self.momentum = torch.zeros_like(self.w)
        self.leaves = (self.x, self.gamma, self.beta, self.w, self.table)

    def by_calls(self):
        """Gradients of the summed loss, call by call: (loss, x, gamma, beta, w, table)."""
        t, p = self.torch, self.plan
        y = p.layer_norm(self.x, self.gamma, self.beta)
        w = self.w.to(t.bfloat16)
        scores = t.zeros((p.B, N1, N1), device="cuda:0")
        p.biaffine_scores(y.view(t.int16), y.view(t.int16), w.view(t.int16), scores=scores, table=self.table,
                          buckets=self.buckets)
        loss, g = p.gold_loss(scores, self.gold)
        gl, gr, gw = p.biaffine_bwd(y, y, w, g)
        _, gt = p.width_bias_bwd(g, self.buckets, K, need=(False, True))
        return (loss, *p.layer_norm_bwd(self.x, self.gamma, gl + gr), gw, gt), scores

    def by_autograd(self):
        t, p = self.torch, self.plan
        leaves = [v.detach().clone().requires_grad_() for v in self.leaves]
        x, gamma, beta, w, table = leaves
        y = B.layer_norm(x, p, gamma, beta)
        scores = B.biaffine(y, y, w, p, table=table, buckets=self.buckets)
        trees = self.gold[:, None].contiguous()
        loss = -B.tree_log_prob(scores, trees, p)[:, 0]
        loss.sum().backward()
        return loss.detach(), [v.grad for v in leaves], scores.detach()

    def update(self, grads):
        B.muon_step(self.w, grads[4], self.momentum, lr=0.02, cols=D + 1)
        for v, g in ((self.gamma, grads[2]), (self.beta, grads[3]), (self.table, grads[5])):
            v.sub_(0.05 * g)


def test_autograd_is_the_calls(torch):
    with B.Plan(LENGTHS, n1=N1, device="cuda:0") as plan:
        s = Step(torch, plan)
        s.table.copy_(torch.linspace(-1, 1, K)[:, None])
        grads, scores = s.by_calls()
        loss, auto, auto_scores = s.by_autograd()
    valid = torch.from_numpy(W.valid_mask(np.asarray(LENGTHS), N1)).to("cuda:0")
    assert torch.equal(auto_scores[valid], scores[valid])
    # two ways to one loss and one gradient: log Z and the trees' sums in float64
    # and in float32 (4 n roundings of sums below 400), marginals by the same sweep
    assert torch.all((loss - grads[0]).abs() <= 4 * 140 * 2.0 ** -24 * 400)
    for name, a, b in zip(("x", "gamma", "beta", "w", "table"), auto, grads[1:]):
        # (the gradient by the scores through either loss differs by float32
        # roundings of marginals, 1e-6 at most, and then by bf16's of rows)
        assert torch.allclose(a, b, rtol=2.0 ** -7, atol=2e-3 * float(b.abs().max())), name


def test_table_gradient_is_the_marginals(torch):
    with B.Plan(LENGTHS, n1=N1, device="cuda:0") as plan:
        s = Step(torch, plan, seed=3)
        (loss, *_, gt), scores = s.by_calls()
    v = W.valid_mask(np.asarray(LENGTHS), N1)
    sc = scores.cpu().numpy()
    lz, mu = orc.marginals(sc, np.asarray(LENGTHS), threads=8)
    gold = s.gold.cpu().numpy()
    for b in range(len(LENGTHS)):
        for i, j in gold[b]:
            if i >= 0:
                mu[b, i, j] -= 1.0
    k = s.buckets.cpu().numpy()[np.maximum(np.arange(N1)[None] - np.arange(N1)[:, None], 0)]
    k = np.broadcast_to(k[None], v.shape)
    for q in range(K):
        mine = mu[v & (k == q)]
        # marginals are within 1e-4 of the oracle's, as the parity tests hold them
        assert abs(float(gt[q, 0]) - mine.sum()) <= 1e-4 * len(mine) + 1e-6


def test_captured_step(torch):
    with B.Plan(LENGTHS, n1=N1, device="cuda:0") as plan:
        eager, held = Step(torch, plan, seed=5), Step(torch, plan, seed=5)

        def one(s):
            grads, _ = s.by_calls()
            s.update(grads)
            return grads[0]

        one(held)   # (the libraries' first calls)
        held = Step(torch, plan, seed=5)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            loss = one(held)
        for v, w in zip(held.leaves, eager.leaves):   # (capturing runs nothing)
            assert torch.equal(v, w)
        seen = []
        for k in range(4):
            new = torch.randn((plan.B, N1, D), generator=torch.Generator().manual_seed(50 + k)).to("cuda:0")
            for s in (eager, held):
                s.x.copy_(new)
            graph.replay()
            want = one(eager)
            torch.cuda.synchronize()
            assert torch.equal(loss, want)
            for v, w in zip((*held.leaves, held.momentum), (*eager.leaves, eager.momentum)):
                assert torch.equal(v, w)
            seen.append(float(loss.sum()))
        assert np.isfinite(seen).all() and len(set(seen)) == 4


def test_captured_autograd(torch):
    # forward and backward through the differentiable forms in one graph; no eager
    # graph of its leaves is alive meanwhile (torch would add to their gradients
    # on that one's stream)
    with B.Plan(LENGTHS, n1=N1, device="cuda:0") as plan:
        s = Step(torch, plan, seed=7)

        def run(leaves):
            for v in leaves:
                v.grad = None
            x, gamma, beta, w, table = leaves
            y = B.layer_norm(x, plan, gamma, beta)
            scores = B.width_bias(B.biaffine(y, y, w, plan, table=table, buckets=s.buckets), table, s.buckets, plan)
            loss, g = plan.gold_loss(scores.detach(), s.gold)
            scores.backward(g)
            return loss

        held = [v.clone().requires_grad_() for v in s.leaves]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(held)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            loss = run(held)
        for k in range(3):
            with torch.no_grad():
                held[0].copy_(torch.randn((plan.B, N1, D), generator=torch.Generator().manual_seed(60 + k)))
                held[4].fill_(0.1 * k)
            graph.replay()
            eager = [v.detach().clone().requires_grad_() for v in held]
            want = run(eager)
            torch.cuda.synchronize()
            assert torch.equal(loss, want)
            for v, w in zip(held, eager):
                assert torch.equal(v.grad, w.grad) and bool(v.grad.abs().sum() > 0)


def test_second_derivatives_raise(torch):
    with B.Plan([3], n1=4, device="cuda:0") as plan:
        x = torch.randn((1, 4, 8), device="cuda:0", requires_grad=True)
        y = B.layer_norm(x, plan)
        (g,) = torch.autograd.grad(y.float().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            g.sum().backward()


def test_only_the_table_is_trained(torch):
    lengths, n1, d = [6, 3], 7, 8
    rl, w = bf16(torch, 2, n1, d), bf16(torch, 1, d, 12, seed=1)
    table = torch.zeros((2, 1), device="cuda:0", requires_grad=True)
    buckets = torch.tensor([0, 0, 0, 1, 1, 1, 1], dtype=torch.int32, device="cuda:0")
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        B.biaffine(rl, rl, w, plan, table=table, buckets=buckets).sum().backward()
        with pytest.raises(ValueError):
            B.biaffine(rl, rl, w, plan, table=table)
        with pytest.raises(ValueError):
            plan.biaffine_scores(rl.view(torch.int16), rl.view(torch.int16), w.view(torch.int16), table=table,
                                 buckets=buckets[:3])
    # spans of width 1 and 2, and of 3 and more
    assert table.grad[:, 0].tolist() == [6 + 5 + 3 + 2, 4 + 3 + 2 + 1 + 1]
