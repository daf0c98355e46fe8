"""The biaffine scorer's backward pass on the GPU against its float64 form.

Tolerances, per entry.  A bf16 rounding is off by at most 2^-8 of the value, a
hi + lo pair by 2^-16, a float32 sum of K terms by K 2^-24 of the terms'
absolute sum (K below 64 blocks of posts or 512 here, and both).
  grad_w    (2 * 2^-16 + K 2^-24) sum |G| |r^l| |r^r|, K the posts plus 128
  grad_rl   the inner product, rounded to bf16 once: of sentences of up to 63
            words (G (R^r W^T)) V = R^r W^T, 2^-8 sum_j |G| |V_j|; of longer
            ones ((G R^r) W^T) U = G R^r, 2^-8 sum_c |U_c| |W_c|; + 2^-8 |result|
            (and the product of the two roundings, 2^-16)
            + (2^-16 + 2^-14) sum |G| |r^r| |W|
  grad_rr   the same with [r^l ; 1], V = [r^l ; 1] W and X = G^T [r^l ; 1]
A pass from the 8-bit form equals the one from the bf16 rows it stands for, bit
for bit: the codes become those rows before the first product.
"""
import numpy as np
import pytest

import tree_reference as T
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


def gradient(lengths, n1, L, seed):
    """float32 [B, N1, N1] (L = 1) or [B, N1, N1, L], NaN where no span is."""
    rng = np.random.default_rng(seed)
    shape = (len(lengths), n1, n1) + ((L,) if L > 1 else ())
    g = (rng.standard_normal(shape) * np.exp(2.0 * rng.standard_normal(shape))).astype(np.float32)
    g[~W.valid_mask(np.asarray(lengths), n1)] = np.nan
    return g


def reference(rl, rr, wt, lengths, g):
    """float64 (dR^l, dR^r, dW [l, c, a]) and the tolerances of each."""
    d, L = rl.shape[2], wt.shape[0]
    f = lambda x: W.from_bf16(x).astype(np.float64)
    w = f(wt)
    out = [np.zeros(rl.shape), np.zeros(rl.shape), np.zeros((L, d, d + 1))]
    tol = [np.zeros_like(x) for x in out]
    for b, n in enumerate(lengths):
        n = int(n)
        one, r = np.concatenate([f(rl[b, :n + 1]), np.ones((n + 1, 1))], 1), f(rr[b, :n + 1])
        for q in range(L):
            gq = np.nan_to_num((g[b, ..., q] if g.ndim == 4 else g[b])[:n + 1, :n + 1].astype(np.float64))
            gq = np.triu(gq, 1)
            u, x = gq @ r, gq.T @ one
            ua, xa = np.abs(gq) @ np.abs(r), np.abs(gq).T @ np.abs(one)
            wl, wa = w[q][:, :d], np.abs(w[q])
            out[0][b, :n + 1] += u @ wl
            out[1][b, :n + 1] += x @ w[q].T
            out[2][q] += u.T @ one
            if n <= 63:
                inner = np.abs(gq) @ np.abs(r @ wl), np.abs(gq).T @ np.abs(one @ w[q].T)
            else:
                inner = np.abs(u) @ wa[:, :d], np.abs(x) @ wa.T
            tol[0][b, :n + 1] += (2.0 ** -8 + 2.0 ** -16) * inner[0] + (2.0 ** -16 + 2.0 ** -14) * ua @ wa[:, :d]
            tol[1][b, :n + 1] += (2.0 ** -8 + 2.0 ** -16) * inner[1] + (2.0 ** -16 + 2.0 ** -14) * xa @ wa.T
            tol[2][q] += ua.T @ np.abs(one)
    tol[0] += 2.0 ** -8 * np.abs(out[0])
    tol[1] += 2.0 ** -8 * np.abs(out[1])
    tol[2] *= 2.0 ** -15 + (sum(int(n) + 1 for n in lengths) + 128) * 2.0 ** -24
    return out, tol


def tensors(torch, inp, ldw, n1):
    dev = torch.device("cuda", 0)
    d, L = inp.d, inp.num_labels
    w = np.full((L, d, ldw), 0x7FC0, np.uint16)   # NaN past the bias: not read
    w[:, :, :d + 1] = inp.wt
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).to(dev)
    return t(inp.rl), t(inp.rr), t(w)


def check(torch, lengths, d, L=1, ldw=None, seed=0, n1=None, packed=False, rows=None):
    inp = W.biaffine_inputs(lengths, d, labels=L, seed=seed, n1=n1)
    n1 = inp.n1
    ldw = ldw or (d + 4) // 4 * 4
    g = gradient(lengths, n1, L, seed + 1)
    dev = torch.device("cuda", 0)
    rl, rr, w = tensors(torch, inp, ldw, n1)
    gt = torch.from_numpy(g).to(dev)
    Bn = len(lengths)
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        def run(a, b):
            out = plan.biaffine_bwd(a, b, w, gt, grad_rl=torch.full((Bn, n1, d), 3.0, dtype=torch.bfloat16, device=dev),
                                    grad_rr=torch.full((Bn, n1, d), 3.0, dtype=torch.bfloat16, device=dev),
                                    grad_w=torch.full((L, d, ldw), 3.0, device=dev))
            torch.cuda.synchronize()
            return out
        if packed:
            pl, pr = plan.pack_rows(rl), plan.pack_rows(rr)
            rl, rr = (plan.unpack_rows(*p, d).view(torch.int16) for p in (pl, pr))
            for x, y in zip(run(pl, pr), run(rl, rr)):
                assert torch.equal(x, y)
            return
        got = run(rl, rr)
        again = run(rl, rr)
    for x, y in zip(got, again):
        assert torch.equal(x, y)   # a fixed order of sums
    keep = np.arange(Bn) if rows is None else np.asarray(rows)
    got = [x.float().cpu().numpy().astype(np.float64) for x in got]
    if rows is None:
        ref, tol = reference(inp.rl, inp.rr, inp.wt, lengths, g)
    else:   # a sample of sentences, and dW left out
        ref, tol = reference(inp.rl[keep], inp.rr[keep], inp.wt, np.asarray(lengths)[keep], g[keep])
    there = np.arange(n1)[None] <= np.asarray(lengths)[:, None]
    for k in range(2):
        assert np.all(got[k][~there] == 3.0)
        err, ok = np.abs(got[k][keep] - ref[k]), there[keep]
        assert np.all(err[ok] <= tol[k][ok] + 1e-30), (k, float((err[ok] / (tol[k][ok] + 1e-30)).max()))
    assert np.all(got[2][:, :, d + 1:] == 3.0)
    if rows is None:
        err = np.abs(got[2][:, :, :d + 1] - ref[2])
        assert np.all(err <= tol[2] + 1e-30), float((err / (tol[2] + 1e-30)).max())


@pytest.mark.parametrize("d", [4, 8, 28, 64, 100, 124, 128, 252, 256, 380, 384, 500, 508])
def test_span_scorer(torch, d):
    # packed blocks, sentences of a block and over several, an odd number of blocks
    check(torch, [1, 2, 5, 30, 62, 63, 64, 99, 130, 20, 7, 200], d, seed=d)


def test_one_word(torch):
    check(torch, [1], 100)


def test_one_sentence(torch):
    check(torch, [23], 500, seed=3)


@pytest.mark.parametrize("lengths", [[63], [64], [127], [128], [300], [1] * 40, [31] * 9 + [1023]])
def test_block_edges(torch, lengths):
    check(torch, lengths, 36, seed=len(lengths), n1=min(max(lengths) + 5, 1024))


@pytest.mark.parametrize("d,L,ldw", [(100, 3, None), (100, 26, 104), (64, 137, 68), (124, 2, 128), (128, 5, 136),
                                     (252, 4, None), (300, 3, None), (500, 2, 520), (4, 70, 8)])
def test_label_scorer(torch, d, L, ldw):
    check(torch, [3, 17, 40, 70, 1, 130], d, L=L, ldw=ldw, seed=d + L)


def test_label_groups(torch):
    # enough blocks that a workgroup takes several labels, in groups that do not divide them
    check(torch, [70, 61, 62, 63] * 6 + [130, 9], 36, L=29, seed=5, rows=[0, 1, 2, 24, 25])


def test_many_sentences(torch):
    m = W.make("mixed")
    check(torch, m.lengths[:1200], 100, seed=2, rows=np.argsort(-m.lengths[:1200])[:4].tolist() + [5, 600, 1199])


@pytest.mark.parametrize("d,L", [(100, 1), (36, 3), (500, 1), (260, 1), (252, 2), (4, 1)])
def test_packed_rows(torch, d, L):
    check(torch, [1, 9, 40, 66, 130, 63], d, L=L, seed=d, packed=True)


def test_some_gradients_only(torch):
    dev = torch.device("cuda", 0)
    lengths, d = [9, 70], 100
    inp = W.biaffine_inputs(lengths, d, seed=1)
    rl, rr, w = tensors(torch, inp, 104, inp.n1)
    g = torch.from_numpy(gradient(lengths, inp.n1, 1, 2)).to(dev)
    with B.Plan(lengths, n1=inp.n1, device=dev) as plan:
        every = plan.biaffine_bwd(rl, rr, w, g)
        for need in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
            got = plan.biaffine_bwd(rl, rr, w, g, need=need)
            for x, y, n in zip(got, every, need):
                assert torch.equal(x, y) if n else x is None


def test_fine_tuning_step(torch):
    # scores, candidates' log-probabilities, policy loss and the way back
    # through the scorer, from 8 bits: by autograd and by the calls, captured too
    dev = torch.device("cuda", 0)
    lengths, d, G = [5, 30, 64, 12], 100, 4
    inp = W.biaffine_inputs(lengths, d, seed=4)
    n1 = inp.n1
    bf = lambda x: torch.nan_to_num(x.view(torch.bfloat16)).requires_grad_(True)
    rl, rr, w = (bf(x) for x in tensors(torch, inp, 104, n1))
    trees = torch.from_numpy(T.random_trees(lengths, n1, G, 4)).to(dev)
    adv = torch.randn((4, G), device=dev, generator=torch.Generator(dev).manual_seed(1))
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        with torch.no_grad():
            old, _ = plan.tree_logprobs(B.biaffine(rl, rr, w, plan), trees)
            ref = old - 0.1
        scores = B.biaffine(rl, rr, w, plan, held="8bit")
        loss = B.policy_loss(scores, trees, adv, old, plan, ref_logp=ref, kl_coef=0.1)
        loss.sum().backward()

        def step(rl, rr, w):
            s = plan.biaffine_scores(*(x.view(torch.int16) for x in (rl, rr, w)),
                                     scores=torch.zeros((4, n1, n1), device=dev))
            kept = plan.pack_rows(rl), plan.pack_rows(rr)
            _, _, g = plan.policy_loss(s, trees, adv, old, ref_logp=ref, kl_coef=0.1)
            return plan.biaffine_bwd(*kept, w, g)
        r, q, v = rl.detach(), rr.detach(), w.detach()
        want = step(r, q, v)
        for x, y in zip((rl, rr, w), want):
            assert torch.equal(x.grad, y.to(torch.bfloat16))
        # ratios are 1 (old is the policy itself), so the trees' coefficients
        # are -adv/G less the KL term's slope
        held, graph = r.clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(held, q, v)
        half = step(r * 0.5, q, v)
        for k in (0, 1, 0):
            held.copy_(r if k == 0 else r * 0.5)
            graph.replay()
            torch.cuda.synchronize()
            step(r, q, v)
            for x, y in zip(out, want if k == 0 else half):
                assert torch.equal(x, y)


def test_refusals(torch):
    dev = torch.device("cuda", 0)
    lengths = [3, 5]
    with B.Plan(lengths, n1=6, device=dev) as plan:
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=dev)
        rl, rr, w, g = bf(2, 6, 8), bf(2, 6, 8), bf(1, 8, 12), torch.zeros((2, 6, 6), device=dev)
        with pytest.raises(B.CrfError, match="ldw"):
            plan.biaffine_bwd(rl, rr, bf(1, 8, 8), g)
        with pytest.raises(B.CrfError, match="multiple of 4"):
            plan.biaffine_bwd(bf(2, 6, 512), bf(2, 6, 512), bf(1, 512, 516), g)
        with pytest.raises(B.CrfError, match="alias"):
            plan.biaffine_bwd(rl, rr, w, g, grad_rl=rl)
        out = bf(2, 6, 8)
        with pytest.raises(B.CrfError, match="alias"):
            plan.biaffine_bwd(rl, rr, w, g, grad_rl=out, grad_rr=out)
        with pytest.raises(ValueError):
            plan.biaffine_bwd(rl, rr, w, g[:1])
        with pytest.raises(ValueError):
            plan.biaffine_bwd(rl.float(), rr, w, g)
        with pytest.raises(ValueError):
            plan.biaffine_bwd(plan.pack_rows(rl), rr, w, g)
        ws = plan._workspace(B.crf_biaffine_bwd_workspace(plan._handle, 8, 1))
        with pytest.raises(B.CrfError, match="workspace"):
            B.crf_biaffine_bwd(plan._handle, rl.data_ptr(), rr.data_ptr(), w.data_ptr(), 8, 12, 1, g.data_ptr(), None, None,
                               None, ws.data_ptr(), ws.numel() - 1, None)


@pytest.mark.parametrize("at", ["first", "last"])
def test_offsets_past_32_bits(torch, at):
    # a labelled gradient of more than 2^31 entries, all zero but for one
    # sentence; small integers, whose sums are exact, so that the bits are those
    # of that sentence alone
    dev = torch.device("cuda", 0)
    n1, n, d, L, Bn = 141, 20, 4, 138, 800
    assert Bn * n1 * n1 * L > 2 ** 31
    k = 0 if at == "first" else Bn - 1
    gen = torch.Generator(dev).manual_seed(3)
    ints = lambda *s: torch.randint(-2, 3, s, device=dev, generator=gen)
    rl, rr, w = (ints(*s).to(torch.bfloat16) for s in ((Bn, n1, d), (Bn, n1, d), (L, d, 8)))
    g = torch.zeros((Bn, n1, n1, L), device=dev)
    g[k] = ints(n1, n1, L)
    with B.Plan([n] * Bn, n1=n1, device=dev) as plan:
        got = plan.biaffine_bwd(rl, rr, w, g)
    one = slice(k, k + 1)
    with B.Plan([n], n1=n1, device=dev) as plan:
        want = plan.biaffine_bwd(rl[one].contiguous(), rr[one].contiguous(), w, g[one].contiguous())
    for x, y in zip(got[:2], want[:2]):
        assert torch.equal(x[one], y) and int(x.count_nonzero()) == int(y.count_nonzero()) > 0
    assert torch.equal(got[2], want[2])


def test_two_graphs_side_by_side(torch):
    # each with the workspace of its own pool, on streams of their own; eager
    # work between the replays
    dev = torch.device("cuda", 0)
    lengths, d = [70, 20, 33, 5], 252
    inp = W.biaffine_inputs(lengths, d, labels=2, seed=6)
    rl, rr, w = tensors(torch, inp, 256, inp.n1)
    g = torch.from_numpy(gradient(lengths, inp.n1, 2, 7)).to(dev)
    grads = [g, g * 0.5]
    with B.Plan(lengths, n1=inp.n1, device=dev) as plan:
        want = [plan.biaffine_bwd(rl, rr, w, x) for x in grads]
        graphs, outs = [], []
        for x in grads:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                outs.append(plan.biaffine_bwd(rl, rr, w, x))
            graphs.append(graph)
        streams = [torch.cuda.Stream() for _ in graphs]
        for _ in range(3):
            for s, graph in zip(streams, graphs):
                s.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(s):
                    graph.replay()
            for s in streams:
                torch.cuda.current_stream().wait_stream(s)
            plan.biaffine_bwd(rl, rr, w, grads[0])
            torch.cuda.synchronize()
            for out, y in zip(outs, want):
                for a, b in zip(out, y):
                    assert torch.equal(a, b)


@pytest.mark.parametrize("packed", [False, True])
def test_some_gradients_of_labelled_scores(torch, packed):
    # any of the three alone, and none: on another stream, from packed rows too
    dev = torch.device("cuda", 0)
    lengths, d, L = [9, 70, 1], 132, 3
    inp = W.biaffine_inputs(lengths, d, labels=L, seed=1)
    rl, rr, w = tensors(torch, inp, 136, inp.n1)
    g = torch.from_numpy(gradient(lengths, inp.n1, L, 2)).to(dev)
    side = torch.cuda.Stream()
    with B.Plan(lengths, n1=inp.n1, device=dev) as plan:
        if packed:
            rl, rr = plan.pack_rows(rl), plan.pack_rows(rr)
        every = plan.biaffine_bwd(rl, rr, w, g)
        for k in range(8):
            need = tuple(bool(k >> q & 1) for q in range(3))
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                got = plan.biaffine_bwd(rl, rr, w, g, need=need)
            torch.cuda.current_stream().wait_stream(side)
            for x, y, n in zip(got, every, need):
                assert torch.equal(x, y) if n else x is None


MANY = np.random.default_rng(17).integers(1, 62, 3000).tolist() + [140, 64, 99, 128, 127, 63] * 10
FEW = [40, 99, 3, 70, 61, 62, 63, 64, 30, 1] * 5


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("lengths,d,L", [(MANY, 100, 1), (MANY, 252, 1), (MANY, 500, 1), (MANY, 380, 1), (FEW, 36, 29),
                                         (FEW, 132, 130), (FEW, 60, 300)])
def test_weight_gradient_of_many_blocks(torch, lengths, d, L, packed):
    """dW over hundreds of shares of several blocks each, or one share of all
    (splits = 1: 130 labels at d = 132, 300 at d = 60), bit for bit.  Integers of
    at most 2: a post's U is below 2^16, which two bf16 parts hold, and the sums,
    of random signs, stay far below 2^24 (the assertion on the reference)."""
    dev = torch.device("cuda", 0)
    n1, Bn = max(lengths) + 1, len(lengths)
    gen = torch.Generator(dev).manual_seed(d + L)
    ints = lambda *s: torch.randint(-2, 3, s, device=dev, generator=gen)
    n = torch.tensor(lengths, device=dev)
    post = torch.arange(n1, device=dev)
    rows = post[None] <= n[:, None]
    spans = (post[:, None] < post[None])[None] & (post[None, None] <= n[:, None, None])
    rl, rr = (torch.where(rows[..., None], ints(Bn, n1, d), 0) for _ in range(2))
    nan = float("nan")
    held = [torch.where(rows[..., None], x.to(torch.bfloat16), nan) for x in (rl, rr)]
    g = torch.where(spans[..., None], ints(Bn, n1, n1, L).float(), nan)
    w = torch.full((L, d, (d + 4) // 4 * 4), nan, dtype=torch.bfloat16, device=dev)
    w[..., :d + 1] = 1.0
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        if packed:
            held = [plan.pack_rows(x) for x in held]
        got = plan.biaffine_bwd(*held, w, g if L > 1 else g[..., 0], need=(False, False, True))[2]
    one = torch.cat([rl, rows[..., None].long()], 2).double().reshape(-1, d + 1)
    for q in range(L):
        u = torch.bmm(torch.nan_to_num(g[..., q]).double().contiguous(), rr.double()).reshape(-1, d)
        want = u.t().contiguous() @ one
        assert float(want.abs().max()) < 2 ** 20
        assert torch.equal(got[q, :, :d + 1].double(), want), q


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("lengths", [[1, 2, 20, 30, 62, 63, 64, 99, 130, 200, 40, 300], [30, 41] * 250 + [80, 140]])
@pytest.mark.parametrize("d,L", [(28, 1), (100, 1), (124, 3), (252, 1), (252, 2), (380, 1), (380, 2), (500, 1), (500, 2)])
def test_row_gradients_are_rounded_once(torch, lengths, d, L, packed):
    """dR^l and dR^r are the bf16 numbers next to their float64 values: the inner
    product keeps two bf16 parts.  Integers, so that everything before the last
    rounding is exact: inner products are below 2^16 (two parts) but often above
    2^8 (one part), sums below 2^24."""
    dev = torch.device("cuda", 0)
    n1, Bn = max(lengths) + 1, len(lengths)
    gen = torch.Generator(dev).manual_seed(d + L)
    ints = lambda m, *s: torch.randint(-m, m + 1, s, device=dev, generator=gen)
    n, post = torch.tensor(lengths, device=dev), torch.arange(n1, device=dev)
    rows = post[None] <= n[:, None]
    spans = (post[:, None] < post[None])[None] & (post[None, None] <= n[:, None, None])
    rl, rr = (torch.where(rows[..., None], ints(8, Bn, n1, d), 0) for _ in range(2))
    held = [x.to(torch.bfloat16) for x in (rl, rr)]
    g = torch.where(spans[..., None], ints(3, Bn, n1, n1, L).float(), float("nan"))
    w = torch.zeros((L, d, (d + 4) // 4 * 4), dtype=torch.bfloat16, device=dev)
    w[..., :d + 1] = ints(4, L, d, d + 1)
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        if packed:
            held = [plan.pack_rows(x) for x in held]
        got = plan.biaffine_bwd(*held, w, g if L > 1 else g[..., 0], need=(True, True, False))
    one = torch.cat([rl, rows[..., None].long()], 2).double()
    want, inner = [torch.zeros((Bn, n1, d), dtype=torch.float64, device=dev) for _ in range(2)], 0.0
    for q in range(L):
        gq, wq = torch.nan_to_num(g[..., q]).double(), w[q, :, :d + 1].double()
        for k, (a, left, right) in enumerate(((gq, rr.double(), wq[:, :d]), (gq.transpose(1, 2).contiguous(), one, wq.t()))):
            v = (left.reshape(-1, left.shape[2]) @ right.contiguous()).reshape(Bn, n1, d)
            inner = max(inner, float(v.abs().max()), float(torch.bmm(a, left).abs().max()))
            want[k] += torch.bmm(a, v)
    assert 2 ** 8 < inner < 2 ** 16 and max(float(x.abs().max()) for x in want) < 2 ** 22
    for x, y in zip(got, want):
        assert torch.equal(x[rows].double(), y[rows].to(torch.bfloat16).double())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("d,L", [(4, 1), (28, 1), (100, 1), (124, 3), (252, 1), (252, 2), (380, 1), (380, 2), (500, 1), (508, 2),
                                 (60, 40)])
def test_a_sentence_that_is_not_finite_keeps_to_itself(torch, d, L, packed):
    """Infinities and NaN in one sentence's representations, at its ends, inside
    and in the last entries of rows: the rows of the others' gradients are
    unchanged, its own hold NaN, and dW has them in the entries that they enter."""
    dev = torch.device("cuda", 0)
    lengths = [20, 9, 13, 30, 1, 25, 62, 5, 63, 64, 100, 7, 18] * 2
    inp = W.biaffine_inputs(lengths, d, labels=L, seed=d)
    n1 = inp.n1
    rl, rr, w = tensors(torch, inp, (d + 4) // 4 * 4, n1)
    rl, rr, w = (x.view(torch.bfloat16) for x in (rl, rr, w))
    g = torch.from_numpy(gradient(lengths, n1, L, 3)).to(dev)
    there = (torch.arange(n1, device=dev)[None] <= torch.tensor(lengths, device=dev)[:, None])
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        rows = lambda x: plan.pack_rows(x) if packed else x
        call = lambda a, b: plan.biaffine_bwd(rows(a), rows(b), w, g)
        want = call(rl, rr)
        assert all(torch.isfinite(x[there]).all() for x in want[:2])
        for b, post, col, bad in ((0, 0, 0, "nan"), (1, 9, d - 1, "inf"), (2, 6, d // 2, "-inf"), (4, 1, d - 1, "nan"),
                                  (6, 62, 1, "nan"), (8, 63, d - 1, "inf"), (9, 64, 2, "nan"), (10, 70, d - 2, "nan"),
                                  (12, 0, d - 1, "inf"), (25, 18, 0, "nan")):
            for side in range(2):   # (dR^l comes from R^r, dR^r from R^l)
                x = [rl.clone(), rr.clone()]
                x[side][b, post, col] = float(bad)
                got = call(*x)
                others = [k for k in range(len(lengths)) if k != b]
                assert torch.equal(got[side], want[side])
                assert torch.equal(got[1 - side][others], want[1 - side][others]), (b, side)
                if not (post == 0 and side) and not (post == lengths[b] and not side):   # (which no span has on that side)
                    assert torch.isnan(got[1 - side][b, :lengths[b] + 1]).any(), (b, side)
                k = slice(None), (col if side else slice(None)), (slice(None, d + 1) if side else col)
                keep = torch.ones_like(got[2], dtype=torch.bool)
                keep[k] = False
                assert torch.equal(got[2][keep], want[2][keep]), (b, side)
        for b, i, j, bad in ((0, 0, 1, "nan"), (3, 0, 30, "inf"), (6, 61, 62, "nan"), (10, 3, 99, "nan")):
            h = g.clone()   # (a span's gradient)
            h[b, i, j] = float(bad)
            got = plan.biaffine_bwd(rows(rl), rows(rr), w, h)
            others = [k for k in range(len(lengths)) if k != b]
            for side, post in ((0, i), (1, j)):
                assert torch.equal(got[side][others], want[side][others])
                assert not torch.isfinite(got[side][b, post]).all()
