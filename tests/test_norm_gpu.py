"""Layer norm of rows and its backward pass on the GPU against their float64 form.

Tolerances, per entry, with u = 2^-24 (float32) and 2^-8 (bf16) of a rounding.
A row's sums are trees of at most 3 + 6 + 15 additions (eight entries of a lane,
64 lanes, 16 wavefronts one after the other), 24 u of the terms' absolute sum.
  m      off by at most e = 26 u mean|x|
  v      off by d e^2 / d (the deviations' common error; their sum is 0) and,
         of itself, 34 u (8 products more): r = 1 / sqrt(v + eps) by 22 u + e^2 r^2 / 2
  h      |h| (24 u + e^2 r^2 / 2) + (e + 2 u |x - m|) r            =: t
  y      |gamma| t + 3 u (|gamma h| + |beta|) + 2^-8 |y|, + 2^-133 (bf16's least)
  means  of U = dy gamma and U h: 27 u mean|U|, 27 u mean|U h| + mean(|U| t)
  dx     r (3 u |U| + e1 + |h| e2 + t |mean Uh| + 4 u (|mean U| + |h mean Uh|))
         + |dx| (24 u + e^2 r^2 / 2), + 2^-8 |dx| (bf16) or u |dx| (float32)
  dgamma sum |dy| t + (rows) u sum |dy h|;  dbeta (rows) u sum |dy|
Products of these are below a hundredth of them; tolerances take 1.01.
"""
import numpy as np
import pytest

from paper_2008_03736_amd import binding as B
from paper_2008_03736_amd import workloads as W

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch as _t

    if not _t.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load()
    return _t


def there(lengths, n1):
    return np.arange(n1)[None] <= np.asarray(lengths)[:, None]


def values(lengths, n1, d, seed, wide, offset=0.3):
    """(x as the device takes it, x in float64), NaN past the sentences."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((len(lengths), n1, d)) * np.exp(rng.standard_normal((len(lengths), n1, 1)))
    x += offset * rng.standard_normal((len(lengths), n1, 1))
    x[~there(lengths, n1)] = np.nan
    if wide:
        return x.astype(np.float32), x.astype(np.float32).astype(np.float64)
    bits = W.to_bf16(x.astype(np.float32))
    bits[~there(lengths, n1)] = 0x7FC0
    return bits, W.from_bf16(bits).astype(np.float64)


def device(torch, v):
    t = torch.from_numpy(v.view(np.int16) if v.dtype == np.uint16 else v).to("cuda:0")
    return t.view(torch.bfloat16) if v.dtype == np.uint16 else t


def statistics(x, eps):
    m = x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt(((x - m) ** 2).mean(-1, keepdims=True) + eps)
    e = 26 * U * np.abs(x).mean(-1, keepdims=True)
    off = 24 * U + 0.5 * (e * r) ** 2
    h = (x - m) * r
    return h, r, np.abs(h) * off + (e + 2 * U * np.abs(x - m)) * r, off


def check(got, want, tol):
    got, want, tol = (np.asarray(v, np.float64) for v in (got, want, tol))
    worst = np.max(np.abs(got - want) - 1.01 * tol)
    assert np.all(np.abs(got - want) <= 1.01 * tol), worst


def rounded(want, wide):
    return (U if wide else 2.0 ** -8) * np.abs(want) + (0 if wide else 2.0 ** -133)


LENGTHS = [1, 2, 30, 62, 63, 64, 70, 5]
N1 = 75


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("d", [4, 8, 100, 128, 132, 252, 260, 500, 512, 516, 1024, 1028, 2052, 4096, 4100, 8188, 8192])
def test_forward(torch, d, wide):
    lengths, n1 = (LENGTHS, N1) if d <= 2052 else ([3, 9], 11)
    raw, x = values(lengths, n1, d, d, wide)
    ok = there(lengths, n1)
    rng = np.random.default_rng(1)
    gamma, beta = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32), rng.standard_normal(d).astype(np.float32)
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        out = torch.full((len(lengths), n1, d), 3.0, dtype=torch.bfloat16, device="cuda:0")
        plan.layer_norm(device(torch, raw), device(torch, gamma), device(torch, beta), eps=1e-5, out=out)
        bare = plan.layer_norm(device(torch, raw))
    out, bare = out.float().cpu().numpy(), bare.float().cpu().numpy()
    assert np.all(out[~ok] == 3.0) and np.all(bare[~ok] == 0.0)
    h, _, t, _ = statistics(x[ok], float(np.float32(1e-5)))
    want = h * gamma + beta
    check(out[ok], want, np.abs(gamma) * t + 3 * U * (np.abs(gamma * h) + np.abs(beta)) + rounded(want, False))
    check(bare[ok], h, t + 3 * U * np.abs(h) + rounded(h, False))


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("d", [4, 12, 100, 128, 200, 256, 500, 508, 516, 1000, 1028, 2048, 3000, 4096, 5000, 8192])
def test_backward(torch, d, wide):
    lengths, n1 = (LENGTHS, N1) if d <= 2048 else ([3, 9], 11)
    raw, x = values(lengths, n1, d, d + 1, wide)
    ok = there(lengths, n1)
    rng = np.random.default_rng(2)
    gamma = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    bits, dy = values(lengths, n1, d, d + 2, False)
    eps = float(np.float32(1e-3))
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        args = (device(torch, raw), device(torch, gamma), device(torch, bits))
        fresh = torch.full(raw.shape, 3.0, dtype=torch.float32 if wide else torch.bfloat16, device="cuda:0")
        got = plan.layer_norm_bwd(*args, eps=eps, grad_x=fresh)
        again = plan.layer_norm_bwd(*args, eps=eps)
        some = [plan.layer_norm_bwd(*args, eps=eps, need=tuple(k == q for q in range(3)))[k] for k in range(3)]
        bare = plan.layer_norm_bwd(args[0], None, args[2], eps=eps)
        for a, b, c in zip(got, again, some):
            sel = torch.from_numpy(ok).to("cuda:0") if a.dim() == 3 else slice(None)
            assert torch.equal(a[sel], b[sel]) and torch.equal(b, c)
    got = [v.float().cpu().numpy() for v in got]
    assert np.all(got[0][~ok] == 3.0)
    for g, (dx, dg, db) in ((gamma, got), (np.ones(d), [v.float().cpu().numpy() for v in bare])):
        h, r, t, off = statistics(x[ok], eps)
        u = dy[ok] * g
        mean = lambda v: v.mean(-1, keepdims=True)
        s, q = mean(u), mean(u * h)
        want = r * (u - s - h * q)
        e1, e2 = 27 * U * mean(np.abs(u)), 27 * U * mean(np.abs(u * h)) + mean(np.abs(u) * t)
        tol = r * (3 * U * np.abs(u) + e1 + np.abs(h) * e2 + t * np.abs(q) + 4 * U * (np.abs(s) + np.abs(h * q)))
        check(dx[ok], want, tol + np.abs(want) * off + rounded(want, wide))
        rows = int(ok.sum())
        check(dg, (dy[ok] * h).sum(0), (np.abs(dy[ok]) * t).sum(0) + rows * U * np.abs(dy[ok] * h).sum(0))
        check(db, dy[ok].sum(0), rows * U * np.abs(dy[ok]).sum(0))


def test_large_offsets_and_constant_rows(torch):
    # a mean a thousand times the deviations; a row of one value (its
    # deviations are the mean's rounding, h at most e r)
    lengths, n1, d = [9], 10, 500
    raw, x = values(lengths, n1, d, 5, True, offset=1000.0)
    raw[0, 3], x[0, 3] = 7.25, 7.25
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        out = plan.layer_norm(device(torch, raw), eps=1e-5).float().cpu().numpy()
    h, _, t, _ = statistics(x, float(np.float32(1e-5)))
    check(out, h, t + 3 * U * np.abs(h) + rounded(h, False))


def corrected(x, eps):
    """h, r and their errors as statistics(), where the deviations' own mean is
    taken off them.  f0 = x - m^ is off by u |f0| from x - m less m^'s error e, and
    |f0| <= |x - m| + e; its mean, e but for 27 u mean|f0|, is taken off with one
    more rounding:
      D = x - m   off by 2.01 u |D| + 28 u (mean|D| + e)
      v           mean f0^2 (34 u of itself) less e^2, which has 2 e times 27 u
                  mean|f0|: by 34 u v + 90 u e (mean|D| + e)
    """
    m = x.mean(-1, keepdims=True)
    dev = np.abs(x - m)
    r = 1.0 / np.sqrt((dev ** 2).mean(-1, keepdims=True) + eps)
    e, size = 26 * U * np.abs(x).mean(-1, keepdims=True), dev.mean(-1, keepdims=True)
    off = 24 * U + 45 * U * e * (size + e) * r ** 2
    h = (x - m) * r
    return h, r, np.abs(h) * off + (2.01 * U * dev + 28 * U * (size + e)) * r, off


@pytest.mark.parametrize("d", [100, 128, 500, 1028, 8192])
@pytest.mark.parametrize("offset", [30.0, 1e3, 1e5])
def test_a_large_mean_costs_no_digits(torch, d, offset):
    # means far past the deviations, which float32 outputs show: dx and dgamma
    lengths, n1 = [9, 20], 22
    rng = np.random.default_rng(d)
    x = (rng.standard_normal((2, n1, d)) + offset * (1 + rng.random((2, n1, 1))) * rng.choice([-1, 1], (2, n1, 1))).astype(np.float32)
    bits, dy = values(lengths, n1, d, d + 2, False)
    gamma = (1 + 0.3 * rng.standard_normal(d)).astype(np.float32)
    eps, ok = float(np.float32(1e-5)), there(lengths, n1)
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        dx, dg, _ = (v.cpu().numpy() for v in plan.layer_norm_bwd(device(torch, x), device(torch, gamma), device(torch, bits)))
    h, r, t, off = corrected(x[ok].astype(np.float64), eps)
    u = dy[ok] * gamma
    mean = lambda v: v.mean(-1, keepdims=True)
    s, q = mean(u), mean(u * h)
    want = r * (u - s - h * q)
    e1, e2 = 27 * U * mean(np.abs(u)), 27 * U * mean(np.abs(u * h)) + mean(np.abs(u) * t)
    tol = r * (3 * U * np.abs(u) + e1 + np.abs(h) * e2 + t * np.abs(q) + 4 * U * (np.abs(s) + np.abs(h * q)))
    check(dx[ok], want, tol + np.abs(want) * off + rounded(want, True))
    check(dg, (dy[ok] * h).sum(0), (np.abs(dy[ok]) * t).sum(0) + int(ok.sum()) * U * np.abs(dy[ok] * h).sum(0))


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("d", [4, 12, 100, 164, 500, 508, 1028, 4100, 6212, 7132, 7684, 8052, 8188, 8192])
def test_rows_of_one_value(torch, d, wide):
    # deviations of 0, whatever the value up to 2^76: what the mean's rounding e leaves
    # of them is 27 u e once their mean is off, over the root of 2^-20 e^2 at least:
    # 2^-9.  (A row of zeros is exact.  The first values: with these d, sums of their
    # deviations over d are not their deviation.)
    sizes = 2.0 ** 76 * 10.0 ** -np.linspace(0, 60, 59)
    sizes[1:9:2] = 2.908594e16, 32087424000000.0, 2.4709912e20, 4.7043146e21
    lengths, n1 = [29, 29], 30
    x = np.zeros((2, n1, d), np.float32)
    x.reshape(60, d)[:59] = (sizes * np.where(np.arange(59) % 2, 1, -0.97))[:, None]
    raw = x if wide else W.to_bf16(x)
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        h = plan.layer_norm(device(torch, raw)).float().cpu().numpy()
        dy = torch.ones((2, n1, d), dtype=torch.bfloat16, device="cuda:0")
        dx, dg, db = (v.float().cpu().numpy() for v in plan.layer_norm_bwd(device(torch, raw), None, dy))
    assert np.all(np.abs(h) <= 2.0 ** -9) and np.all(h[1, 29] == 0)
    assert np.all(np.abs(dg) <= 60 * 2.0 ** -9) and np.all(db == 60) and np.isfinite(dx).all()


@pytest.mark.parametrize("scale", [1e-20, 1e-19, 1e-18])
def test_the_least_eps(torch, scale):
    # squares about float32's least normal number, which eps is: each square, their
    # mean and the square that is taken off it are off by 2^-150 at most, which is
    # 3 u / 2 of 1 / sqrt(v + eps) at v + eps >= 2^-126
    lengths, n1, d, eps = [9], 10, 500, 2.0 ** -126
    raw, _ = values(lengths, n1, d, 19, True, offset=0.0)
    raw = (raw * scale).astype(np.float32)
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        out = plan.layer_norm(device(torch, raw), eps=eps).float().cpu().numpy()
    h, _, t, _ = statistics(raw.astype(np.float64), eps)
    check(out, h, t + 5 * U * np.abs(h) + rounded(h, False))


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("d", [100, 252, 500, 1500])
def test_one_row_is_not_finite(torch, d, bad):
    raw, _ = values(LENGTHS, N1, d, 6, True)
    hurt = raw.copy()
    hurt[2, 7, d - 3] = bad
    bits, _ = values(LENGTHS, N1, d, 7, False)
    with B.Plan(LENGTHS, n1=N1, device="cuda:0") as plan:
        dy = device(torch, bits)
        clean, got = (plan.layer_norm(device(torch, v)) for v in (raw, hurt))
        back, sore = (plan.layer_norm_bwd(device(torch, v), None, dy, need=(True, False, True)) for v in (raw, hurt))
    for a, b in ((clean, got), (back[0], sore[0])):
        assert torch.isnan(b[2, 7]).all()
        b[2, 7] = a[2, 7]
        assert torch.equal(a, b)
    assert torch.equal(back[2], sore[2])


def test_squares_past_float32(torch):
    # finite entries whose squared deviations sum to more than float32 holds: the
    # row says so, the others are as without it
    raw, _ = values(LENGTHS, N1, 100, 16, True)
    hurt = raw.copy()
    hurt[2, 7, 3] = 1e25
    with B.Plan(LENGTHS, n1=N1, device="cuda:0") as plan:
        clean, got = (plan.layer_norm(device(torch, v)) for v in (raw, hurt))
    assert torch.isnan(got[2, 7]).all()
    got[2, 7] = clean[2, 7]
    assert torch.equal(clean, got)


def test_offsets_past_32_bits(torch):
    # 2.2e9 entries in all, 4.4 GB of bf16; the last sentence is checked
    lengths, n1, d = [1] * 549 + [1000], 1001, 4000
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    x = torch.zeros((550, n1, d), dtype=torch.bfloat16, device="cuda:0")
    assert x.numel() > 1 << 31
    raw, want = values([1000], n1, d, 17, False)
    bits, dy = values([1000], n1, d, 18, False)
    x[-1] = device(torch, raw)[0]
    up = torch.zeros_like(x)
    up[-1] = device(torch, bits)[0]
    eps = float(np.float32(1e-5))
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        y = plan.layer_norm(x)[-1].float().cpu().numpy()
        dx, dg, db = plan.layer_norm_bwd(x, None, up)
        dx = dx[-1].float().cpu().numpy()
    h, r, t, off = statistics(want[0], eps)
    check(y, h, t + 3 * U * np.abs(h) + rounded(h, False))
    mean = lambda v: v.mean(-1, keepdims=True)
    u = dy[0]
    s, q = mean(u), mean(u * h)
    e1, e2 = 27 * U * mean(np.abs(u)), 27 * U * mean(np.abs(u * h)) + mean(np.abs(u) * t)
    tol = r * (3 * U * np.abs(u) + e1 + np.abs(h) * e2 + t * np.abs(q) + 4 * U * (np.abs(s) + np.abs(h * q)))
    grad = r * (u - s - h * q)
    check(dx, grad, tol + np.abs(grad) * off + rounded(grad, False))
    rows = 1001 + 2 * 549
    check(db.cpu(), u.sum(0), rows * U * np.abs(u).sum(0))
    check(dg.cpu(), (u * h).sum(0), (np.abs(u) * t).sum(0) + rows * U * np.abs(u * h).sum(0))


def test_gradient_by_differences(torch):
    lengths, n1, d = [4, 2], 6, 24
    _, x = values(lengths, n1, d, 8, True, offset=0.0)
    ok = there(lengths, n1)
    rng = np.random.default_rng(3)
    gamma, beta = 1 + 0.3 * rng.standard_normal(d), rng.standard_normal(d)
    _, dy = values(lengths, n1, d, 9, False)

    def loss(x, gamma, beta):
        v = x[ok]
        v = v - v.mean(-1, keepdims=True)
        return ((v / np.sqrt((v * v).mean(-1, keepdims=True) + 1e-3) * gamma + beta) * dy[ok]).sum()

    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        t = [torch.from_numpy(np.nan_to_num(v).astype(np.float32)).to("cuda:0").requires_grad_() for v in (x, gamma, beta)]
        y = B.layer_norm(t[0], plan, t[1], t[2], eps=1e-3)
        y.backward(torch.from_numpy(np.nan_to_num(dy)).to("cuda:0").to(torch.bfloat16))
        got = [v.grad.cpu().numpy() for v in t]
        assert (got[0][~ok] == 0).all() and (y.detach().cpu().float().numpy()[~ok] == 0).all()
    # central differences at step s = 2^-9 in float64: their own error is s^2 / 6
    # of a third derivative, here below 100 of the gradient's size (eps keeps
    # 1 / r above 0.03): 1e-4 and float32's 1e-5 of it
    args, s = [np.nan_to_num(x), gamma, beta], 2.0 ** -9
    for k, a in enumerate(args):
        for at in [tuple(rng.integers(0, q) for q in a.shape) for _ in range(12)]:
            if k == 0 and not ok[at[:2]]:
                continue
            moved = [[v.copy() for v in args] for _ in range(2)]
            moved[0][k][at] += s
            moved[1][k][at] -= s
            want = (loss(*moved[0]) - loss(*moved[1])) / (2 * s)
            assert abs(got[k][at] - want) <= 2e-4 * np.abs(got[k]).max(), (k, at)


def test_streams_and_graphs(torch):
    lengths, n1, d = [3, 40, 66], 70, 500
    dev = torch.device("cuda", 0)
    xs = [device(torch, values(lengths, n1, d, k, False)[0]) for k in (1, 2)]
    dy = device(torch, values(lengths, n1, d, 3, False)[0])
    gamma = torch.rand(d, device=dev)
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        call = lambda x: (plan.layer_norm(x, gamma), *plan.layer_norm_bwd(x, gamma, dy))
        want = [call(x) for x in xs]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = call(xs[0])
        torch.cuda.current_stream().wait_stream(side)
        held, graphs = xs[0].clone(), []
        for _ in range(2):   # two graphs, each with its own workspace
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                graphs.append((g, call(held)))
        for k in (0, 1, 0):
            held.copy_(xs[k])
            for g, _ in graphs:
                g.replay()
            torch.cuda.synchronize()
            call(xs[1])
            for _, out in graphs:
                for a, b in zip(out, want[k]):
                    assert torch.equal(a, b)
        for a, b in zip(other, want[0]):
            assert torch.equal(a, b)


def test_batches_of_many_rows(torch):
    # more workgroups than shares of the sums; a benchmark batch's lengths
    batch = W.make("mixed")
    lengths, n1, d = np.tile(batch.lengths[:400], 2), int(batch.lengths[:400].max()) + 3, 100
    raw, x = values(lengths, n1, d, 11, False)
    bits, dy = values(lengths, n1, d, 12, False)
    ok = there(lengths, n1)
    with B.Plan(lengths, n1=n1, device="cuda:0") as plan:
        dx, dg, db = plan.layer_norm_bwd(device(torch, raw), None, device(torch, bits), eps=1e-5)
    h, _, t, _ = statistics(x[ok], float(np.float32(1e-5)))
    rows = int(ok.sum())
    check(dg.cpu(), (dy[ok] * h).sum(0), (np.abs(dy[ok]) * t).sum(0) + rows * U * np.abs(dy[ok] * h).sum(0))
    check(db.cpu(), dy[ok].sum(0), rows * U * np.abs(dy[ok]).sum(0))
    assert (dx.cpu().float().numpy()[~ok] == 0).all()


def test_refusals(torch):
    dev = torch.device("cuda", 0)
    with B.Plan([3, 5], n1=6, device=dev) as plan:
        x = lambda d, t=torch.bfloat16: torch.zeros((2, 6, d), dtype=t, device=dev)
        for d in (2, 6, 8196):
            with pytest.raises(B.CrfError, match="multiple of 4"):
                plan.layer_norm(x(d))
        for eps in (0.0, -1.0, float("nan"), float("inf")):
            with pytest.raises(B.CrfError, match="eps"):
                plan.layer_norm(x(8), eps=eps)
            with pytest.raises(B.CrfError, match="eps"):
                plan.layer_norm_bwd(x(8), None, x(8), eps=eps)
        with pytest.raises(ValueError):
            plan.layer_norm(x(8, torch.float16))
        with pytest.raises(ValueError):
            plan.layer_norm(x(16)[..., :8])
        with pytest.raises(ValueError):
            plan.layer_norm(x(8), gamma=torch.ones(7, device=dev))
        with pytest.raises(ValueError):
            plan.layer_norm_bwd(x(8), None, x(8, torch.float32))
        with pytest.raises(ValueError):
            plan.layer_norm_bwd(x(8, torch.float32), None, x(8), grad_x=x(8))
        v = x(8)
        with pytest.raises(B.CrfError, match="alias"):
            plan.layer_norm(v, out=v)
