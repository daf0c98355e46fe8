"""Orthogonalised matrices and the update of weights by them, on the GPU,
against the products in float64.

Tolerance, of the 2-norm of all of a matrix's entries.  One step's local error is
eta |X|_F (|a| + 3 |b| s^2 + 5 |c| s^4), s the largest singular value, a term a
factor of each of the polynomial's monomials; eta is what a product loses of its
operands: 2^-20 for their parts (2^-22 each, and lo lo) and a float32 sum of K
terms whose roundings have independent signs, 4 deviations of 2^-24 sqrt(K).
Later steps multiply an error by at most the largest slope of their polynomials
on the singular values' range (a function of singular values has in this norm the
Lipschitz constant of the function of numbers).
Precision: an operand's parts are off by at most 2^-23 of its binade (float32:
2^-24) and lo lo is at most 2^-22 of a product, 2^-21 in all against float32's
2^-23 of its two operands: the error is at most four times that of the same
products in float32 (numpy's); and, where eps rules, what the steps make of
2^-37 an entry: parts are whole multiples of 2^-24 / 4096.  That compares what
roundings did and not their bounds, which says something only where many of
them add up: float32's can all but vanish by chance in a matrix of a few entries
(1 x 1 at x = 0.99978: 1.1e-7, the parts 1.8e-6, the bounds above 4e-5 and
1e-5).  It is asked of matrices of 1024 entries and more.
"""
import numpy as np
import pytest

from paper_2008_03736_amd import binding as B

pytestmark = pytest.mark.gpu
CUBIC = ((1.5, -0.5, 0.0),) * 4
FIFTH = ((15 / 8, -10 / 8, 3 / 8),) * 3


@pytest.fixture(scope="module")
def torch():
    import torch as _t

    if not _t.cuda.is_available():
        pytest.fail("GPU tests need a ROCm device")
    B.load()
    return _t


def matrices(count, rows, cols, ld, seed):
    rng = np.random.default_rng(seed)
    k = min(rows, cols, 8)
    x = rng.standard_normal((count, rows, k)) * np.exp(-0.3 * np.arange(k)) @ rng.standard_normal((count, k, ld))
    return (1e-3 * (x + 0.5 * rng.standard_normal((count, rows, ld)))).astype(np.float32)


def products(u, steps, eps, dtype):
    """Of one matrix, in dtype (the norm in float64)."""
    y = (u.astype(np.float64) / (np.linalg.norm(u.astype(np.float64)) + eps)).astype(dtype)
    tall = y.shape[0] > y.shape[1]
    y = y.T.copy() if tall else y
    for a, b, c in np.asarray(steps, dtype=np.float32).astype(dtype):
        gram = y @ y.T
        y = a * y + (b * gram + c * (gram @ gram)) @ y
    return y.T if tall else y


def tolerance(u, steps, eps):
    y = u.astype(np.float64) / (np.linalg.norm(u.astype(np.float64)) + eps)
    s = np.linalg.svd(y, compute_uv=False)
    top, size, off = 1.0, 1.0, 2.0 ** -22
    for a, b, c in np.asarray(steps, np.float32).astype(np.float64):
        t = np.linspace(0, top, 20001)
        slope = np.abs(a + 3 * b * t ** 2 + 5 * c * t ** 4).max()
        eta = 2.0 ** -20 + 4 * np.sqrt(max(u.shape)) * 2.0 ** -24
        high = s.max()
        off = off * slope + eta * size * (abs(a) + 3 * abs(b) * high ** 2 + 5 * abs(c) * high ** 4)
        s = np.abs(a * s + b * s ** 3 + c * s ** 5)
        top, size = np.abs(a * t + b * t ** 3 + c * t ** 5).max(), np.linalg.norm(s)
    return off


def check(got, u, steps, eps):
    want = products(u, steps, eps, np.float64)
    off = np.linalg.norm(got.astype(np.float64) - want)
    assert off <= tolerance(u, steps, eps), (off, tolerance(u, steps, eps))
    if u.size < 1024:
        return
    plain = np.linalg.norm(products(u, steps, eps, np.float32).astype(np.float64) - want)
    grown = np.prod([max(1.0, np.abs(a)) for a, _, _ in steps])
    assert off <= 4 * plain + 2.0 ** -24 * np.linalg.norm(want) + grown * 2.0 ** -37 * np.sqrt(u.size), (off, plain)


SHAPES = [(1, 1, 1, 1), (1, 1, 9, 9), (2, 9, 1, 3), (3, 2, 3, 5), (1, 15, 16, 16), (2, 16, 17, 20), (5, 31, 33, 33),
          (3, 33, 31, 40), (2, 64, 64, 64), (3, 63, 65, 68), (7, 100, 101, 104), (2, 101, 100, 100),
          (2, 112, 128, 128), (2, 128, 128, 130), (2, 128, 129, 132), (1, 129, 127, 127), (2, 40, 300, 304),
          (1, 300, 40, 41), (1, 7, 1000, 1000), (1, 500, 501, 504), (1, 512, 512, 512), (1, 513, 260, 263),
          (1, 700, 1030, 1030), (40, 20, 130, 130), (9, 200, 300, 300), (3, 1, 1024, 1024), (1, 9, 1200, 1200),
          (2, 2048, 16, 19), (1, 5, 2049, 2049), (4, 11, 385, 385), (3, 700, 13, 13), (2, 3, 17, 17),
          (2, 16, 1007, 1007), (2, 1024, 15, 17), (2, 17, 513, 513), (3, 32, 500, 500), (2, 257, 31, 31),
          (2, 48, 400, 401), (1, 417, 48, 48), (2, 64, 256, 256), (2, 64, 257, 257), (1, 80, 241, 241),
          (2, 190, 95, 95), (2, 112, 160, 160), (1, 112, 161, 161), (2, 128, 129, 129), (1, 2, 8192, 8192),
          (1, 1537, 1030, 1030), (3, 1025, 1290, 1290)]


@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalize(torch, shape):
    count, rows, cols, ld = shape
    x = matrices(count, rows, cols, ld, rows)
    x[:, :, cols:] = np.nan
    dev = torch.from_numpy(x).to("cuda:0")
    out = torch.full(x.shape, 3.0, device="cuda:0")
    assert B.orthogonalize(dev, cols=cols, out=out) is out
    again = B.orthogonalize(dev, cols=cols)
    got = out.cpu().numpy()
    assert (got[:, :, cols:] == 3.0).all() and (again[:, :, cols:] == 0).all()
    assert torch.equal(again[:, :, :cols], out[:, :, :cols])
    for q in range(count):
        check(got[q, :, :cols], x[q, :, :cols], B.MUON_STEPS, float(np.float32(1e-7)))


# Matrices of which there are enough for each of the tiles: pp (the shorter side, padded)
# a multiple of 128 with qq an odd and an even number of 64s, and pp an odd one.
MANY = [(138, 100, 300), (160, 128, 192), (64, 200, 300), (43, 256, 320), (22, 384, 448), (13, 512, 576),
        (128, 300, 120), (42, 256, 320), (43, 250, 330), (13, 512, 640), (44, 320, 190), (130, 65, 515)]


@pytest.mark.parametrize("shape", MANY)
def test_many_matrices(torch, shape):
    count, rows, cols = shape
    x, w, m = (matrices(count, rows, cols, cols, k) for k in (rows, 1, 2))
    dev = [torch.from_numpy(v).to("cuda:0") for v in (w, x, m)]
    got = B.orthogonalize(dev[1]).cpu().numpy()
    B.muon_step(*dev, lr=0.5, mu=0.5, nesterov=False, scale=1.0)
    moved, momentum = dev[0].cpu().numpy(), dev[2].cpu().numpy()
    for q in sorted({0, 1, count // 2, count - 1}):
        check(got[q], x[q], B.MUON_STEPS, float(np.float32(1e-7)))
        u = 0.5 * m[q].astype(np.float64) + x[q]
        assert np.all(np.abs(momentum[q] - u) <= 2.0 ** -24 * np.abs(u))
        new = w[q] - 0.5 * products(u, B.MUON_STEPS, 1e-7, np.float64)
        # (U's own rounding is within the tolerance's 2^-22 of it; one more in the last addition)
        assert np.linalg.norm(moved[q] - new) <= 0.5 * tolerance(u, B.MUON_STEPS, 1e-7) + 1.01 * 2.0 ** -24 * np.linalg.norm(new)


@pytest.mark.parametrize("steps", [CUBIC, FIFTH, ((1.0, 0.0, 0.0),), ((3.4445, -4.775, 2.0315),), FIFTH + CUBIC + FIFTH])
@pytest.mark.parametrize("shape", [(2, 50, 60, 60), (1, 200, 140, 144), (3, 12, 90, 90), (2, 24, 400, 400)])
def test_coefficients(torch, steps, shape):
    count, rows, cols, ld = shape
    x = matrices(count, rows, cols, ld, 3)
    got = B.orthogonalize(torch.from_numpy(x).to("cuda:0"), cols=cols, coefficients=steps, eps=1e-3).cpu().numpy()
    for q in range(count):
        check(got[q, :, :cols], x[q, :, :cols], steps, float(np.float32(1e-3)))


def test_singular_values_near_one(torch):
    # the fifth-order steps converge: from singular values of 0.3 to 1 of a
    # matrix of norm 1 ... 10 steps of factor 15/8 and then quadratic
    rng = np.random.default_rng(0)
    u, _ = np.linalg.qr(rng.standard_normal((90, 70)))
    v, _ = np.linalg.qr(rng.standard_normal((70, 70)))
    x = (u * np.linspace(0.3, 1.0, 70)) @ v.T
    got = B.orthogonalize(torch.from_numpy(x.astype(np.float32)).to("cuda:0"), coefficients=FIFTH * 4).cpu().numpy()
    assert np.abs(got.T.astype(np.float64) @ got - np.eye(70)).max() < 1e-4
    assert np.abs(got - u @ v.T).max() < 1e-4


@pytest.mark.parametrize("scale", [1e-38, 1e-25, 1.0, 1e18, 1e37])
@pytest.mark.parametrize("rows,cols", [(60, 70), (14, 130), (30, 300)])
def test_scales(torch, rows, cols, scale):
    # squares past float32's range on either side; eps has no share in the
    # large ones and rules the smallest
    x = (matrices(1, rows, cols, cols, 5).astype(np.float64) * (scale * 100)).astype(np.float32)[0]
    assert np.isfinite(x).all()
    got = B.orthogonalize(torch.from_numpy(x).to("cuda:0")).cpu().numpy()
    assert np.isfinite(got).all()
    check(got, x, B.MUON_STEPS, float(np.float32(1e-7)))


@pytest.mark.parametrize("shape", [(4, 30, 40, 40), (4, 200, 150, 150), (4, 10, 300, 300), (4, 90, 7, 7), (4, 20, 200, 200)])
def test_zeros_and_what_is_not_finite(torch, shape):
    count, rows, cols, ld = shape
    x = matrices(count, rows, cols, ld, 6)
    clean = B.orthogonalize(torch.from_numpy(x).to("cuda:0"))
    hurt = x.copy()
    hurt[0] = 0
    hurt[1, 3, 5], hurt[3, 0, 0] = np.nan, np.inf
    got = B.orthogonalize(torch.from_numpy(hurt).to("cuda:0"))
    assert (got[0] == 0).all() and torch.isnan(got[1]).all() and torch.isnan(got[3]).all()
    assert torch.equal(got[2], clean[2])


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (5, 20, 21, 24), (7, 100, 101, 104), (1, 300, 200, 200), (1, 500, 501, 504),
                                   (2, 40, 300, 304), (3, 200, 60, 64), (2, 12, 700, 703), (2, 300, 70, 72), (1, 129, 190, 191), (1, 257, 330, 330),
                                   (9, 260, 500, 500), (2, 1030, 1100, 1101)])
def test_muon_step(torch, shape, nesterov):
    count, rows, cols, ld = shape
    w, g, m = (matrices(count, rows, cols, ld, k) * np.float32(f) for k, f in ((1, 100), (2, 1), (3, 5)))
    for v in (w, g, m):
        v[:, :, cols:] = 9.0
    g[:, :, cols:] = np.nan
    dev = [torch.from_numpy(v).to("cuda:0") for v in (w, g, m)]
    kw = dict(lr=0.02, cols=cols, weight_decay=0.1, mu=0.9, nesterov=nesterov)
    outs = torch.full(w.shape, 4.0, device="cuda:0"), torch.full(w.shape, 5.0, device="cuda:0")
    B.muon_step(*dev, **kw, w_out=outs[0], momentum_out=outs[1])
    assert [np.array_equal(a.cpu().numpy(), b, equal_nan=True) for a, b in zip(dev, (w, g, m))] == [True] * 3
    B.muon_step(*dev, **kw)
    for a, b, c in ((dev[0], outs[0], 4.0), (dev[2], outs[1], 5.0)):
        assert torch.equal(a[:, :, :cols], b[:, :, :cols])
        assert (a[:, :, cols:] == 9.0).all() and (b[:, :, cols:] == c).all()
    mu, rate = float(np.float32(0.9)), float(np.float32(0.02 * np.sqrt(max(1.0, rows / cols))))
    keep = float(np.float32(1) - np.float32(0.02 * 0.1))
    for q in range(count):
        wq, gq, mq = (v[q, :, :cols].astype(np.float64) for v in (w, g, m))
        want = mu * mq + gq
        got = outs[1][q, :, :cols].cpu().numpy()
        assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want))
        u = gq + mu * want if nesterov else want
        new = keep * wq - rate * products(u, B.MUON_STEPS, 1e-7, np.float64)
        # (U's own two roundings are within the tolerance's 2^-22 of it)
        off = np.linalg.norm(outs[0][q, :, :cols].cpu().numpy() - new)
        assert off <= rate * tolerance(u, B.MUON_STEPS, 1e-7) + 2.0 ** -22 * np.linalg.norm(wq)


@pytest.mark.parametrize("rows,cols,ld", [(40, 50, 30_000_000), (200, 190, 6_000_000), (10, 200, 110_000_000), (30, 200, 40_000_000)])
def test_offsets_past_32_bits(torch, rows, cols, ld):
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    x = torch.zeros((2, rows, ld), device="cuda:0")
    assert x.numel() > 1 << 31
    m = matrices(2, rows, cols, cols, 9)
    x[:, :, :cols] = torch.from_numpy(m).to("cuda:0")
    out = torch.full_like(x, 2.0)
    B.orthogonalize(x, cols=cols, out=out)
    assert bool((out[:, :, cols:cols + 1000] == 2.0).all()) and bool((out[:, :, -1000:] == 2.0).all())
    for q in range(2):
        check(out[q, :, :cols].cpu().numpy(), m[q], B.MUON_STEPS, float(np.float32(1e-7)))


def test_two_dimensions_streams_and_graphs(torch):
    x = [torch.from_numpy(matrices(1, r, c, c, k)[0]).to("cuda:0") for k, (r, c) in enumerate(((90, 101), (300, 260), (16, 300)))]
    want = [B.orthogonalize(v) for v in x]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = [B.orthogonalize(v) for v in x]
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, other):
        assert torch.equal(a, b)
    # two training loops captured, each with its own state and workspace
    states = [[v.clone() for v in x] + [torch.zeros_like(v) for v in x] for _ in range(2)]
    held = [v.clone() for v in x]
    graphs = []
    for state in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for w, h, m in zip(state[:3], held, state[3:]):
                B.muon_step(w, h, m, lr=0.1)
        graphs.append(g)
    eager = [v.clone() for v in x] + [torch.zeros_like(v) for v in x]
    for k in range(3):
        for v, h in zip(x, held):
            h.copy_(v * (1.0 - 0.3 * k) + 0.01 * v.flip(0))
        for g in graphs:
            g.replay()
        for w, h, m in zip(eager[:3], held, eager[3:]):
            B.muon_step(w, h, m, lr=0.1)
        torch.cuda.synchronize()
        for st in states:
            for a, b in zip(st, eager):
                assert torch.equal(a, b)


def test_refusals(torch):
    x = torch.zeros((2, 8, 12), device="cuda:0")
    for bad in (x.double(), x[:, :, :8], x[0, 0], x.cpu()):
        with pytest.raises(ValueError):
            B.orthogonalize(bad)
    for cols in (0, 13):
        with pytest.raises(B.CrfError):
            B.orthogonalize(x, cols=cols)
    with pytest.raises(B.CrfError, match="alias"):
        B.orthogonalize(x, out=x)
    with pytest.raises(ValueError):
        B.muon_step(x, x[:1], x.clone(), lr=0.1)
    with pytest.raises(B.CrfError, match="alias"):
        B.muon_step(x, x, x.clone(), lr=0.1)
    for kw in (dict(lr=-0.1), dict(lr=float("nan")), dict(lr=0.1, mu=-1.0), dict(lr=1.0, weight_decay=2.0)):
        with pytest.raises(B.CrfError):
            B.muon_step(x, x.clone(), x.clone(), **kw)
