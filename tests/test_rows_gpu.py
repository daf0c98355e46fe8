"""Activation rows in 8 bits: the codes, the scales and the values they stand
for against the definition in float64.  Everything is exact: the scale is a
power of two, a bf16 value times it is exact, the code is that product's
nearest e4m3 value, ties to even, and a code times its scale is a bf16 value (of the codes that are taken: see
reference)."""
import numpy as np
import pytest

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


def e4m3_values():
    """The 256 codes' values (NaN for 0x7f and 0xff)."""
    c = np.arange(256)
    e, m = c >> 3 & 15, c & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7), m / 8.0 * 2.0 ** -6)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >> 7, -v, v)


def reference(x):
    """(scales, values) of float64 rows [..., d], finite entries."""
    d = x.shape[-1]
    v = np.concatenate([x, np.zeros(x.shape[:-1] + (-d % 32,))], -1).reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(v).max(-1)
    m, e = np.frexp(top)
    s = np.where(top > 0, e - 9 + (m > 0.875), -127).clip(-127)
    scaled = v * 2.0 ** -s[..., None].astype(np.float64)
    # s = 120 only for magnitudes above 1.75 2^127, codes up to 256: the code
    # 256 would stand for 2^128, past bf16's largest (1.9922 2^127), and 240
    # (1.875 2^127) is the largest that stands for a bf16 value
    scaled = np.where(s[..., None] == 120, np.clip(scaled, -240, 240), scaled)
    step = 2.0 ** (np.maximum(np.frexp(scaled)[1] - 1, -6) - 3.0)
    return s, (np.rint(scaled / step) * step * 2.0 ** s[..., None]).reshape(x.shape[:-1] + (-1,))[..., :d]


def rows(lengths, n1, d, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((len(lengths), n1, d)) * np.exp(spread * rng.standard_normal((len(lengths), n1, d)))
    return W.to_bf16(x)


def there(lengths, n1):
    return np.arange(n1)[None] <= np.asarray(lengths)[:, None]


@pytest.mark.parametrize("d", [4, 28, 32, 36, 64, 100, 124, 500, 508, 1024, 8192])
def test_pack_and_unpack(torch, d):
    lengths = [1, 2, 30, 63, 64, 70, 5]
    n1 = 75
    bits = rows(lengths, n1, d, d, spread=2.0)
    ok = there(lengths, n1)
    bits[~ok] = 0x7FC0   # NaN rows past the sentences: not read
    dev = torch.device("cuda", 0)
    x = torch.from_numpy(bits.view(np.int16)).to(dev)
    wide = (d + 31) // 32 * 32
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        codes, scales = plan.pack_rows(x, codes=torch.full((7, n1, wide), 0xAB, dtype=torch.uint8, device=dev),
                                       scales=torch.full((7, n1, wide // 32), 0xCD, dtype=torch.uint8, device=dev))
        back = plan.unpack_rows(codes, scales, d, out=torch.full((7, n1, d), 3.0, dtype=torch.bfloat16, device=dev))
        torch.cuda.synchronize()
    codes, scales = codes.cpu().numpy(), scales.cpu().numpy()
    back = back.view(torch.int16).cpu().numpy().view(np.uint16)
    assert np.all(codes[~ok] == 0xAB) and np.all(scales[~ok] == 0xCD) and np.all(back[~ok] == 0x4040)
    s, want = reference(W.from_bf16(bits[ok]).astype(np.float64))
    assert np.array_equal(scales[ok].astype(int) - 127, s)
    value = e4m3_values()[codes[ok]].reshape(s.shape + (32,)) * 2.0 ** s[..., None]
    value = value.reshape(s.shape[0], wide)
    assert np.array_equal(value[:, :d], want) and np.all(codes[ok][:, d:] == 0)
    assert np.array_equal(W.from_bf16(back[ok]).astype(np.float64), want)


def test_edges_of_the_range(torch):
    # blocks of: zeros; the largest bf16; 448 and just past it (the next
    # power); bf16's smallest; ties; infinities and NaN beside finite entries
    d = 32
    x = np.zeros((8, d), np.float32)
    x[1, 0], x[1, 1] = W.from_bf16(np.uint16(0x7F7F)), 1.0
    x[2, :3] = 448.0, 1.0, -17.0
    x[3, :3] = 450.0, 1.0, -17.0
    x[4, :2] = W.from_bf16(np.uint16(0x0001)), -W.from_bf16(np.uint16(0x0003))
    x[5, :6] = 256.0, 17.0, 19.0, 21.0, -1.0 / 512, 2.0 ** -10
    x[6, :4] = np.inf, -np.inf, np.nan, 2.0
    x[7, :3] = W.from_bf16(np.uint16(0x00FF)), 2.0 ** -126, -2.0 ** -130
    bits = W.to_bf16(x)
    bits[6, 0], bits[6, 1], bits[6, 2] = 0x7F80, 0xFF80, 0x7FC1
    lengths = [7]
    dev = torch.device("cuda", 0)
    with B.Plan(lengths, n1=8, device=dev) as plan:
        codes, scales = plan.pack_rows(torch.from_numpy(bits.view(np.int16)[None]).to(dev))
        back = plan.unpack_rows(codes, scales, d)
        codes, scales, back = codes[0].cpu().numpy(), scales[0].cpu().numpy(), back[0].float().cpu().numpy()
    fin = W.from_bf16(bits).astype(np.float64)
    bad = ~np.isfinite(fin)
    s, want = reference(np.where(bad, 0.0, fin))
    assert np.array_equal(scales.astype(int)[:, 0] - 127, s[:, 0])
    got = e4m3_values()[codes] * 2.0 ** s
    assert np.array_equal(got[~bad], want[~bad]) and np.all((codes[bad] & 0x7F) == 0x7F)
    assert np.isnan(back[bad]).all()
    normal = ~bad & (np.abs(want) >= 2.0 ** -126)
    assert np.array_equal(back[normal].astype(np.float64), want[normal])
    assert np.all(np.abs(back - want)[~bad & ~normal] <= 2.0 ** -134)   # half of bf16's smallest step


def test_captured(torch):
    lengths, n1, d = [3, 40, 66], 70, 100
    dev = torch.device("cuda", 0)
    xs = [torch.from_numpy(rows(lengths, n1, d, k).view(np.int16)).to(dev) for k in (1, 2)]
    with B.Plan(lengths, n1=n1, device=dev) as plan:
        call = lambda x: (lambda c, s: (c, s, plan.unpack_rows(c, s, d)))(*plan.pack_rows(x))
        want = [call(x) for x in xs]
        held, graph = xs[0].clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call(held)
        for k in (0, 1, 0):
            held.copy_(xs[k])
            graph.replay()
            torch.cuda.synchronize()
            call(xs[1])
            for a, b in zip(out, want[k]):
                assert torch.equal(a, b)


def test_refusals(torch):
    dev = torch.device("cuda", 0)
    with B.Plan([3, 5], n1=6, device=dev) as plan:
        x = lambda d: torch.zeros((2, 6, d), dtype=torch.bfloat16, device=dev)
        for d in (2, 6, 8196):
            with pytest.raises(B.CrfError, match="multiple of 4"):
                plan.pack_rows(x(d))
        with pytest.raises(ValueError):
            plan.pack_rows(x(8).float())
        with pytest.raises(ValueError):
            plan.pack_rows(x(16)[..., :8])
        with pytest.raises(ValueError):
            plan.pack_rows(x(8), codes=torch.zeros((2, 6, 8), dtype=torch.uint8, device=dev))
        c, s = plan.pack_rows(x(8))
        with pytest.raises(B.CrfError, match="16-byte"):
            B.crf_unpack_rows(plan._handle, c.data_ptr() + 1, s.data_ptr(), 8, x(8).data_ptr(), None)
        with pytest.raises(B.CrfError, match="8-byte"):
            B.crf_pack_rows(plan._handle, x(8).data_ptr() + 2, 8, c.data_ptr(), s.data_ptr(), None)


def test_refused_aliases(torch):
    dev = torch.device("cuda", 0)
    with B.Plan([3, 5], n1=6, device=dev) as plan:
        x, s = torch.zeros((2, 6, 32), dtype=torch.bfloat16, device=dev), torch.zeros((2, 6, 1), dtype=torch.uint8, device=dev)
        with pytest.raises(B.CrfError, match="alias"):
            B.crf_pack_rows(plan._handle, x.data_ptr(), 32, x.data_ptr(), s.data_ptr(), None)
        with pytest.raises(B.CrfError, match="alias"):
            B.crf_unpack_rows(plan._handle, x.data_ptr(), s.data_ptr(), 32, x.data_ptr(), None)
