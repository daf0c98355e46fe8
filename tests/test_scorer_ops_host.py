"""Layer norm, the width bias and the orthogonalised update without a GPU: what
they refuse, on the host, before any HIP call; the buckets of widths; and
overlapping buffers and launches on a HIP runtime of host memory
(tests/scorer_ops_stub.cpp)."""
import ctypes
import csv
import math
import os
import re
import shutil
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from paper_2008_03736_amd import binding as B
from paper_2008_03736_amd import build as BLD

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM_INCLUDE = "/opt/rocm/include"
P, Q, R = (ctypes.c_void_p(k << 40) for k in (1, 2, 3))   # stand for device memory: never dereferenced by a refused call
S, T = ctypes.c_void_p(4 << 40), ctypes.c_void_p(5 << 40)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.fail("libcrfinside.so is not built (run __graft_entry__.build())")
    return B.load()


def steps(*co):
    a = np.asarray(co, np.float32)
    return a, a.ctypes.data, len(a)


def test_null_arguments(lib):
    n = ctypes.c_int64()
    assert lib.crf_layer_norm(None, P, 0, 8, None, None, 1e-5, Q, None) == B.CRF_EINVAL
    assert lib.crf_layer_norm_bwd_workspace(None, 8, ctypes.byref(n)) == B.CRF_EINVAL
    assert lib.crf_layer_norm_bwd(None, P, 0, 8, None, Q, 1e-5, R, None, None, S, 1 << 20, None) == B.CRF_EINVAL
    assert lib.crf_width_bias(None, P, 1, Q, R, 4, S, None) == B.CRF_EINVAL
    assert lib.crf_width_bias_bwd_workspace(None, 1, ctypes.byref(n)) == B.CRF_EINVAL
    assert lib.crf_width_bias_bwd(None, P, 1, R, 4, None, S, T, 1 << 20, None) == B.CRF_EINVAL
    assert lib.crf_biaffine_scores_biased(None, P, Q, R, 8, 12, 1, S, T, 4, P, None) == B.CRF_EINVAL
    assert "plan" in B.crf_last_error()
    _, co, k = steps((1.5, -0.5, 0.0))
    assert lib.crf_orthogonalize(None, 1, 8, 8, 8, co, k, 1e-7, Q, R, 1 << 30, None) == B.CRF_EINVAL
    assert lib.crf_orthogonalize(P, 1, 8, 8, 8, None, k, 1e-7, Q, R, 1 << 30, None) == B.CRF_EINVAL
    assert lib.crf_orthogonalize(P, 1, 8, 8, 8, co, k, 1e-7, Q, None, 1 << 30, None) == B.CRF_EINVAL
    assert lib.crf_muon_step(P, Q, None, 1, 8, 8, 8, 0.9, 1, 0.1, 0.0, co, k, 1e-7, P, R, S, 1 << 30, None) == B.CRF_EINVAL
    assert lib.crf_orthogonalize_workspace(1, 8, 8, None) == B.CRF_EINVAL


@pytest.mark.parametrize("count,rows,cols,ld", [(0, 8, 8, 8), (4097, 8, 8, 8), (1, 0, 8, 8), (1, 8, 0, 8), (1, 8193, 8, 8),
                                                (1, 8, 8193, 8193), (1, 8, 8, 7), (-1, 8, 8, 8)])
def test_sizes_of_matrices(lib, count, rows, cols, ld):
    _, co, k = steps((1.5, -0.5, 0.0))
    assert lib.crf_orthogonalize(P, count, rows, cols, ld, co, k, 1e-7, Q, R, 1 << 40, None) == B.CRF_EINVAL
    if ld >= cols:
        assert lib.crf_orthogonalize_workspace(count, rows, cols, ctypes.byref(ctypes.c_int64())) == B.CRF_EINVAL


@pytest.mark.parametrize("co", [((5.0, 0.0, 0.0),), ((3.0, 0.0, 0.0),) * 2, ((1.0, -61.0, 0.0),), ((1.0, 0.0, 70.0),),
                                ((1.0, float("nan"), 0.0),), ((float("inf"), 0.0, 0.0),), ((0.5, 1e30, -1e30),),
                                ((3.4445, -4.7750, 2.0315),) * 33])
def test_steps_that_leave_the_range(lib, co):
    _, at, k = steps(*co)
    assert lib.crf_orthogonalize(P, 1, 8, 8, 8, at, k, 1e-7, Q, R, 1 << 30, None) == B.CRF_EINVAL


def test_what_steps_reach():
    # the check's bound by dense sampling: the usual coefficients pass, for as many steps as are allowed
    s = np.linspace(0, 1, 100001)
    most = 1.0
    for a, b, c in B.MUON_STEPS * 6:
        t = s * most
        assert np.abs(b * t ** 2 + c * t ** 4).max() < 60
        most = np.abs(a * t + b * t ** 3 + c * t ** 5).max()
        assert most < 4


@pytest.mark.parametrize("eps", [0.0, -1.0, float("nan"), float("inf")])
def test_eps(lib, eps):
    _, co, k = steps((1.5, -0.5, 0.0))
    assert lib.crf_orthogonalize(P, 1, 8, 8, 8, co, k, eps, Q, R, 1 << 30, None) == B.CRF_EINVAL


def test_constants_match_header():
    text = open(os.path.join(os.path.dirname(B.PKG), "include", "crf_inside.h")).read()
    for name in ("CRF_MAX_BUCKETS", "CRF_MAX_STEPS", "CRF_BF16", "CRF_F32"):
        assert f"#define {name} {getattr(B, name)} " in text


@pytest.mark.parametrize("n1,K,reach", [(2, 1, 1), (40, 1, 7), (60, 2, 2), (102, 16, 64), (300, 5, 81), (300, 9, 80), (64, 64, 40),
                                        (1024, 32, 256), (1024, 1024, 600)])
def test_width_buckets(n1, K, reach):
    got = B.width_buckets(n1, K, reach)
    single = (K + 1) // 2
    assert got.dtype == np.int32 and got.shape == (n1,) and got.min() >= 0 and got.max() < K
    for w in range(1, n1):
        if w <= single or K == 1:
            assert got[w] == min(w, K) - 1
            continue
        far = (K - single) * math.log(w / single) / math.log(reach / single)
        want = min(K - 1, single + math.floor(far))
        if abs(far - round(far)) < 1e-9:   # a border: by whole numbers
            up = Fraction(reach, single) ** round(far) <= Fraction(w, single) ** (K - single)
            want = min(K - 1, single + (round(far) if up else round(far) - 1))
        assert got[w] == want, w


def test_width_buckets_refuses():
    for args in ((1, 4, 8), (8, 0, 8), (8, 1025, 2000), (8, 4, 2)):
        with pytest.raises(ValueError):
            B.width_buckets(*args)


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("needs g++ and the HIP headers")
    if not os.path.exists(B.LIB_PATH):
        pytest.fail("libcrfinside.so is not built (run __graft_entry__.build())")
    out = str(tmp_path_factory.mktemp("ops") / "scorer_ops")
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I" + ROCM_INCLUDE,
                    "-I" + os.path.join(HERE, "..", "include"), "-o", out, os.path.join(HERE, "scorer_ops_stub.cpp"),
                    "-ldl", "-pthread"], check=True, capture_output=True, text=True)
    return out


def run(harness, *args):
    res = subprocess.run([harness, args[0], B.LIB_PATH, *map(str, args[1:])], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-2000:]
    return [line.split() for line in res.stdout.splitlines()]


IN_PLACE = [["width", "out", "scores", "same"], ["muon", "w_out", "w", "same"], ["muon", "momentum_out", "momentum", "same"]]


def test_overlapping_buffers_are_refused(harness):
    rows = run(harness, "alias")
    assert len(rows) > 150
    for *what, status in rows:
        ok = what[1] == "none" or what[-1] == "beside" or what in IN_PLACE
        assert int(status) == (B.CRF_OK if ok else B.CRF_EINVAL), what
    assert sum(what[:-1] in IN_PLACE for what in rows) == len(IN_PLACE)


@pytest.mark.parametrize("lengths", [[1], [1023], [5] * 3000, list(range(1, 141)) * 3])
@pytest.mark.parametrize("d,labels", [(4, 1), (100, 138), (500, 15), (8192, 4096)])
def test_launches_fit_the_device(harness, lengths, d, labels):
    rows = run(harness, "grids", d, labels, *lengths)
    assert len(rows) >= 5
    for _, name, gx, gy, gz, threads, lds in rows:
        assert 1 <= int(gx) < 2 ** 31 and 1 <= int(gy) < 65536 and 1 <= int(gz) < 65536, name
        assert int(threads) <= 1024 and int(lds) <= 160 * 1024, name


@pytest.mark.parametrize("shape", [(1, 1, 1), (4096, 1, 1), (1, 8192, 8192), (138, 100, 101), (1, 500, 501), (4096, 16, 300), (1, 16, 2048),
                                   (2, 2049, 16), (300, 32, 500), (2, 112, 160), (1, 512, 17), (1, 128, 129)])
def test_update_launches_fit_the_device(harness, shape):
    rows = run(harness, "update", *shape)
    assert rows
    for _, name, gx, gy, gz, threads, lds in rows:
        assert 1 <= int(gx) < 2 ** 31 and 1 <= int(gy) < 65536 and 1 <= int(gz) < 65536, name
        assert int(threads) <= 1024 and int(lds) <= 160 * 1024, name


def test_eps_of_a_norm(harness):
    # a variance beside an eps below float32's least normal number, 2^-126, would be
    # one of squares of few digits
    least = 2.0 ** -126
    bad = [0.0, -1.0, float("nan"), float("inf"), 2.0 ** -149, 1e-40, least * (1 - 2.0 ** -23)]
    good = [least, 1.2e-38, 1e-12, 1e-5, 1.0]
    for status in run(harness, "eps", *map(repr, bad)):
        assert status == [str(B.CRF_EINVAL)] * 2
    for status in run(harness, "eps", *map(repr, good)):
        assert status == [str(B.CRF_OK)] * 2


def reach(co, most=1.0):
    """(what singular values up to `most` grow to at most, the polynomial's largest value) by dense sampling."""
    s = most * np.sqrt(np.linspace(0, 1, 200001))
    a, b, c = np.asarray(co, np.float32).astype(np.float64)
    poly = np.abs(a + b * s ** 2 + c * s ** 4)
    return (s * poly).max(), poly.max()


# (a, b, 0)'s largest value inside (0, 1), as c goes to 0 from either side; and c
# that rules, with a root of the derivative near 0
SMALL_C = [(50, -50, c) for c in (0, 1e-30, -1e-30, 1e-16, -1e-16, 1e-12, 1e-6, -1e-6)] + \
    [(-20, 20, 1e-20), (30, -40, -1e-25), (10.5, -10.5, 1e-18), (10.3, -10.3, 1e-18), (1e-25, 10, -10), (-1e-25, 11, -11),
     (1e-20, 30, -30), (0, 12, -12), (10, 0, -10), (3, 1e-20, -3)]


def test_steps_are_judged_by_what_they_reach(harness):
    # every set is refused exactly where sampling says so (none lies within 1e-3 of a bound)
    rng = np.random.default_rng(0)
    sets = list(SMALL_C)
    for _ in range(400):
        a, b = rng.uniform(-30, 30), rng.uniform(-60, 60)
        sets.append((a, rng.choice([b, -a, -2 * a]), rng.choice([1.0, 0.0, 1e-7, 1e-15, 1e-24]) * rng.uniform(-40, 40)))
    bounds = [(g / 4, q / 60) for g, q in map(reach, sets)]
    sets, bounds = zip(*[(co, max(b)) for co, b in zip(sets, bounds) if all(abs(v - 1) > 1e-3 for v in b)])
    flat = [repr(float(np.float32(v))) for co in sets for v in co]
    got = [int(r[0]) for r in run(harness, "steps", 1, *flat)]
    assert len(got) == len(sets) > 380
    for co, bound, status in zip(sets, bounds, got):
        assert status == (B.CRF_EINVAL if bound > 1 else B.CRF_OK), (co, bound)
    assert 50 < sum(bound > 1 for bound in bounds) < len(sets) - 50


def test_coefficients_past_a_thousand(harness):
    # refused whatever they reach: a first step to 0.01, where b s^2 is 0.15 at most
    sets = [(0.01, 0, 0, 1, b, c) for b, c in ((999, 0), (1500, 0), (-1500, 0), (1000, 0), (0, 1000), (0, 2000), (1, -1001))]
    got = [int(r[0]) for r in run(harness, "steps", 2, *(v for co in sets for v in co))]
    assert got == [B.CRF_EINVAL if max(abs(v) for v in co) > 1000 else B.CRF_OK for co in sets]


def test_tiles_take_whole_rounds_of_k(harness):
    # a product in tiles of 64 M x 64 M runs its K in rounds of 64 M: a rule that
    # picks the tile by the result's sides alone repeats K's last blocks.  Every
    # pair of padded sides up to 640, and counts past each threshold on the way
    # from small tiles to large ones (128 tiles: 128, 43, 22, 13, 9 matrices).
    rows = [tuple(map(int, r[1:])) for r in run(harness, "products", 10, 132)]
    assert {(kind, tiles) for kind, tiles, _ in rows} == {(kind, tiles) for kind in range(4) for tiles in (1, 2)}
    for kind, tiles, k in rows:
        assert 64 <= k <= 640 and k % 64 == 0
        assert k % (64 * tiles) == 0, (kind, tiles, k)


def test_attributes_of_the_scorer_with_a_bias(harness):
    # set once a device, before any thread's first launch there; a plan sets those
    # of the scorer without one alone
    rows = run(harness, "biased")
    plans = [" ".join(r[1:]) for r in rows if r[0] == "A"]
    assert len(plans) == 10 and all(re.search(r"_kernel<[^>]*, false>", name) for name in plans)
    assert rows[-1] == ["launches", "2", "status", "0", "0"]
    assert not [r for r in rows if r[0] == "EARLY"]


def test_scratch_memory():
    with open(BLD.TRAIN_RESOURCES) as f:
        rows = list(csv.DictReader(f, delimiter="\t"))
    mine = [r for r in rows if any(x in r["kernel"] for x in ("norm_kernel", "norm_bwd_kernel", "norm_join", "width_", "ortho_"))]
    assert len(mine) > 30
    for r in mine:
        assert int(r["ScratchSize [bytes/lane]"]) == 0, r["kernel"]
