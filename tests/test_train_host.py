"""The fine-tuning operators' host side: the tables that their kernels index
memory by (tests/train_tables_stub.cpp, built for the CPU), and their kernels'
registers and scratch memory as the build reports them."""
import csv
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2008_03736_amd import build as BLD

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM_INCLUDE = "/opt/rocm/include"
ROWS, CELLS = 64, 2048


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("needs g++ and the HIP headers")
    out = str(tmp_path_factory.mktemp("tables") / "train_tables")
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I" + ROCM_INCLUDE, "-I" + os.path.join(HERE, "..", "include"), "-o", out,
                    os.path.join(HERE, "train_tables_stub.cpp")], check=True, capture_output=True, text=True)
    return out


def tables(harness, tmp_path, lengths):
    f = tmp_path / "lengths.txt"
    f.write_text("\n".join(str(int(v)) for v in lengths))
    res = subprocess.run([harness, str(f)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-2000:]
    out = dict(P=[], F=[], T=[])
    for line in res.stdout.splitlines():
        t = line.split()
        if t[0] == "H":
            out["H"] = list(map(int, t[1:]))
        else:
            out[t[0]].append(list(map(int, t[1:])))
    return {k: np.asarray(v, np.int64) for k, v in out.items()}


LENGTHS = {"one": [1], "edges": [62, 63, 64, 65, 127, 128, 129, 1, 2], "long": [1023, 300, 5],
           "batch": np.random.default_rng(0).integers(1, 141, 700).tolist(), "equal": [25] * 200}


@pytest.mark.parametrize("name", sorted(LENGTHS))
def test_posts_and_cells(harness, tmp_path, name):
    n = np.asarray(LENGTHS[name])
    t = tables(harness, tmp_path, n)
    Bn, n1, blocks, long_blocks, _, _, cells = t["H"]
    square, compact, rest, ids = t["P"].T
    assert len(t["F"]) == blocks and len(ids) == ROWS * blocks and cells == int((n * n).sum())
    here = ids >= 0
    want = np.concatenate([b * n1 + np.arange(k + 1) for b, k in enumerate(n)])
    assert np.array_equal(np.sort(ids[here]), want), "every fence post once"
    b, i = ids[here] // n1, ids[here] % n1
    assert np.array_equal(rest[here], n[b] - i) and np.all(rest[~here] == 0)
    # cells (i, j), j = i+1 .. n, of a row with some: where they are, and inside the arrays
    some, base = rest[here] > 0, np.concatenate([[0], np.cumsum(n * n)])
    assert np.array_equal(square[here][some], (b * n1 * n1 + i * n1 + i)[some])
    assert np.array_equal(compact[here][some], (base[b] + i * n[b] + i - 1)[some])
    # (cell j = i + 1 is read for every place, also for an empty one)
    assert np.all(square + 1 >= 0) and np.all(square + np.maximum(rest, 1) < Bn * n1 * n1)
    assert np.all(compact + 1 >= 0) and np.all(compact + np.maximum(rest, 1) < cells)
    owner = np.where(here, ids // n1, -1).reshape(blocks, ROWS)
    for q, (first, last) in enumerate(t["F"]):
        mine = set(owner[q]) - {-1}
        assert mine and first <= q <= last < blocks
        if q < long_blocks:   # of one sentence, whose blocks are neighbours and in order
            (s,) = mine
            assert n[s] + 1 > ROWS and last - first + 1 == -(-(n[s] + 1) // ROWS)
            at = ids.reshape(blocks, ROWS)[first:last + 1].ravel()
            assert np.array_equal(at[:n[s] + 1], s * n1 + np.arange(n[s] + 1)) and np.all(at[n[s] + 1:] < 0)
        else:                 # whole sentences, each one's posts side by side
            assert first == last == q
            for s in mine:
                at = np.flatnonzero(owner[q] == s)
                assert len(at) == n[s] + 1 and np.array_equal(at, at[0] + np.arange(len(at)))


@pytest.mark.parametrize("name", sorted(LENGTHS))
def test_stripes(harness, tmp_path, name):
    n = np.asarray(LENGTHS[name])
    t = tables(harness, tmp_path, n)
    rows = [np.zeros(k, int) for k in n]
    most = 0
    for b, k, first, count in t["T"]:
        assert k == n[b] and count >= 1 and (count * k <= CELLS or count == 1)
        rows[b][first:first + count] += 1
        assert first + count <= k
        most = max(most, count * k)
    assert all((r == 1).all() for r in rows), "every row once"
    assert t["H"][5] >= most and len(t["T"]) == t["H"][4]


def test_scratch_memory():
    """A spill in these kernels' loops sits between the loads and the matrix
    instructions that they feed."""
    with open(BLD.TRAIN_RESOURCES) as f:
        rows = list(csv.DictReader(f, delimiter="\t"))
    names = [r["kernel"] for r in rows]
    for part in ("tree_kernel", "pack_rows_kernel", "unpack_rows_kernel", "bwd_weights_kernel", "bwd_compact_kernel",
                 "bwd_posts_kernel", "bwd_long_kernel", "bwd_weight_kernel", "bwd_join_rows_kernel",
                 "bwd_join_weight_kernel"):
        assert any(part in x for x in names), part
    # (two builds that decode 8-bit rows, once an item, outside the loops over K and labels)
    least = {"bwd_posts_kernel<4, 8, 4, true, false>": 8, "bwd_posts_kernel<1, 4, 2, true, true>": 16}
    for r in rows:
        allowed = max([v for k, v in least.items() if k in r["kernel"]], default=0)
        assert int(r["ScratchSize [bytes/lane]"]) <= allowed, r["kernel"]
