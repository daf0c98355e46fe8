"""What the built library would launch, and what it refuses, on a HIP runtime of
host memory (tests/launch_host_stub.cpp): no device, no kernel runs."""
import os
import shutil
import subprocess

import pytest

from paper_2008_03736_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
ROCM_INCLUDE = "/opt/rocm/include"


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("needs g++ and the HIP headers")
    if not os.path.exists(B.LIB_PATH):
        pytest.fail("libcrfinside.so is not built (run __graft_entry__.build())")
    out = str(tmp_path_factory.mktemp("launch") / "launch_host")
    # (-rdynamic: the library's calls of the runtime find this program's functions first)
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I" + ROCM_INCLUDE,
                    "-I" + os.path.join(HERE, "..", "include"), "-o", out, os.path.join(HERE, "launch_host_stub.cpp"),
                    "-ldl", "-pthread"], check=True, capture_output=True, text=True)
    return out


def run(harness, *args):
    res = subprocess.run([harness, args[0], B.LIB_PATH, *map(str, args[1:])], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-2000:]
    return [line.split() for line in res.stdout.splitlines()]


def test_overlapping_buffers_are_refused(harness):
    rows = run(harness, "alias")
    assert len(rows) > 400
    for *what, status in rows:
        ok = what[1] == "none" or what[-1] == "beside"   # (buffers that touch share nothing)
        assert int(status) == (B.CRF_OK if ok else B.CRF_EINVAL), what


def test_first_calls_of_two_threads(harness):
    # the LDS attributes of the scorer's backward kernels are set before either launches
    rows = run(harness, "attributes")
    assert [r for r in rows if r[0] == "EARLY"] == []
    (last,) = [r for r in rows if r[0] == "launches"]
    assert int(last[1]) >= 8 and last[3:] == ["0", "0"]


TEAM = "inside_kernel<%s, true, false, true>"


@pytest.mark.parametrize("call,reverse", [("logprobs", "false"), ("policy", "true")])
def test_log_z_is_missing_until_a_team_has_it(harness, call, reverse):
    # a launch whose teams never assemble writes nothing: what the pass over
    # the trees then reads has to say so
    rows = run(harness, "launches", call, 0, 460, 12, 500, 30)
    names = [" ".join(r[1:]) for r in rows if r[0] == "K"]
    team = [k for k, x in enumerate(names) if TEAM % reverse in x]
    mark = [k for k, x in enumerate(names) if "mark_missing" in x]
    assert len(team) == len(mark) == 1 and mark[0] < team[0] < len(names) - 1 and "tree_kernel" in names[-1], names
    assert [r for r in rows if r[0] == "A"] == [["A", "2", "0", "workspace"]]   # both long ones, longest first


@pytest.mark.parametrize("call,flags,lengths", [("logprobs", 0, (12, 30, 300)), ("policy", B.CRF_NO_TEAMS, (460, 12)),
                                                ("logprobs_bwd", 0, (460, 12)), ("inside", 0, (460, 12))])
def test_calls_without_that_mark(harness, call, flags, lengths):
    assert not any("mark_missing" in " ".join(r) for r in run(harness, "launches", call, flags, *lengths))


@pytest.mark.parametrize("lengths", [[25], list(range(1, 100)) * 2, [20, 300, 7], [460, 12]])
def test_a_plan_is_made_with_few_device_calls(harness, lengths):
    # the tables in one allocation (then the workspace and the team area, where
    # there are any) and few copies: each is a call of its own on the device, of
    # 3 to 10 us, in plans that a training loop makes for every batch (the small
    # tables in one copy, and three of the 198 sentences are past 64 KB)
    (row,) = run(harness, "creation", *lengths)
    assert int(row[1]) <= 1 + 2 * (max(lengths) > 96) and int(row[3]) <= 1 + 3 * (len(lengths) > 100)


def test_host_memory_that_runs_out(harness):
    # a status, not an exception out of a C function, and nothing left behind
    rows = run(harness, "memory", 25, 60, 70, 300, 460)
    assert [r[:2] for r in rows[:-1]] == [["status", str(B.CRF_ENOMEM)], ["status", str(B.CRF_OK)]]
    assert int(rows[0][3]) > 50 and rows[-1] == ["left", "0"]
