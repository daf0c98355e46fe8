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
