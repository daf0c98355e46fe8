"""Refusals of the fine-tuning entry points, on the host, before any HIP call."""
import ctypes
import os

import numpy as np
import pytest

from paper_2008_03736_amd import binding as B

P = ctypes.c_void_p(0x100000)     # stands for device memory: never dereferenced by a refused call
Q = ctypes.c_void_p(0x200000)
ODD = ctypes.c_void_p(0x100004)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.fail("libcrfinside.so is not built (run __graft_entry__.build())")
    return B.load()


def test_null_plan(lib):
    n = ctypes.c_int64()
    assert lib.crf_tree_workspace(None, ctypes.byref(n)) == B.CRF_EINVAL
    assert lib.crf_tree_logprobs(None, P, P, 1, None, P, None, P, 1 << 20, None) == B.CRF_EINVAL
    assert lib.crf_tree_logprobs_bwd(None, P, P, 1, None, P, Q, None) == B.CRF_EINVAL
    assert lib.crf_policy_loss(None, P, P, 1, None, P, P, None, 0.2, 0.2, 0.0, None, P, None, Q, P, 1 << 20,
                               None) == B.CRF_EINVAL
    assert lib.crf_pack_rows(None, P, 100, P, P, None) == B.CRF_EINVAL
    assert lib.crf_unpack_rows(None, P, P, 100, P, None) == B.CRF_EINVAL
    assert lib.crf_biaffine_bwd_workspace(None, 100, 1, ctypes.byref(n)) == B.CRF_EINVAL
    assert lib.crf_biaffine_bwd(None, P, P, P, 100, 104, 1, P, Q, Q, None, P, 1 << 20, None) == B.CRF_EINVAL
    assert lib.crf_biaffine_bwd_packed(None, P, P, P, P, P, 100, 104, 1, P, Q, Q, None, P, 1 << 20, None) == B.CRF_EINVAL
    assert "plan" in B.crf_last_error()


def test_constants_match_header():
    text = open(os.path.join(os.path.dirname(B.PKG), "include", "crf_inside.h")).read()
    assert f"#define CRF_MAX_TREES {B.CRF_MAX_TREES} " in text
    assert f"#define CRF_MAX_ROW {B.CRF_MAX_ROW} " in text
