"""How far packed rows may be off, as crf_rows.hip states it, from the codec's
definition in float64 (no GPU)."""
import numpy as np

from paper_2008_03736_amd import workloads as W
from test_rows_gpu import reference


def error_of(top, x):
    """Relative error of x's code in a block whose largest value is top."""
    rows = np.zeros((len(x), 32))
    rows[:, 0], rows[:, 1] = top, x
    s, v = reference(rows)
    return np.abs(v[:, 1] - x) / x, np.abs(v[:, 1] - x) / 2.0 ** s[:, 0], x / 2.0 ** s[:, 0]


def test_stated_bound():
    every = W.from_bf16(np.arange(0x3000, 0x4000, dtype=np.uint16)).astype(np.float64)   # 2^-31 to 2
    for top in W.from_bf16(np.arange(0x3F80, 0x4080, 3, dtype=np.uint16)).astype(np.float64):   # 1 to 4
        x = every[every <= top]
        rel, steps, scaled = error_of(top, x)
        normal = scaled >= 2.0 ** -6
        assert rel[normal].max() <= 2.0 ** -4 and steps[~normal].max() <= 2.0 ** -10
        assert normal[x >= 2.0 ** -13 * top].all()
    # 2^-14 of the largest is too far: below 2^-6 of the scale codes are 2^-9 apart
    rel, _, _ = error_of(225.0, np.array([7.46875 / 512]))
    assert 7.46875 / 512 > 2.0 ** -14 * 225.0 and rel[0] > 2.0 ** -4
