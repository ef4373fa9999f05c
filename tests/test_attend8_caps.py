"""Caps of scores whose arithmetic fp32 does not hold are refused, without a GPU; the largest ones that are not leave scores as they are."""
import ctypes as C
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_cache8_plain import ARG, attend_params, lib  # noqa: E402,F401


@pytest.mark.parametrize("change", [dict(cap=3e38), dict(cap=2.4e38), dict(cap=3e38, scale=100.0), dict(cap=1e38), dict(cap=1e37, scale=0.088), dict(cap=1e30, scale=1e-9)])
def test_caps_that_are_too_large(lib, change):  # noqa: F811
    """cap / ln 2 beyond fp32 makes a score of 0 NaN (0 times infinity); a scale over the cap below the normal numbers loses bits of every score."""
    need, some = C.c_uint64(0), C.c_void_p(256)
    p = attend_params(**change)
    assert lib.kvp_attend8_workspace(C.byref(p), 1, 1, C.byref(need)) == ARG
    assert lib.kvp_attend8(C.byref(p), some, some, some, some, some, some, some, some, some, some, C.c_uint64(1 << 40), None) == ARG


def test_caps_that_are_served(lib):  # noqa: F811
    need = C.c_uint64(0)
    for change in (dict(cap=1e30), dict(cap=1e36), dict(cap=1e36, scale=0.0), dict(cap=2e38, scale=10.0), dict(cap=1e-30), dict(cap=3e38, scale=0.0)):
        p = attend_params(**change)
        assert lib.kvp_attend8_workspace(C.byref(p), 1, 1, C.byref(need)) == (ARG if change["cap"] == 3e38 else 0), change


@pytest.mark.gpu
def test_large_caps_leave_scores_as_they_are():
    import numpy as np
    from paper_2508_13231_b200 import kvp
    from test_gpu_attend8 import check, problem
    for cap in (1e6, 1e30, 1e36):
        for rows in (1, 20):
            p = problem(kvp, 2, 1, 2, rows, 128, 16, 16, [300, 17])
            check(kvp, *p, 16, cap=float(np.float32(cap)))
