"""The offsets that a plan takes, found out on the host before the GPU is asked anything."""
import ctypes
import os

import numpy as np
import pytest

import __graft_entry__ as entry
from paper_2607_27744_b200 import binding

SEGMENTS = -4


@pytest.fixture(scope="module")
def status():
    if not os.path.exists(binding.LIB_PATH):
        entry.build()
    L = ctypes.CDLL(binding.LIB_PATH)
    vp = ctypes.c_void_p
    L.rocs_plan_create.argtypes = [ctypes.POINTER(vp), ctypes.c_int32, ctypes.c_int64, vp, vp, vp]
    L.rocs_plan_destroy.argtypes = [vp]

    def of(off, N):
        off = np.asarray(off, np.int32)
        plan = vp()
        code = L.rocs_plan_create(ctypes.byref(plan), len(off) - 1, N, vp(1 << 20), off.ctypes.data, None)
        if plan:
            L.rocs_plan_destroy(plan)
        return code
    return of


@pytest.mark.parametrize("R", [1, 2, 7, 33, 1000])
def test_a_fall_anywhere_is_found(status, R):
    off = np.arange(R + 1) * 3
    assert status(off, 3 * R) != SEGMENTS
    assert status(off, 3 * R - 1) == SEGMENTS and status(off + 1, 3 * R + 1) == SEGMENTS
    for r in {1, R // 2, R - 1} - {0, R}:
        broken = off.copy()
        broken[r] = off[r + 1] + 1
        assert status(broken, 3 * R) == SEGMENTS
        broken[r] = -1
        assert status(broken, 3 * R) == SEGMENTS


def test_differences_that_leave_32_bits(status):
    most = 2 ** 31 - 1
    assert status([0, most], most) != SEGMENTS
    assert status([0, 0, most, most], most) != SEGMENTS
    assert status([0, most, -2 ** 31, 5], 5) == SEGMENTS      # the fall wraps to a rise of one
    assert status([0, -2 ** 31, most], most) == SEGMENTS
    assert status([0], 0) != SEGMENTS and status([0, 0, 0], 0) != SEGMENTS
