"""Rotary positions whose base is next to zero, so that a pair's frequency leaves the range of 64 bits: refused on the host (no GPU: the pointers below are
never followed)."""
import ctypes as C

import pytest

from paper_2510_01565_b200 import binding as B
from paper_2510_01565_b200 import build


@pytest.mark.parametrize("base,trained", [(5e-324, 0.0), (5e-324, 4096.0), (1e-322, 0.0), (1e-305, 0.0)])
def test_frequencies_without_a_value_are_refused(base, trained):
    build.build_library()
    lib = B.load_library()
    n = (C.c_int32 * 1)(7)
    a = B.DitRotaryArgs(1 << 20, 1 << 21, 512, 512, 7, 0, 2, 256, 256, 0, 0, base, 2.0, trained, 1.0, 4.0, 1.0, None, 1, n, None)
    assert lib.dit_rotary(C.byref(a), None) == 1                          # DIT_ERR_INVALID_ARG
