"""Refusals of the 4-bit cache's calls, each told by its own text or status."""
import ctypes

import pytest

from paper_2604_00754_b200 import binding as sa
from test_cache_host import FAKE, append, cache


def test_append_checks_the_holders_it_is_given():
    assert append(cache(refs=FAKE + 2)) == 1
    c = cache(refs=FAKE + 2, lens=None)                  # a read looks at no holders
    st = (ctypes.c_int64 * 3)(1024, 128, 60)             # and stops at its strides
    assert sa.load_library().sa_cache_read(ctypes.byref(c), 0, 1, 1, FAKE, 2 * FAKE, sa.BF16, st, None, None, None, None) == 1
