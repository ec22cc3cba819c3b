"""Sizes beyond which a call on the paged cache is refused (CPU: a call that
passes the checks ends at the missing device)."""
import ctypes as C
import os

import pytest

import paper_2609_22335_amd as V
from test_paged_binding import cache, on_device_0  # noqa: F401

X, Y, Z = (C.c_void_p(a << 28) for a in (1, 2, 3))


def test_a_fork_that_would_hold_the_gpu_is_refused():
    p = C.byref(cache())
    for n in ((1 << 17) + 1, 1 << 20, 1 << 24, 2 ** 31 - 1):
        assert V._lib.vla_pages_fork(p, n, X, Y, Z, None) == -4
        assert "2^17" in V.vla_last_error()


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="the addresses are made up: not beside a GPU")
def test_the_largest_fork_is_taken():
    assert V._lib.vla_pages_fork(C.byref(cache()), 1 << 17, X, Y, Z, None) == -3
