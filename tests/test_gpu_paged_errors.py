"""Errors of the HIP runtime as the paged cache's calls report them."""
import ctypes

import pytest
import torch

import paged_util as U
import test_gpu_paged as P
from test_gpu_paged import T16, V  # noqa: F401  (V is the fixture)

pytestmark = pytest.mark.gpu


def hip():
    """The runtime that this process has loaded."""
    for ln in open("/proc/self/maps"):
        if "libamdhip64.so" in ln:
            return ctypes.CDLL(ln.split()[-1])
    pytest.skip("no HIP runtime in this process")


def test_an_error_of_the_runtime_keeps_its_name(V):
    """An invalid-argument error that some other call has left (the runtime
    reports it with the next launch) is not taken for a grid that is too
    large. The copy is refused on the host; nothing reaches the GPU."""
    P.say("an error left by another call")
    d = P.Dev(V, U.Model(1, 4, 1, 16, 32, 2, 2), T16)
    torch.cuda.synchronize()
    lib = hip()
    calls = [lambda: V.vla_pages_init(d.p), lambda: V.vla_pages_release(d.p, P.i32([0])),
             lambda: V.vla_pages_commit(d.p, V.make_rows(P.i32([0, 0, 0]), 1))]
    for call in calls:
        lib.hipGetLastError()
        assert lib.hipMemcpy(None, None, 1, 99) != 0
        try:
            call()
        except V.VlaError as e:
            assert e.code == -3 and "grid" not in str(e), str(e)
        lib.hipGetLastError()
    torch.cuda.synchronize()
    V.vla_pages_init(d.p)
    d.same(contents=False)
