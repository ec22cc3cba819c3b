"""How attention in a window deals its blocks of keys to workgroups, checked on
the host as in test_deal.py: nothing before a tile's window is dealt, everything
from there on exactly once.
"""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def prog(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("deal") / "deal")
    subprocess.run(["g++", "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-o", out,
                    os.path.join(HERE, "deal_window_host.cpp")], check=True)
    return out


@pytest.mark.parametrize("seed", range(4))
def test_every_block_in_a_window_is_dealt_once(prog, seed):
    p = subprocess.run([prog, str(seed), "60"], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout + p.stderr
