"""How the attention over pages deals its blocks of keys to workgroups, checked
on the host: deal_host.cpp goes through every workgroup of a launch with the
arithmetic that the kernels compile (csrc/deal.h), for batches of up to 300
entries, uneven, padded and empty ones among them, both tile heights and counts
of workgroups.
"""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def prog(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("deal") / "deal")
    subprocess.run(["g++", "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-o", out,
                    os.path.join(HERE, "deal_host.cpp")], check=True)
    return out


@pytest.mark.parametrize("seed", range(4))
def test_every_block_is_dealt_once(prog, seed):
    p = subprocess.run([prog, str(seed), "40"], capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stdout + p.stderr
