"""The attention kernel with tiles of 128 rows sends for four stages of K and V
before it begins and then waits by count: for the first two, later for the
third. The stages lie in different LDS objects, so the order in which their
loads go out is the compiler's unless something holds it. It is read off the
library built here.
"""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_22335_amd", "libvla.so")
LLVM = "/opt/rocm/llvm/bin/"

WAIT = re.compile(r"s_waitcnt vmcnt\((\d+)\)")
LOAD = re.compile(r"buffer_load_dwordx4 .* lds\b")
WRITE = re.compile(r"\s*s_(\w+) (m0|s\d+), (\S+?)(?:, (\S+))?\s*(?://|$)")


def number(x):
    return int(x, 0) if re.fullmatch(r"-?(0x[0-9a-f]+|\d+)", x or "") else None


def places(lines, wait):
    """The constant part of the LDS address of each load before the first wait
    for all but `wait` loads, in the order in which they go out. (The rest of
    the address is the wave's place in a load, less than a stage.)"""
    known, out = {}, []
    for ln in lines:
        w = WRITE.match(ln)
        if w:
            op, dst, a, b = w.groups()
            val = known.get(a) if number(a) is None else number(a)
            if op in ("mov_b32", "movk_i32"):
                new = val
            elif op == "lshl_b32":
                new = 0  # the wave's place
            elif op in ("add_i32", "or_b32", "add_u32") and number(b) is not None and val is not None:
                new = val + number(b)
            else:
                new = None
            known.pop(dst, None)
            if new is not None:
                known[dst] = new
        elif LOAD.search(ln):
            assert "m0" in known, "an address that the test cannot follow"
            out.append(known["m0"])
        elif (m := WAIT.search(ln)):
            if out and int(m.group(1)) == wait:
                return out
    raise AssertionError("no such wait")


def check(lines, head_dim):
    stage = 64 * 2 * head_dim  # 32 keys' K and V
    seq = [p // stage for p in places(lines, 2 * head_dim // 32)]
    n = seq.count(3)
    assert seq == [0] * (n // 2) + [1] * n + [2] * n + [3] * n and n, seq


@pytest.mark.parametrize("head_dim", [64, 128, 256])
def test_stages_go_out_in_order(tmp_path, head_dim):
    tools = [LLVM + t for t in ("llvm-objdump", "llvm-readelf")]
    if not os.path.exists(LIB) or not all(shutil.which(t) for t in tools):
        pytest.skip("library or LLVM tools not here")
    lib = shutil.copy(LIB, tmp_path / "lib.so")
    subprocess.run([tools[0], "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    found = False
    for obj in sorted(p for p in os.listdir(tmp_path) if p.endswith("gfx950")):
        sym = subprocess.run([tools[1], "-sW", obj], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        for name in re.findall(rf"FUNC.*\s(\S*k_tree_manyILi{head_dim}E\S*)", sym):
            text = subprocess.run([tools[0], "-d", "--no-show-raw-insn", f"--disassemble-symbols={name}", obj],
                                  cwd=tmp_path, check=True, capture_output=True, text=True).stdout
            check(text.splitlines(), head_dim)
            found = True
    assert found


def test_check_sees_a_moved_load():
    """The check refuses a listing in which a load of a later stage went out
    before one that the first wait is for."""
    stage, load = 64 * 2 * 64, "buffer_load_dwordx4 v2, s[12:15], 0 offen lds"
    head = ["s_lshl_b32 s9, s3, 10"]

    def at(i):
        return [f"s_add_i32 s8, s9, {hex(i * stage)}", "s_mov_b32 m0, s8", load]

    def listing(order):
        return head + [ln for i in order for ln in at(i)] + ["s_waitcnt vmcnt(4)", "s_barrier"]

    check(listing([0, 1, 1, 2, 2, 3, 3]), 64)
    with pytest.raises(AssertionError):
        check(listing([0, 1, 2, 1, 2, 3, 3]), 64)
    with pytest.raises(AssertionError):
        check(listing([0, 1, 1, 2, 3, 2, 3]), 64)
