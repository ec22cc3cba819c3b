"""Which layouts of its operands a call on the paged cache takes: every overlap
of what it writes with what it reads is refused, slices of one tensor that
share no element are not. Compared with the sets of bytes, on the CPU, where a
call that passes the checks ends at the missing device.
"""
import ctypes as C
import os
import random

import pytest
import torch

import paper_2609_22335_amd as V
from test_paged_binding import Dev, cache, on_device_0, refused  # noqa: F401

BF, I = torch.bfloat16, torch.int32
BASE = 0x100000
no_gpu = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="the addresses are made up: not beside a GPU")


def taken(p, ld, w, n):
    """The bytes of n rows of w elements of two bytes, ld elements apart."""
    return {p + 2 * (i * ld + j) for i in range(n) for j in range(0, w, 8)}


def layouts(seed, many):
    """Random places of rows: anywhere, or slices of rows of one width."""
    rng = random.Random(seed)
    for _ in range(many):
        n = rng.choice([1, 1, 2, 3, 5])
        wide = rng.choice([0, 160, 192, 256])
        out = []
        for heads in (2, 2, 1, 1):
            w = 32 * heads
            ld = wide or w + 8 * rng.randrange(0, 20)
            at = 8 * rng.randrange(0, (wide - w) // 8 + 1) if wide else 8 * rng.randrange(0, 60)
            out.append((BASE + 2 * at + 2 * ld * rng.randrange(0, n + 1) * (rng.random() < 0.3), ld, w))
        yield n, out


@no_gpu
@pytest.mark.parametrize("seed", range(3))
def test_overlaps_are_refused_and_slices_are_not(seed):
    p = cache(k=Dev((1, 10, 1, 16, 32), BF), v=Dev((1, 10, 1, 16, 32), BF))
    rope, seen = V.make_rope_norm(), {0: 0, 1: 0}
    for n, ((q, ldq, wq), (o, ldo, wo), (k, ldk, wk), (v, ldv, wv)) in layouts(seed, 3000):
        r = V.make_rows(Dev((2,)), n)
        bytes_o, bytes_q = taken(o, ldo, wo, n), taken(q, ldq, wq, n)
        clash = bool(bytes_o & bytes_q)
        rc = V._lib.vla_tree_attention(C.byref(p), 0, C.byref(r), None, 0, 2, 1.0, q, ldq, o, ldo, 0x900000, 1 << 30,
                                       None)
        assert rc == (-1 if clash else -3), (n, q, ldq, o, ldo, V.vla_last_error())
        seen[clash] += 1
        if q == o and (ldq == ldo or n == 1):
            clash = False
        clash = clash or bool(bytes_o & (taken(k, ldk, wk, n) | taken(v, ldv, wv, n)))
        rc = V._lib.vla_qk_norm_rope(C.byref(p), 0, C.byref(r), C.byref(rope), None, 2, q, ldq, k, ldk, v, ldv, o, ldo,
                                     None)
        assert rc == (-1 if clash else -3) or (q == o and ldq != ldo), (n, q, ldq, o, ldo, k, ldk, v, ldv)
    assert min(seen.values()) > 100, seen


def test_scratch_and_made_are_apart():
    p, r = cache(), V.make_rows(Dev((3,)), 7)
    q, out = Dev((7, 4, 64), BF, ptr=0x100000), Dev((7, 4, 64), BF, ptr=0x200000)
    for what in (0x100000, 0x200000, 0x100000 + 7 * 512 - 16, 0x200000 - 16):
        with pytest.raises(V.VlaError) as e:
            V.vla_tree_attention(p, 0, r, q, out, Dev((1 << 30,), torch.uint8, ptr=what))
        assert e.value.code in (-1, -3)  # (without a device the scratch's size is not known)
    a, b = Dev((4,), ptr=0x10000), Dev((4,), ptr=0x20000)
    for made in (0x10000, 0x1000C, 0x1FFF4, 0x2000C):
        refused("made must be an array of its own", V.vla_pages_fork, p, a, b, Dev((4,), ptr=made))
