"""What is no tensor, or no integer of 32 bits, is refused by name (CPU)."""
import numpy as np
import pytest
import torch

import paper_2609_22335_amd as V
from test_paged_binding import Dev, cache, on_device_0, refused  # noqa: F401

BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("bad", [None, 7, [1, 2], np.zeros((7, 4, 64), np.float32)])
def test_no_tensors(bad):
    p, r, rope = cache(), V.make_rows(Dev((3,)), 7), V.make_rope_norm()
    q, k, scr = Dev((7, 4, 64), BF), Dev((7, 2, 64), BF, ptr=0x90000), Dev((1 << 20,), torch.uint8, ptr=0x200000)
    refused("q must be a device", V.vla_tree_attention, p, 0, r, bad, q, scr)
    refused("out must be a device", V.vla_tree_attention, p, 0, r, q, bad, scr)
    refused("scratch must be a device", V.vla_tree_attention, p, 0, r, q, Dev((7, 4, 64), BF, ptr=0x50000), bad)
    refused("v must be a device", V.vla_qk_norm_rope, p, 0, r, rope, q, k, bad, q)
    refused("q_out must be a device", V.vla_qk_norm_rope, p, 0, r, rope, q, k, k, bad)
    refused("src must be", V.vla_pages_fork, p, bad, Dev((2,)), Dev((2,)))
    refused("seqs must be", V.vla_pages_release, p, bad)
    refused("start must be", V.make_rows, bad, 7)
    if bad is not None:
        refused("mask must be", V.vla_tree_attention, p, 0, r, q, Dev((7, 4, 64), BF, ptr=0x50000), scr, mask=bad)
        refused("cos must be", V.make_rope_norm, bad, bad)
        refused("q_gain must be", V.make_rope_norm, q_gain=bad)


@pytest.mark.parametrize("bad", [1 << 32, -(1 << 32), 1 << 31, "0", 0.5, float("inf"), None])
def test_no_integers_of_32_bits(bad):
    """(2^32 would be layer 0 and sequence 0)"""
    p, r = cache(), V.make_rows(Dev((3,)), 7)
    q, k, scr = Dev((7, 4, 64), BF), Dev((7, 2, 64), BF, ptr=0x90000), Dev((1 << 20,), torch.uint8, ptr=0x200000)
    refused("layer", V.vla_tree_attention, p, bad, r, q, Dev((7, 4, 64), BF, ptr=0x50000), scr)
    refused("layer", V.vla_qk_norm_rope, p, bad, r, V.make_rope_norm(), q, k, k, q)
    refused("nq", V.vla_tree_attention_scratch, p, r, bad)
    refused("n_rows", V.make_rows, Dev((3,)), bad)
    refused("seq", V.vla_ctx_to_pages, 1, 1, p, bad)


@pytest.mark.parametrize("n", [7, 7.0, np.int64(7), np.float64(7), torch.tensor(7)])
def test_integers_of_any_kind(n):
    assert V.make_rows(Dev((3,)), n).n_rows == 7
