"""A single row has no row stride: whatever its tensor says there is no ground
for a refusal. On the CPU, where a call that passes the checks ends at the
missing device."""
import os

import pytest
import torch

import paper_2609_22335_amd as V
from test_paged_binding import Dev, cache, on_device_0  # noqa: F401

pytestmark = pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="the addresses are made up: not beside a GPU")
BF = torch.bfloat16


@pytest.mark.parametrize("stride", [0, 1, 260, 512, 1 << 40])
@pytest.mark.parametrize("other", [256, 260, 4096])
def test_stride_of_a_single_row(stride, other):
    p, r = cache(), V.make_rows(Dev((2,)), 1)
    q, same = (Dev((1, 4, 64), BF, stride=(s, 64, 1), ptr=0x100000) for s in (stride, other))
    k = Dev((1, 2, 64), BF, stride=(stride, 64, 1), ptr=0x300000)
    for call in (lambda: V.vla_qk_norm_rope(p, 0, r, V.make_rope_norm(), q, k, k, same),
                 lambda: V.vla_tree_attention(p, 0, r, q, Dev((1, 4, 64), BF, stride=(other, 64, 1), ptr=0x200000),
                                              Dev((1 << 20,), torch.uint8, ptr=0x400000))):
        with pytest.raises(V.VlaError) as e:
            call()
        assert e.value.code == -3, str(e.value)
