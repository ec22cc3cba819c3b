"""Reserving pages for a batch whose start array is not one: what an entry asks
for is bounded, and no page is given that the pool does not have."""
import pytest
import torch

import test_gpu_paged as P
from test_gpu_paged import T16, V  # noqa: F401  (V is the fixture)

pytestmark = pytest.mark.gpu


def test_entries_that_ask_for_more_than_31_bits_of_pages(V):
    """Every other entry names all 2^28 rows: 2^31 + 512 pages between them."""
    P.say("reserve, start up and down")
    n, wide, pool = 1024, (1 << 22) + 1, 100
    table = torch.full((n, wide), -1, dtype=torch.int32, device="cuda")  # 17 GB
    k = torch.zeros((1, pool, 1, 16, 32), dtype=T16, device="cuda")
    lens, held, refs, status = P.i32([0] * n), P.i32([0] * n), P.i32([0] * pool), P.i32([0])
    p = V.make_pages(k, k.clone(), table, lens, held, refs, status)
    start = P.i32([(e % 2) << 28 for e in range(n + 1)])
    V.vla_pages_reserve(p, V.make_rows(start, 1 << 28))
    torch.cuda.synchronize()
    assert held.tolist() == [pool] + [0] * (n - 1) and status.item() == V.PAGES_OUT
    assert table[0, :pool].tolist() == list(range(pool)) and refs.tolist() == [1] * pool
    assert not (table[1:] + 1).any() and not (table[0, pool:] + 1).any()
    assert not lens.any()
