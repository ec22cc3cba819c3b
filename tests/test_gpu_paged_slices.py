"""Operands of the paged cache's calls that are slices of one tensor, and
single rows of any stride."""
import numpy as np
import pytest
import torch

import test_gpu_paged as P
from test_gpu_paged import T16, T32, V  # noqa: F401  (V is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,n", [(T16, 21), (T32, 21), (T16, 1)])
def test_q_k_v_and_results_side_by_side(V, T, n):
    """One tensor holds a row's q, its normed q, k, v and the attention's result."""
    P.say(f"slices of one tensor {T} rows={n}")
    rng = np.random.default_rng(n)
    hd, nq, nkv = 64, 4, 2
    m = P.filled(rng, T, [40], [n], nkv=nkv, hd=hd)
    d = P.Dev(V, m, T)
    x = P.rounded(rng.standard_normal((n, 3 * nq + 2 * nkv, hd)), T)
    t = torch.from_numpy(x).to(T).cuda()
    q, qr, k, v, out = t[:, :nq], t[:, nq:2 * nq], t[:, 2 * nq:2 * nq + nkv], t[:, 2 * nq + nkv:2 * nq + 2 * nkv], \
        t[:, 2 * nq + 2 * nkv:]
    r = V.make_rows(P.i32([0, n]), n)
    V.vla_qk_norm_rope(d.p, 0, r, V.make_rope_norm(), q, k, v, qr)
    scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, nq), dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(d.p, 0, r, qr, out, scratch)
    torch.cuda.synchronize()
    for i in range(n):
        p, at = m.where(0, 40 + i)
        m.k[0, p, :, at], m.v[0, p, :, at] = x[i, 2 * nq:2 * nq + nkv], x[i, 2 * nq + nkv:2 * nq + 2 * nkv]
    want, tol = P.expect(m, T, 0, [0], [0], [n], x[:, :nq], None, hd ** -0.5, n)
    got = P.vals(t)
    assert np.array_equal(got[:, :nq], x[:, :nq]) and np.array_equal(got[:, nq:2 * nq], x[:, :nq])
    assert np.array_equal(got[:, 2 * nq:2 * nq + 2 * nkv], x[:, 2 * nq:2 * nq + 2 * nkv])
    assert np.all(np.abs(got[:, 2 * nq + 2 * nkv:] - want) <= tol)
    d.same()


def test_overlaps_are_refused(V):
    P.say("overlaps")
    rng = np.random.default_rng(3)
    m = P.filled(rng, T16, [5], [8], nkv=1, hd=64)
    d = P.Dev(V, m, T16)
    r = V.make_rows(P.i32([0, 8]), 8)
    t = torch.zeros((8, 10, 64), dtype=T16, device="cuda")
    big = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    inside = big[4096:4096 + 8 * 4 * 64 * 2].view(T16).reshape(8, 4, 64)
    for f in (lambda: V.vla_tree_attention(d.p, 0, r, t[:, :4], t[:, 3:7], big),
              lambda: V.vla_tree_attention(d.p, 0, r, t[:, :4], inside, big),
              lambda: V.vla_tree_attention(d.p, 0, r, inside, t[:, :4], big),
              lambda: V.vla_qk_norm_rope(d.p, 0, r, V.make_rope_norm(), t[:, :4], t[:, 5:6], t[:, 6:7], t[:, 2:6]),
              lambda: V.vla_qk_norm_rope(d.p, 0, r, V.make_rope_norm(), t[:, :4], t[:, 4:5], t[:, 5:6], t[:, 5:9])):
        with pytest.raises(V.VlaError) as e:
            f()
        assert e.value.code == -1 and "overlap" in str(e.value)
    d.same()
