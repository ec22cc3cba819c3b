"""What an infinite key does to the rows that see it: it enters by its score. A
score of minus infinity has no weight, so the slot is as good as hidden, and a
row with no other scores is zero; plus infinity and NaN make the row NaN.
Tolerances as in test_gpu_paged.py; each batch runs another kernel.
"""
import numpy as np
import pytest
import torch

import test_gpu_paged as P
from paged_util import attention_row
from test_gpu_paged import T16, T32, V  # noqa: F401  (V is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,hd,nq,rows", [(T16, 64, 2, 6), (T16, 128, 2, 6), (T16, 256, 2, 6), (T32, 64, 2, 6),
                                          (T32, 128, 2, 6), (T16, 64, 8, 40), (T16, 128, 8, 40), (T16, 256, 8, 40),
                                          (T32, 64, 16, 40), (T32, 128, 16, 40)])
@pytest.mark.parametrize("lens", [3, 150])
def test_infinite_keys(V, T, hd, nq, rows, lens):
    P.say(f"infinite keys {T} hd={hd} nq={nq} rows={rows} len={lens}")
    rng = np.random.default_rng(hd + rows + lens)
    m = P.filled(rng, T, [lens], [rows], hd=hd)
    d = P.Dev(V, m, T)
    q = P.rounded(rng.standard_normal((rows, nq, hd)), T)
    q[:, :, 5] = 1.0
    q[1, :, 5], q[2, :, 5] = -1.0, 0.0  # scores of +inf and NaN
    r = V.make_rows(P.i32([0, rows]), rows)
    scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, nq), dtype=torch.uint8, device="cuda")
    qd = torch.from_numpy(q).to(T).cuda()
    own = np.zeros((rows, 32 * ((rows + 31) // 32)), bool)
    own[np.arange(rows), np.arange(rows)] = True
    mask = torch.from_numpy(P.pack(own)).cuda()
    for slots in ([1], range(lens), range(lens + rows)):
        k = d.k.clone()
        for s in slots:
            p, at = m.where(0, s)
            d.k[0, p, 0, at, 5] = -float("inf")
        out = torch.full((rows, nq, hd), float("nan"), dtype=T, device="cuda")
        V.vla_tree_attention(d.p, 0, r, qd, out, scratch, mask=mask)
        torch.cuda.synchronize()
        d.k.copy_(k)
        got = P.vals(out)
        fine = [i for i in range(rows) if i not in (1, 2)]
        assert np.isnan(got[1]).all() and np.isnan(got[2]).all()
        # the other rows: the slots hidden
        gone = np.isin(np.arange(lens + rows), list(slots))
        for i in fine:
            see = np.zeros(lens + rows, bool)
            see[:lens] = True
            see[lens + i] = True
            see &= ~gone
            if not see.any():
                assert not got[i].any()
                continue
            pages, places = m.table[0][np.arange(lens + rows) // m.page], np.arange(lens + rows) % m.page
            kk, vv = m.k[0, pages, 0, places], m.v[0, pages, 0, places]
            for h in range(nq):
                o, mag, ds = attention_row(q[i, h], kk, vv, see, hd ** -0.5)
                one = 0.0 if T is T32 else 2.0 ** -8 if rows * nq > (128 if hd > 64 else 192) else 2.0 ** -16
                rel = np.expm1(2 * ds * (hd + 4) * 2.0 ** -24) + (lens + rows + 16) * 2.0 ** -24 + one
                off = np.abs(got[i, h] - o) - rel * (mag + np.abs(o)) - P.HALF[T] * np.abs(o) * (1 + rel)
                assert np.all(off <= 1e-38), (i, h, float(off.max()))
