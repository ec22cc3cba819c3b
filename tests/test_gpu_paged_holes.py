"""Attention where a sequence's table has no page for slots in front of its last
one (no entry, or one outside the pool): such slots are not seen, whatever the
kernel, and what lies beside them is seen as ever. Tolerances as in
test_gpu_paged.py.
"""
import numpy as np
import pytest
import torch

import test_gpu_paged as P
from test_gpu_paged import T16, T32, V  # noqa: F401  (V is the fixture)

pytestmark = pytest.mark.gpu


def expect(m, T, s, a, c, q, bits, scale, mean_rows, gone):
    """Entry s's rows a .. a + c - 1 in 64 bits; the places in `gone` (indices of
    the table) have no page."""
    nq, hd = q.shape[1:]
    nkv = m.dims[2]
    group, L, end = nq // nkv, int(m.lens[s]), int(m.lens[s]) + c
    at = np.arange(end)
    pages, places = m.table[s][at // m.page], at % m.page
    see = np.ones((c, end), bool)
    j = at[L:] - L
    see[:, L:] = j <= np.arange(c)[:, None] if bits is None else bits[a:a + c][:, j]
    see &= ~np.isin(at // m.page, list(gone))
    want, tol = np.empty((c, nq, hd)), np.empty((c, nq, hd))
    some = see.any(1)[:, None, None]
    see = see[:, None, :]
    for h in range(nkv):
        k, v = m.k[0, pages, h, places], m.v[0, pages, h, places]
        x = q[a:a + c, h * group:(h + 1) * group]
        score = np.where(see, np.matmul(x, k.T) * scale, -np.inf)
        p = np.exp(score - np.where(some, score.max(-1, keepdims=True), 0))
        p /= np.where(some, p.sum(-1, keepdims=True), 1)
        o, mag = np.matmul(p, v), np.matmul(p, np.abs(v))
        ds = np.where(see, np.matmul(np.abs(x), np.abs(k).T), 0).max(-1)[..., None] * scale * (hd + 4) * 2.0 ** -24
        one = 0.0 if T is T32 else 2.0 ** -8 if mean_rows * group > (128 if hd > 64 else 192) else 2.0 ** -16
        rel = np.expm1(2 * ds) + (end + 16) * 2.0 ** -24 + one
        want[:, h * group:(h + 1) * group] = o
        tol[:, h * group:(h + 1) * group] = rel * (mag + np.abs(o)) + P.HALF[T] * np.abs(o) * (1 + rel) + 1e-38
    return want, tol


# the tables' places without a page, for each sequence; page 16 is half a block
CASES = [
    # T, hd, nq, nkv, page, mask, lens, rows, gone
    (T16, 64, 4, 1, 16, None, [100, 40], [1, 1], [{1, 4}, {0}]),
    (T16, 128, 8, 2, 16, "tree", [300, 33], [20, 9], [{2, 9, 18}, {0, 1, 2}]),
    (T16, 256, 2, 1, 64, None, [700], [3], [{0, 5}]),
    (T32, 64, 2, 1, 16, "tree", [70, 20], [30, 12], [{3}, {1}]),
    (T32, 128, 2, 1, 32, None, [900], [1], [{20}]),
    (T16, 64, 8, 1, 16, None, [100, 40], [60, 50], [{1, 4, 8}, {0}]),          # tiles of 128 rows from here on
    (T16, 128, 8, 1, 16, "tree", [300, 33], [40, 39], [{2, 9, 18}, {0, 1, 2}]),
    (T16, 256, 8, 1, 32, None, [310], [40], [{0, 5}]),
    (T16, 256, 8, 1, 16, "tree", [290], [33], [{17}]),
    (T32, 64, 16, 1, 16, "tree", [70, 20], [40, 33], [{3}, {1}]),
    (T32, 128, 16, 1, 32, None, [900], [33], [{20, 28}]),
    (T32, 96, 8, 1, 16, None, [30], [70], [{1, 5}]),
    (T16, 64, 32, 8, 16, None, [3001, 1500], [300, 257], [{150}, {2}]),        # a run's later places
    (T16, 128, 16, 8, 32, None, [2500, 3100], [300, 260], [{70, 86}, {1, 40}]),
]


@pytest.mark.parametrize("T,hd,nq,nkv,page,kind,lens,rows,gone", CASES)
def test_slots_without_a_page_are_not_seen(V, T, hd, nq, nkv, page, kind, lens, rows, gone):
    P.say(f"holes {T} hd={hd} nq={nq} nkv={nkv} page={page} mask={kind} lens={lens} rows={rows}")
    rng = np.random.default_rng(hd + nq + sum(lens))
    m = P.filled(rng, T, lens, rows, nkv=nkv, page=page, hd=hd)
    d = P.Dev(V, m, T)
    n = sum(rows)
    q = P.rounded(rng.standard_normal((n, nq, hd)) * 1.3, T)
    qd = torch.from_numpy(q).to(T).cuda()
    bits, mask = None, None
    if kind:
        words = (max(rows) + 31) // 32
        bits = np.concatenate([P.tree_mask(rng, c, words, kind) for c in rows])
        mask = torch.from_numpy(P.pack(bits)).cuda()
    start = np.concatenate([[0], np.cumsum(rows)])
    r = V.make_rows(P.i32(start), n)
    scratch = torch.full((V.vla_tree_attention_scratch(d.p, r, nq),), 255, dtype=torch.uint8, device="cuda")
    table = m.table.copy()
    for s, g in enumerate(gone):
        for i, place in enumerate(sorted(g)):
            table[s, place] = (-1, m.n_pages, 2 ** 31 - 1)[i % 3]
    d.table.copy_(P.i32(table))

    def attend():
        out = torch.full((n, nq, hd), float("nan"), dtype=T, device="cuda")
        V.vla_tree_attention(d.p, 0, r, qd, out, scratch, mask=mask)
        torch.cuda.synchronize()
        return P.vals(out)

    got = attend()
    ends = {}
    for s, (a, c) in enumerate(zip(start, rows)):
        want, tol = ends[s] = expect(m, T, s, a, c, q, bits, hd ** -0.5, n / len(rows), gone[s])
        off = np.abs(got[a:a + c] - want) / tol
        assert np.all(off <= 1), (s, float(np.nanmax(off)))
    # an infinite value beside the first place without a page, on either side,
    # shows in its own column of every row (infinite, or NaN: a probability in two
    # bf16 values may count it with both signs), and nowhere else
    place = min(gone[0])
    want, tol = ends[0]
    rest = [i for i in range(hd) if i != 9]
    for slot in ((place + 1) * page, place * page - 1):
        if not 0 <= slot < lens[0] or slot // page in gone[0]:
            continue
        at = m.table[0, slot // page], slice(None), slot % page, 9
        d.v[0][at] = float("inf")
        got = attend()
        d.v[0][at] = torch.from_numpy(m.v[0][at]).to(d.v)
        assert not np.isfinite(got[:rows[0], :, 9]).any(), slot
        assert np.all(np.abs(got[:rows[0]] - want)[..., rest] <= tol[..., rest]), slot
    d.table.copy_(P.i32(m.table))
    d.same()
