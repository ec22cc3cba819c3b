"""Attention over pages in fp32 with tiles of 128 rows (more than 256 rows of a
KV head to a sequence, on average): masks, rows that see nothing, odd values in
masked and in seen places, odd queries, parts that are joined. Each test makes
sure that its batch is of those. Tolerances as in test_gpu_paged.py.
"""
import numpy as np
import pytest
import torch

import test_gpu_paged as P
from test_gpu_paged import T32, V  # noqa: F401  (V is the fixture)

pytestmark = pytest.mark.gpu


def tall(V, d, r, nq):
    """Scratch for this batch, whose tiles have 128 rows: four times the
    workspace of the same entries with a row each, whose tiles have 32."""
    size = V.vla_tree_attention_scratch(d.p, r, nq)
    few = V.make_rows(P.i32(np.arange(r._entries + 1)), r._entries)
    assert size > 3 * V.vla_tree_attention_scratch(d.p, few, d.p.kv_heads)
    return torch.full((size,), 255, dtype=torch.uint8, device="cuda")


ATTEND = [
    # hd, nq, nkv, page, mask, lens, rows
    (64, 16, 1, 16, "tree", [70, 0], [60, 41]),
    (64, 16, 1, 64, "random", [33], [61]),
    (32, 12, 1, 16, "random", [5, 300], [50, 49]),
    (96, 12, 1, 16, "random", [33, 90], [61, 40]),
    (96, 24, 2, 32, "tree", [0, 41], [33, 64]),
    (128, 16, 1, 32, "tree", [77, 300], [45, 40]),
    (128, 32, 2, 16, "random", [31, 32, 0], [30, 31, 33]),
    (128, 8, 1, 64, None, [5, 200], [100, 60]),
    (96, 8, 1, 16, None, [0, 47], [97, 70]),
    (64, 8, 1, 128, None, [1], [129]),
]


@pytest.mark.parametrize("hd,nq,nkv,page,kind,lens,rows", ATTEND)
def test_masks(V, hd, nq, nkv, page, kind, lens, rows):
    P.say(f"attend fp32 tall hd={hd} nq={nq} nkv={nkv} page={page} mask={kind} lens={lens} rows={rows}")
    rng = np.random.default_rng(hd * 5 + nq * 3 + sum(lens))
    m = P.filled(rng, T32, lens, rows, nkv=nkv, page=page, hd=hd)
    d = P.Dev(V, m, T32)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = int(start[-1])
    q = P.rounded(rng.standard_normal((n, nq, hd)) * 1.5, T32)
    bits = mask = None
    if kind:
        bits = np.concatenate([P.tree_mask(rng, c, (max(rows) + 31) // 32, kind) for c in rows])
        mask = torch.from_numpy(P.pack(bits)).cuda()
    r = V.make_rows(P.i32(start), n)
    out = torch.full((n, nq, hd), float("nan"), device="cuda")
    scratch = tall(V, d, r, nq)
    for scale in (hd ** -0.5, 0.31):
        V.vla_tree_attention(d.p, 0, r, torch.from_numpy(q).to(T32).cuda(), out, scratch, mask=mask, scale=scale)
        torch.cuda.synchronize()
        want, tol = P.expect(m, T32, 0, range(len(lens)), start, rows, q, bits, scale, n / len(lens))
        off = np.abs(P.vals(out) - want) / tol
        assert np.all(off <= 1), float(np.nanmax(off))
    d.same()


@pytest.mark.parametrize("hd", [64, 96, 128])
@pytest.mark.parametrize("lens,rows", [(37, 90), (3000, 40)])
def test_masked_drafts_may_hold_anything(V, hd, lens, rows):
    P.say(f"odd drafts fp32 tall hd={hd} len={lens} rows={rows}")
    rng = np.random.default_rng(rows + hd)
    nq = 16
    m = P.filled(rng, T32, [lens], [rows], hd=hd)
    bad = {3: (np.nan, None), 7: (None, np.inf), 11: (None, np.nan), 12: (np.inf, None), 25: (-np.inf, -np.inf)}
    for j, (a, b) in bad.items():
        p, at = m.where(0, lens + j)
        if a is not None:
            m.k[0, p, 0, at, 5] = a
        if b is not None:
            m.v[0, p, 0, at, 9] = b
    d = P.Dev(V, m, T32)
    q = P.rounded(rng.standard_normal((rows, nq, hd)), T32)
    q[1] *= 64  # scores far apart
    r = V.make_rows(P.i32([0, rows]), rows)
    out = torch.full((rows, nq, hd), float("nan"), device="cuda")
    scratch = tall(V, d, r, nq)
    bits = np.zeros((rows, 32 * ((rows + 31) // 32)), bool)
    for j in range(rows):
        bits[j, j] = j not in bad
        bits[j, 0] = True
    bits[5, 7] = bits[6, 11] = True  # these see an odd draft
    qd = torch.from_numpy(q).to(T32).cuda()
    V.vla_tree_attention(d.p, 0, r, qd, out, scratch, mask=torch.from_numpy(P.pack(bits)).cuda())
    torch.cuda.synchronize()
    got = P.vals(out)
    m.k, m.v = (np.nan_to_num(x, nan=0, posinf=0, neginf=0) for x in (m.k, m.v))
    want, tol = P.expect(m, T32, 0, [0], [0], [rows], q, bits, hd ** -0.5, rows)
    clean = [j for j in range(rows) if j not in (5, 6)]
    assert np.all(np.abs(got[clean] - want[clean]) <= tol[clean])
    assert np.all(np.isposinf(got[5, :, 9])) and np.all(np.isnan(got[6, :, 9]))
    rest = [c for c in range(hd) if c != 9]
    for j in (5, 6):
        assert np.all(np.abs(got[j][:, rest] - want[j][:, rest]) <= tol[j][:, rest])
    # causal: rows in front of the first odd draft are clean, it and later ones are not
    V.vla_tree_attention(d.p, 0, r, qd, out, scratch)
    torch.cuda.synchronize()
    got = P.vals(out)
    assert np.all(np.isfinite(got[:3])) and np.all(np.isnan(got[3]))


@pytest.mark.parametrize("hd", [64, 96, 128])
def test_odd_queries_stay_alone(V, hd):
    P.say(f"odd queries fp32 tall hd={hd}")
    rng = np.random.default_rng(hd)
    rows, nq = 40, 16
    m = P.filled(rng, T32, [300], [rows], hd=hd, page=32)
    d = P.Dev(V, m, T32)
    q = P.rounded(rng.standard_normal((rows, nq, hd)), T32)
    odd = q.copy()
    odd[1, 0, 5], odd[2, 1, 9], odd[rows - 1, nq - 1, 0] = np.nan, np.inf, -np.inf
    r = V.make_rows(P.i32([0, rows]), rows)
    out = torch.full((rows, nq, hd), float("nan"), device="cuda")
    V.vla_tree_attention(d.p, 0, r, torch.from_numpy(odd).to(T32).cuda(), out, tall(V, d, r, nq))
    torch.cuda.synchronize()
    got = P.vals(out)
    want, tol = P.expect(m, T32, 0, [0], [0], [rows], q, None, hd ** -0.5, rows)
    spoilt = ~np.isfinite(odd).all(-1)
    assert spoilt.sum() == 3 and np.all(np.isnan(got[1, 0]))
    assert np.all(np.abs(got - want)[~spoilt] <= tol[~spoilt])


@pytest.mark.parametrize("hd,nq,nkv,lens,rows", [
    (128, 16, 1, [9000], [40]),                       # one tile shared by many workgroups
    (64, 16, 2, [12000, 100], [64, 33]),
    (96, 32, 8, [2500, 1900, 40], [90, 70, 100]),     # runs that begin and end inside tiles
    (128, 8, 1, [400] * 66, [40] * 66)])              # more entries than lanes
def test_shared_tiles(V, hd, nq, nkv, lens, rows):
    P.say(f"shared tiles fp32 tall hd={hd} nq={nq} nkv={nkv} entries={len(lens)}")
    rng = np.random.default_rng(hd + nq)
    m = P.filled(rng, T32, lens, rows, nkv=nkv, page=64, hd=hd)
    d = P.Dev(V, m, T32)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = int(start[-1])
    q = P.rounded(rng.standard_normal((n, nq, hd)), T32)
    qd = torch.from_numpy(q).to(T32).cuda()
    r = V.make_rows(P.i32(start), n)
    scratch, outs = tall(V, d, r, nq), []
    for fill in (255, 0):
        scratch.fill_(fill)
        outs.append(torch.full((n, nq, hd), float("nan"), device="cuda"))
        V.vla_tree_attention(d.p, 0, r, qd, outs[-1], scratch)
    torch.cuda.synchronize()
    want, tol = P.expect(m, T32, 0, range(len(lens)), start, rows, q, None, hd ** -0.5, n / len(lens))
    off = np.abs(P.vals(outs[0]) - want) / tol
    assert np.all(off <= 1), float(np.nanmax(off))
    assert torch.equal(outs[0], outs[1])
