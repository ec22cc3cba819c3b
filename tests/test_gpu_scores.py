"""Attention with shaped scores on the GPU, through the binding, against 64
bits (scores_util, where the tolerances stand): caps, slopes over the distance,
windows, spans, trees with depths, and what those leave of a row."""
import numpy as np
import pytest
import torch

import scores_util as S
from test_gpu_paged import T16, T32, V, Dev, filled, i32, pack, rounded, say, tree_mask, vals  # noqa: F401

pytestmark = pytest.mark.gpu


def depths(rng, order, counts, kind):
    if kind == "any":
        return rng.integers(-2, 40, sum(counts))
    out = []
    for c in counts:
        d = []
        for j in range(c):
            d.append(0 if j < 3 else d[int(rng.integers(0, j))] + 1)
        out += d
    return np.array(out, np.int64)


# T, hd, nq, nkv, page, cap, bias, window, span, tree (mask and depths), lens, rows
CASES = [
    (T16, 64, 1, 1, 16, 5.0, False, 0, None, None, [0], [1]),
    (T16, 256, 8, 1, 32, 50.0, False, 0, None, None, [305, 420, 31, 0], [1, 1, 1, 1]),
    (T16, 128, 32, 8, 64, 0.0, True, 0, None, None, [127, 128, 1290], [1, 1, 1]),
    (T16, 64, 4, 1, 16, 3.0, True, 7, None, None, [0, 1, 15, 16, 17, 31, 33, 500], [1] * 8),
    (T16, 128, 8, 2, 16, 0.0, False, 200, None, None, [1000, 3, 130], [1, 2, 0]),
    (T16, 96, 6, 2, 16, 20.0, True, 33, None, "tree", [50, 0, 9], [61, 31, 1]),
    (T16, 128, 6, 2, 16, 20.0, True, 5, None, "any", [50, 0, 9], [61, 31, 1]),
    (T16, 64, 2, 2, 256, 0.0, True, 0, "any", None, [5, 0, 256], [70, 20, 33]),
    (T16, 256, 8, 1, 32, 10.0, True, 100, "docs", None, [300, 64, 0], [40, 33, 7]),
    (T16, 32, 4, 4, 16, 2.0, False, 0, "prefix", None, [0, 40], [9, 12]),
    # tiles of 128 rows
    (T16, 96, 5, 1, 16, 30.0, False, 40, None, None, [0, 70], [150, 33]),
    (T16, 128, 4, 1, 64, 15.0, True, 0, None, None, [500], [300]),
    (T16, 128, 8, 2, 16, 0.0, False, 64, None, None, [0, 700], [400, 350]),
    (T16, 128, 8, 2, 16, 4.0, True, 0, "docs", None, [30, 200], [300, 257]),
    (T16, 64, 4, 1, 32, 0.0, False, 0, "prefix", None, [10, 0], [190, 300]),
    (T16, 64, 8, 1, 32, 8.0, True, 50, "any", None, [100], [130]),
    (T16, 256, 16, 1, 128, 25.0, True, 90, None, None, [200], [170]),
    (T16, 256, 4, 1, 16, 25.0, False, 0, "docs", "tree", [70], [129]),
    (T16, 128, 16, 2, 16, 6.0, True, 17, None, "tree", [300, 0], [90, 40]),
    (T16, 160, 4, 2, 64, 0.0, True, 0, None, "any", [10], [290]),
    (T32, 64, 4, 1, 16, 4.0, True, 0, None, None, [0, 33, 17], [1, 1, 1]),
    (T32, 128, 8, 2, 32, 0.0, True, 25, None, "tree", [77, 0], [40, 12]),
    (T32, 96, 6, 2, 16, 2.5, False, 0, "any", None, [30, 0, 50], [61, 17, 3]),
    (T32, 128, 8, 1, 64, 12.0, True, 60, None, None, [5, 200], [64, 100]),
    (T32, 64, 8, 1, 16, 1.0, True, 30, "docs", None, [70, 0], [150, 41]),
    (T32, 96, 6, 1, 16, 6.0, True, 11, None, "any", [33], [91]),
    # caps that bend next to nothing
    (T16, 128, 8, 2, 16, 1e4, False, 0, None, None, [300, 20], [1, 1]),
    (T16, 64, 4, 1, 16, 1e4, False, 0, None, None, [100], [250]),
    (T32, 64, 4, 1, 16, 1e6, False, 0, None, None, [100], [25]),
    # groups that do not divide a step, or are longer than one
    (T16, 64, 40, 1, 16, 0.0, True, 0, None, None, [150, 0], [1, 20]),
    (T16, 128, 72, 1, 16, 7.0, False, 50, None, None, [90], [9]),
    (T32, 64, 80, 1, 16, 0.0, False, 0, None, None, [130], [3]),
    # capped, not biased, in tiles of 128 rows at the other head dims
    (T16, 64, 4, 1, 32, 9.0, False, 0, None, None, [50], [260]),
    (T16, 160, 4, 2, 16, 12.0, False, 33, "prefix", None, [20], [200]),
    (T16, 224, 3, 1, 16, 5.0, False, 0, None, "tree", [100], [90]),
    # tiles that many workgroups share, with the slots before a window left out
    (T16, 128, 8, 1, 64, 20.0, True, 20000, None, None, [30000], [2]),
    (T16, 64, 4, 1, 64, 20.0, False, 5000, None, None, [8000], [260]),
    (T16, 128, 16, 4, 64, 0.0, True, 0, None, None, [5000, 300, 9000], [1, 1, 1]),
    (T32, 64, 4, 2, 32, 0.0, False, 3000, None, None, [6000, 40], [1, 200]),
]


def batch(V, rng, T, hd, nq, nkv, page, cap, bias, window, span, tree, lens, rows):
    m = filled(rng, T, lens, rows, layers=2, nkv=nkv, page=page, hd=hd)
    used = np.zeros(m.dims[:4], bool)
    for s in range(len(lens)):
        for i in range(lens[s] + rows[s]):
            p, at = m.where(s, i)
            used[:, p, :, at] = True
    m.k[~used], m.v[~used] = np.nan, np.inf  # must not show
    order = list(rng.permutation(len(lens))) + [-1]
    counts = [rows[s] for s in order[:-1]] + [2]
    start = np.concatenate([[0], np.cumsum(counts)])
    n_rows = int(start[-1]) + 2
    q = rounded(rng.standard_normal((n_rows, nq, hd)) * 2.5, T)
    pad = lambda x: np.concatenate([x, np.zeros((2, *x.shape[1:]), x.dtype)])  # noqa: E731
    bits = depth = None
    if tree:
        words = (max(rows) + 31) // 32
        bits = np.concatenate([tree_mask(rng, c, words, "tree") for c in counts] + [np.ones((2, 32 * words), bool)])
        depth = pad(depths(rng, order, counts, tree))
    sc = S.Scores(hd ** -0.5, cap, rng.uniform(0.0, 0.6, nq).astype(np.float32) if bias else None, window, depth,
                  pad(S.spans(rng, lens, order, counts, span)) if span else None, bits)
    return m, order, counts, start, n_rows, q, sc


@pytest.mark.parametrize("T,hd,nq,nkv,page,cap,bias,window,span,tree,lens,rows", CASES)
def test_score_attention(V, T, hd, nq, nkv, page, cap, bias, window, span, tree, lens, rows):
    say(f"scores {T} hd={hd} nq={nq} nkv={nkv} page={page} cap={cap} bias={bias} window={window} span={span} "
        f"tree={tree} lens={lens} rows={rows}")
    rng = np.random.default_rng(hd * 5 + nq * 3 + len(lens) + sum(lens) + window)
    m, order, counts, start, n_rows, q, sc = batch(V, rng, T, hd, nq, nkv, page, cap, bias, window, span, tree, lens, rows)
    d = Dev(V, m, T)
    qd = torch.from_numpy(q).to(T).cuda()
    out = torch.full((n_rows, nq + 1, hd), 5.0, dtype=T, device="cuda")
    lse = torch.full((n_rows, nq), 5.0, device="cuda")
    mask = None if sc.bits is None else torch.from_numpy(pack(sc.bits)).cuda()
    r = V.make_rows(i32(start), n_rows, i32(order))
    scratch = torch.full((V.vla_score_attention_scratch(d.p, r, nq),), 255, dtype=torch.uint8, device="cuda")
    V.vla_score_attention(d.p, 1, r, sc.make(V, d.p, torch), qd, out[:, :nq], scratch, lse=lse, mask=mask)
    want, tol, ln, ltol = S.attention(m, T is T32, 1, order, start, counts, q, sc, n_rows / len(order))
    torch.cuda.synchronize()
    got, gl = vals(out), vals(lse)
    live = ~np.isnan(want)
    assert np.all(got[:, nq] == 5.0) and np.all(got[:, :nq][~live] == 5.0)
    off = np.abs(got[:, :nq][live] - want[live]) / tol[live]
    assert np.all(off <= 1), float(np.nanmax(off))
    rows_live = live[..., 0]
    assert np.all(gl[~rows_live] == 5.0)
    none = np.isneginf(ln)
    assert np.array_equal(np.isneginf(gl), none & rows_live)
    ok = rows_live & ~none
    off = np.abs(gl[ok] - ln[ok]) / ltol[ok]
    assert np.all(off <= 1), float(np.nanmax(off))
    d.same()


def weights_dev(rng, m, layers=2):
    slots = m.max_pages * m.page
    return rng.random((layers, m.n_seqs, m.dims[2], slots)).astype(np.float32)


@pytest.mark.parametrize("T,hd,nq,nkv,page,cap,bias,window,span,tree,lens,rows", CASES + [
    (T16, 128, 4, 1, 16, 0.0, False, 0, None, None, [3000], [1]),
    (T16, 64, 8, 8, 16, 0.0, False, 0, None, None, [2000, 130], [1, 1]),
    (T16, 128, 8, 1, 64, 0.0, False, 0, None, None, [0], [700]),
    (T32, 64, 3, 1, 16, 0.0, False, 0, None, None, [0, 129], [200, 5]),
])
def test_attention_mass(V, T, hd, nq, nkv, page, cap, bias, window, span, tree, lens, rows):
    say(f"mass {T} hd={hd} nq={nq} nkv={nkv} page={page} cap={cap} bias={bias} window={window} span={span} "
        f"tree={tree} lens={lens} rows={rows}")
    rng = np.random.default_rng(hd * 5 + nq * 3 + len(lens) + sum(lens) + window)
    m, order, counts, start, n_rows, q, sc = batch(V, rng, T, hd, nq, nkv, page, cap, bias, window, span, tree, lens, rows)
    d = Dev(V, m, T)
    qd = torch.from_numpy(q).to(T).cuda()
    lse = S.attention(m, T is T32, 1, order, start, counts, q, sc, 1)[2].astype(np.float32)
    lse[rng.random(lse.shape) < 0.05] = np.nan
    lse[rng.random(lse.shape) < 0.05] = np.inf
    mask = None if sc.bits is None else torch.from_numpy(pack(sc.bits)).cuda()
    r = V.make_rows(i32(start), n_rows, i32(order))
    scratch = torch.full((max(16, V.vla_attention_mass_scratch(d.p, r, nq)),), 255, dtype=torch.uint8, device="cuda")
    before = weights_dev(rng, m)
    # drafts' slots may hold anything
    for s in range(len(lens)):
        before[1, s, :, lens[s]:lens[s] + rows[s]] = np.nan
    mass = torch.from_numpy(before).cuda()
    V.vla_attention_mass(d.p, 1, r, sc.make(V, d.p, torch), qd, torch.from_numpy(lse).cuda(), mass, scratch, mask=mask)
    want, tol = S.mass(m, T is T32, 1, order, start, counts, q, sc, lse, before[1])
    torch.cuda.synchronize()
    got = mass.cpu().numpy()
    assert np.array_equal(got[0], before[0])
    left = tol == 0
    assert np.array_equal(got[1][left], before[1][left])
    off = np.abs(got[1][~left].astype(np.float64) - want[~left]) / tol[~left]
    assert np.all(off <= 1), float(np.nanmax(off))
    d.same()
