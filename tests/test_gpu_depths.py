"""Rows whose places are given as depths and that no mask holds (chunks and
documents whose places do not follow their order), in windows and without, on
the GPU through the binding against 64 bits: what a row sees of its step's
drafts hangs on their places, one by one. Attention and slot weights have to
agree on it: the weights are taken with the log-sum-exps that the attention
wrote."""
import numpy as np
import pytest
import torch

import scores_util as S
from test_gpu_paged import T16, T32, V, filled, rounded, say  # noqa: F401
from test_gpu_scores_together import Call

pytestmark = pytest.mark.gpu


def depths(rng, counts, kind):
    """Rows in their order, in the reverse one, three places apart, or at any
    place (negative ones count as 0)."""
    make = {"order": np.arange, "back": lambda c: np.arange(c)[::-1], "apart": lambda c: 3 * np.arange(c),
            "any": lambda c: rng.integers(-2, 60, c)}[kind]
    return np.concatenate([make(c) for c in counts]).astype(np.int64)


# T, hd, nq, nkv, page, cap, bias, window, span, depth, lens, rows
CASES = [
    # tiles of 32 rows
    (T16, 64, 1, 1, 16, 0.0, False, 8, None, "order", [0], [64]),
    (T16, 64, 1, 1, 16, 0.0, False, 16, None, "order", [64, 5], [100, 70]),
    (T16, 128, 2, 1, 16, 5.0, False, 16, None, "any", [64, 0], [60, 58]),
    (T16, 96, 2, 2, 32, 0.0, True, 33, None, "apart", [7, 90], [110, 97]),
    (T16, 256, 2, 1, 64, 20.0, True, 64, "docs", "any", [30], [65]),
    (T16, 64, 3, 1, 16, 0.0, False, 9, "prefix", "back", [0, 33], [64, 61]),
    (T16, 64, 1, 1, 16, 0.0, False, 24, "any", "order", [40], [130]),
    (T16, 32, 2, 2, 16, 3.0, True, 0, None, "any", [20], [80]),
    (T32, 64, 2, 1, 16, 0.0, False, 8, None, "order", [0], [100]),
    (T32, 96, 2, 2, 16, 4.0, True, 40, "docs", "any", [70, 3], [97, 64]),
    # tiles of 128 rows
    (T16, 128, 4, 1, 16, 0.0, False, 8, None, "order", [0], [190]),
    (T16, 128, 4, 1, 64, 9.0, False, 32, None, "order", [70], [200]),
    (T16, 64, 4, 2, 32, 0.0, True, 17, None, "any", [33], [301]),
    (T16, 64, 4, 1, 16, 7.0, False, 50, "prefix", "order", [10, 0], [260, 170]),
    (T16, 256, 4, 1, 32, 25.0, False, 64, None, "apart", [100], [140]),
    (T16, 160, 4, 1, 16, 0.0, True, 20, "docs", "back", [65], [150]),
    (T16, 96, 8, 1, 16, 0.0, False, 40, "any", "any", [50], [129]),
    (T16, 128, 4, 1, 16, 1e4, False, 12, None, "any", [20], [200]),
    (T16, 128, 4, 1, 16, 0.0, False, 0, "prefix", "order", [20], [200]),
    (T32, 64, 8, 1, 16, 0.0, False, 16, None, "order", [0, 40], [150, 141]),
    (T32, 128, 8, 1, 32, 6.0, True, 48, "prefix", "any", [200], [120]),
    (T32, 96, 16, 2, 16, 2.0, False, 30, None, "back", [9], [170]),
    # windows as long as the rows' places reach, one shorter, and far longer
    (T16, 128, 4, 1, 16, 0.0, False, 150, None, "order", [90], [150]),
    (T16, 128, 4, 1, 16, 11.0, False, 149, None, "order", [90], [150]),
    (T16, 64, 1, 1, 16, 0.0, True, 69, None, "order", [33, 0], [70, 64]),
    (T16, 128, 4, 1, 16, 0.0, True, 300, None, "any", [400], [200]),
    (T32, 64, 8, 1, 16, 0.0, False, 99, "prefix", "order", [50], [100]),
]


@pytest.mark.parametrize("T,hd,nq,nkv,page,cap,bias,window,span,depth,lens,rows", CASES)
def test_depths_without_a_mask(V, T, hd, nq, nkv, page, cap, bias, window, span, depth, lens, rows):
    say(f"depths {T} hd={hd} nq={nq} nkv={nkv} cap={cap} bias={bias} window={window} span={span} depth={depth} "
        f"lens={lens} rows={rows}")
    rng = np.random.default_rng(hd + 7 * nq + window + sum(rows))
    m = filled(rng, T, lens, rows, nkv=nkv, page=page, hd=hd)
    order = [int(s) for s in rng.permutation(len(lens))]
    counts = [rows[s] for s in order]
    q = rounded(rng.standard_normal((sum(counts), nq, hd)) * 2, T)
    span = S.spans(rng, lens, order, counts, span) if span else None
    sc = S.Scores(hd ** -0.5, cap, rng.uniform(0.0, 0.4, nq).astype(np.float32) if bias else None, window,
                  depths(rng, counts, depth), span)
    call = Call(V, m, T, order, counts, q, sc)
    call.check()
    none = np.isneginf(S.attention(m, T is T32, 0, order, call.start, counts, q, sc, 1)[2])
    assert np.array_equal(np.isneginf(call.lse.cpu().numpy()), none)
    call.d.same()


@pytest.mark.parametrize("T,nq,rows", [(T16, 1, 100), (T16, 4, 150), (T32, 1, 90), (T32, 8, 140)])
def test_depths_of_the_order_change_nothing(V, T, nq, rows):
    """Rows that are given the places that they have anyway see what they see
    without, so results and log-sum-exps are the same up to a sum's order: both
    are within the tolerance of the same number."""
    say(f"depths of the order {T} nq={nq} rows={rows}")
    rng = np.random.default_rng(rows)
    m = filled(rng, T, [70], [rows], page=16, hd=64)
    q = rounded(rng.standard_normal((rows, nq, 64)) * 2, T)
    got = []
    for depth in (None, np.arange(rows)):
        sc = S.Scores(0.125, 0.0, None, 24, depth)
        c = Call(V, m, T, [0], [rows], q, sc)
        c.attend()
        torch.cuda.synchronize()
        got.append((c.out.double().cpu().numpy(), c.lse.double().cpu().numpy()))
    want, tol, ln, ltol = S.attention(m, T is T32, 0, [0], [0, rows], [rows], q, sc, rows)
    assert np.all(np.abs(got[0][0] - got[1][0]) <= 2 * tol)
    assert np.all(np.abs(got[0][1] - got[1][1]) <= 2 * ltol)
