"""Shaped scores over a paged cache in 64-bit NumPy, with what their errors in
32 bits are at most, and batches of rows to try them on.

A score x is off by delta: the product's hd roundings, (hd + 4) 2^-24 scale
sum |q k|; the cap's. e^{2 y} (1 step, 2^-23, of which half reaches tanh), the
sum with 1, the reciprocal (1 step of at most 2) and the last product and sum
make 9 2^-24 of the cap, in bf16; fp32 takes its odd series below |y| = 1/2,
where seven roundings and the terms that are cut off (1.5 2^-24 of y) count
against the score itself, and above, where tanh y > 0.46, 9 / 0.46 = 20 of
them: 24 2^-24 |score|; so does bf16 with caps from 178 on. The slope times the distance 3 2^-24 of it, and 4 2^-24
of |x| and of |x - max|, which is what the exponential takes. A weight is then
off by a factor of e^delta.
"""
from __future__ import annotations

import numpy as np

E = 2.0 ** -24


class Scores:
    """What make_scores takes: scale, cap, slopes [nq], window, depth [rows],
    span [rows, 2] (rows of the whole batch), and a mask's bits [rows, 32 words]."""

    def __init__(self, scale, cap=0.0, slopes=None, window=0, depth=None, span=None, bits=None):
        self.scale, self.cap, self.slopes, self.window = scale, cap, slopes, window
        self.depth, self.span, self.bits = depth, span, bits

    def make(self, V, pages, torch):
        def dev(x, T):
            return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(T).cuda()
        return V.make_scores(pages, scale=self.scale, cap=self.cap, slopes=dev(self.slopes, torch.float32),
                             window=self.window, depth=dev(self.depth, torch.int32), span=dev(self.span, torch.int32))


def seen(sc, L, end, a, c):
    """[c, end]: which slots rows a .. a + c - 1 of a sequence with L committed
    slots see, and the rows' and keys' places."""
    slot = np.arange(end)
    j = slot - L
    depth = np.arange(c) if sc.depth is None else np.maximum(sc.depth[a:a + c], 0)
    place = L + depth
    key = np.where(j < 0, slot, L + depth[np.clip(j, 0, max(c - 1, 0))] if c else slot)
    see = np.ones((c, end), bool)
    if sc.bits is not None:
        most = sc.bits.shape[1]
        see &= (j < 0) | ((j < most) & sc.bits[a:a + c][:, np.clip(j, 0, most - 1)])
    elif sc.span is None:
        see &= j[None, :] <= np.arange(c)[:, None]
    if sc.span is not None:
        see &= (slot >= sc.span[a:a + c, :1]) & (slot < sc.span[a:a + c, 1:])
    gap = place[:, None] - key[None, :]
    if sc.window:
        see &= gap < sc.window
    return see, gap


def scores(m, fp32, layer, s, a, c, q, h, sc):
    """Scores of rows a .. a + c - 1 with sequence s and KV head h: x [c,
    group, end], delta, see [c, end], and the values [end, hd]. Slots without a
    page are not seen."""
    hd, group = q.shape[2], q.shape[1] // m.dims[2]
    L, cap = int(m.lens[s]), int(m.held[s]) * m.page
    end = min(L + c, cap)
    see, gap = seen(sc, L, end, a, c)
    ids = m.table[s][np.arange(end) // m.page]
    see = see & (ids >= 0)[None, :]
    pages, places = np.maximum(ids, 0), np.arange(end) % m.page
    shown = see.any(0)
    k = np.where(shown[:, None], m.k[layer, pages, h, places], 0)
    v = np.where(shown[:, None], m.v[layer, pages, h, places], 0)
    qh = q[a:a + c, h * group:(h + 1) * group]
    x = np.matmul(qh, k.T) * sc.scale
    delta = np.matmul(np.abs(qh), np.abs(k).T) * sc.scale * (hd + 4) * E
    if sc.cap:
        x = sc.cap * np.tanh(x / sc.cap)
        delta = delta + (24 * E * np.abs(x) if fp32 or sc.cap >= 178 else 9 * E * sc.cap)
    if sc.slopes is not None:
        b = sc.slopes[h * group:(h + 1) * group].astype(np.float64)[None, :, None] * np.abs(gap)[:, None, :]
        x = x - b
        delta = delta + 3 * E * np.abs(b)
    top = np.where(see[:, None], x, -np.inf).max(-1, keepdims=True, initial=-np.inf)
    top = np.where(np.isfinite(top), top, 0)
    delta = delta + 4 * E * (np.abs(x) + np.abs(x - top))
    return np.where(see[:, None], x, -np.inf), np.where(see[:, None], delta, 0), see, v


def attention(m, fp32, layer, order, start, counts, q, sc, mean_rows):
    """Results and log-sum-exps of every row with their tolerances (rows of
    nobody: nan)."""
    nq, hd = q.shape[1:]
    group = nq // m.dims[2]
    half = E if fp32 else 2.0 ** -8
    one = 0.0 if fp32 else 2.0 ** -8 if mean_rows * group > (128 if hd > 64 else 192) else 2.0 ** -16
    want, tol = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, ltol = np.full(q.shape[:2], np.nan), np.full(q.shape[:2], np.nan)
    for s, a, c in zip(order, start, counts):
        if s < 0 or c == 0:
            continue
        for h in range(m.dims[2]):
            x, delta, see, v = scores(m, fp32, layer, s, a, c, q, h, sc)
            some = see.any(1)[:, None, None]
            top = np.where(some, x.max(-1, keepdims=True, initial=-np.inf), 0)
            p = np.exp(x - top)
            total = p.sum(-1, keepdims=True)
            with np.errstate(divide="ignore"):
                ln = np.log(total) + top
            p = p / np.where(some, total, 1)
            eps = np.expm1(delta) * p
            n = (x.shape[-1] + 16) * E
            o, mag = np.matmul(p, v), np.matmul(p, np.abs(v))
            es = eps.sum(-1, keepdims=True)
            to = np.matmul(eps, np.abs(v)) + np.abs(o) * es + (n + one) * (mag + np.abs(o))
            hs = slice(h * group, (h + 1) * group)
            want[a:a + c, hs], tol[a:a + c, hs] = o, to * 1.01 + half * (np.abs(o) + to) + 1e-37
            lse[a:a + c, hs] = ln[..., 0]
            ltol[a:a + c, hs] = (np.log1p(es + n) * 1.01 + 6 * E * (np.abs(top) + np.abs(np.where(some, ln, 0)) + 1))[..., 0]
    return want, tol, lse, ltol


def mass(m, fp32, layer, order, start, counts, q, sc, lse, before):
    """What vla_attention_mass makes of one layer's weights `before` [n_seqs,
    nkv, slots], in 64 bits, and the tolerance."""
    nkv = m.dims[2]
    group = q.shape[1] // nkv
    want, tol = before.astype(np.float64), np.zeros(before.shape)
    for s, a, c in zip(order, start, counts):
        if s < 0 or c == 0:
            continue
        L = int(m.lens[s])
        for h in range(nkv):
            x, delta, see, _ = scores(m, fp32, layer, s, a, c, q, h, sc)
            ln = lse[a:a + c, h * group:(h + 1) * group, None].astype(np.float64)
            with np.errstate(invalid="ignore"):
                p = np.where(np.isfinite(ln) & see[:, None], np.exp(x - np.where(np.isfinite(ln), ln, 0)), 0)
            err = (p * np.expm1(delta + 4 * E * np.abs(np.where(np.isfinite(ln), ln, 0)))).sum((0, 1))
            got = p.sum((0, 1))
            err = err + got * (c * group + 16) * E
            end = len(got)
            old = np.where(np.arange(end) < L, want[s, h, :end], 0)
            if sc.bits is not None:
                got, err = np.where(np.arange(end) < L, got, 0), np.where(np.arange(end) < L, err, 0)
            want[s, h, :end] = old + got
            tol[s, h, :end] = err * 1.01 + 2 * E * np.abs(old + got) + 1e-37
    return want, tol


def spans(rng, lens, order, counts, kind):
    """Spans [rows, 2]: documents, prefixes, or anything (empty ones, ones that
    lie outside the slots)."""
    out = []
    for s, c in zip(order, counts):
        n = int(lens[s]) if s >= 0 else 0
        cuts = [0]
        while cuts[-1] < n + c:
            cuts.append(cuts[-1] + int(rng.integers(1, 60)))
        pre = int(rng.integers(0, c + 1))
        for i in range(c):
            if kind == "docs":
                out.append((max(x for x in cuts if x <= n + i), n + i + 1))
            elif kind == "prefix":
                out.append((0, n + max(pre, i + 1)))
            else:
                lo, hi = sorted(int(x) for x in rng.integers(-5, n + c + 6, 2))
                out.append((hi, lo) if rng.random() < 0.2 else (lo, hi))
    return np.array(out, np.int64).reshape(-1, 2)
