"""Sequences of a paged cache cut back to their weightiest slots, on the GPU
through the binding, against a plain model: which slots stay, where their K, V
and weights go, which pages are freed, shared and replaced. All of it bit for
bit; weights are summed in 64 bits on both sides. (Of n weights in 32 bits
the sums in two orders differ by n 2^-53 of them at most; weights here are drawn
at random, or whole numbers whose sums have no error, so that no two sums lie
that close without being equal.)"""
import numpy as np
import pytest
import torch

from test_gpu_paged import T16, T32, V, Dev, filled, i32, say, vals  # noqa: F401

pytestmark = pytest.mark.gpu


def evict(m, seqs, keep, first, last, mass, out, kept):
    """The definition, one sequence after another. mass and out [layers,
    n_seqs, nkv, slots], kept [n, slots]."""
    seen, plans = set(), []
    refs0 = m.refs.copy()
    total = np.zeros(mass.shape[1::2], np.float64)
    for layer in mass:
        for h in range(mass.shape[2]):
            total += layer[:, h].astype(np.float64)
    free = [p for p in range(m.n_pages) if m.refs[p] == 0]
    for i, (s, k) in enumerate(zip(seqs, keep)):
        if not 0 <= s < m.n_seqs or s in seen:
            continue
        seen.add(s)
        if k < 0:
            m.status |= 2
            continue
        n = int(m.lens[s])
        stay = list(range(n))
        if n > k:
            w = np.where(total[s, :n] > 0, total[s, :n], 0)
            key = [(0 if j < first or j >= n - last else 1, -w[j], j) for j in range(n)]
            key = [(a, 0 if a == 0 else b, j) for a, b, j in key]
            stay = sorted(j for _, _, j in sorted(key)[:k])
        fresh = {}
        if len(stay) < n:
            gap = min(set(range(n)) - set(stay))
            need = [p for p in range(gap // m.page, -(-len(stay) // m.page)) if refs0[m.table[s, p]] > 1]
            if len(need) > len(free):
                m.status |= 1
                stay = list(range(n))
            else:
                fresh = dict(zip(need, free))
                free = free[len(need):]
        plans.append((i, int(s), n, stay, fresh))
    k0, v0, old = m.k.copy(), m.v.copy(), mass.copy()
    for i, s, n, stay, fresh in plans:
        kept[i, :len(stay)] = stay
        cap = int(m.held[s]) * m.page
        out[:, s, :, :len(stay)] = old[:, s][..., stay]
        out[:, s, :, len(stay):cap] = 0
        if len(stay) == n:
            continue
        where = [(int(m.table[s, j // m.page]), j % m.page) for j in range(n)]
        for p, q in fresh.items():
            m.refs[m.table[s, p]] -= 1
            m.refs[q] = 1
            m.table[s, p] = q
        for r, j in enumerate(stay):
            to = (int(m.table[s, r // m.page]), r % m.page)
            for c, c0 in ((m.k, k0), (m.v, v0)):
                c[:, to[0], :, to[1]] = c0[:, where[j][0], :, where[j][1]]
        held = -(-len(stay) // m.page)
        for p in range(held, int(m.held[s])):
            m.refs[m.table[s, p]] -= 1
            m.table[s, p] = -1
        m.held[s], m.lens[s] = held, len(stay)


def check(V, m, T, seqs, keep, first, last, mass, inplace=False):
    d = Dev(V, m, T)
    slots = m.max_pages * m.page
    n = len(seqs)
    mt = torch.from_numpy(mass).cuda()
    want_out = mass.copy() if inplace else np.full_like(mass, 7.0)
    out = mt if inplace else torch.from_numpy(want_out.copy()).cuda()
    kept = torch.full((n, slots), -5, dtype=torch.int32, device="cuda")
    want_kept = np.full((n, slots), -5, np.int32)
    scratch = torch.full((V.vla_pages_evict_scratch(d.p, n),), 255, dtype=torch.uint8, device="cuda")
    V.vla_pages_evict(d.p, i32(seqs), i32(keep), mt, out, kept, scratch, first=first, last=last)
    evict(m, seqs, keep, first, last, mass, want_out, want_kept)
    d.same()
    assert np.array_equal(kept.cpu().numpy(), want_kept)
    assert np.array_equal(out.cpu().numpy(), want_out, equal_nan=True)
    if not inplace:
        assert np.array_equal(mt.cpu().numpy(), mass, equal_nan=True)
    return d


def weights(rng, m, kind):
    w = rng.random((m.dims[0], m.n_seqs, m.dims[2], m.max_pages * m.page)).astype(np.float32) ** 6
    if kind == "ties":
        w = np.round(w * 3).astype(np.float32)
    elif kind == "same":
        w[:] = 0.25
    elif kind == "odd":  # negative sums, zeros, NaN, infinities
        u = rng.random(w.shape[1::2])
        w[0, :, 0] = np.where(u < 0.1, np.nan, np.where(u < 0.2, -50, np.where(u < 0.25, np.inf, w[0, :, 0])))
        w[:, :, :][..., u[0] > 0.9] = 0
    elif kind == "tiny":
        w *= np.float32(1e-42)
    elif kind == "wide":
        w = (w * 10.0 ** rng.integers(-30, 30, w.shape[1:])).astype(np.float32)
    return w


CASES = [
    # T, layers, nkv, hd, page, lens, rows, keep, first, last, weights, in place
    (T16, 2, 1, 64, 16, [40, 1, 100], [5, 3, 0], [16, 1, 33], 2, 5, "", False),
    (T16, 3, 2, 128, 32, [700, 33, 0, 300], [40, 1, 2, 9], [100, 32, 5, 299], 4, 20, "", True),
    (T16, 1, 8, 128, 64, [1500], [0], [700], 0, 0, "wide", False),
    (T16, 2, 1, 256, 16, [1100, 64], [1, 1], [1099, 1], 1, 0, "ties", True),
    (T16, 2, 3, 32, 256, [900, 257], [7, 0], [513, 0], 7, 200, "ties", False),
    (T16, 2, 1, 96, 16, [333], [4], [50], 100, 100, "", True),
    (T16, 1, 2, 160, 16, [500, 20], [3, 3], [499, 19], 0, 1, "same", False),
    (T16, 1, 1, 224, 128, [800], [2], [400], 0, 0, "odd", True),
    (T32, 2, 2, 96, 16, [250, 16, 17], [3, 0, 0], [77, 15, 16], 3, 4, "odd", False),
    (T32, 1, 1, 128, 32, [2100], [30], [1300], 4, 64, "tiny", True),
    (T32, 1, 4, 32, 64, [1000, 999, 3], [0, 0, 0], [1, 998, 3], 0, 0, "wide", True),
    (T16, 1, 1, 64, 16, [9000], [1], [4100], 4, 128, "", False),
]


@pytest.mark.parametrize("T,layers,nkv,hd,page,lens,rows,keep,first,last,kind,inplace", CASES)
def test_evict(V, T, layers, nkv, hd, page, lens, rows, keep, first, last, kind, inplace):
    say(f"evict {T} layers={layers} nkv={nkv} hd={hd} page={page} lens={lens} keep={keep} {kind}")
    rng = np.random.default_rng(sum(lens) + hd)
    m = filled(rng, T, lens, rows, layers=layers, nkv=nkv, page=page, hd=hd, extra_seqs=1)
    # entries in another order, one of them padding, one listed again, one refused
    order = list(rng.permutation(len(lens)))
    seqs = order + [-1, order[0], m.n_seqs, len(lens)]
    check(V, m, T, seqs, [keep[s] for s in order] + [3, 0, 1, -2], first, last, weights(rng, m, kind), inplace)


@pytest.mark.parametrize("inplace", [False, True])
def test_shared_pages_are_replaced(V, inplace):
    """Children share the full pages of their parents; those that would be
    written to, or would be left half full, become pages of their own. Both
    sequences of a page may be cut in one call; where pages run out, a sequence
    stays as it is."""
    rng = np.random.default_rng(3)
    for spare in (60, 9, 0):
        m = filled(rng, T16, [200, 90, 64], [4, 4, 0], layers=2, nkv=2, page=16, hd=64, spare=spare + 2, extra_seqs=3)
        m.fork([(0, 3), (1, 4), (2, 5)])
        say(f"evict shared spare={spare}")
        check(V, m, T16, [3, 0, 4, 2], [77, 40, 89, 33], 20, 6, weights(rng, m, ""), inplace)
        check(V, m, T16, [5, 1, 0], [64, 5, 16], 0, 0, weights(rng, m, "ties"), inplace)


def test_many_sequences(V):
    """More sequences than threads that list pages, all of them short."""
    say("evict 1300 sequences")
    rng = np.random.default_rng(8)
    lens = [int(x) for x in rng.integers(0, 40, 1300)]
    m = filled(rng, T16, lens, [1] * 1300, layers=1, nkv=1, page=16, hd=32)
    check(V, m, T16, list(rng.permutation(1300)), [int(x) for x in rng.integers(0, 30, 1300)], 1, 3, weights(rng, m, ""))
