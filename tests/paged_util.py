"""A paged cache in plain Python and 64-bit NumPy, and device tensors of one.

The model follows the definitions one token at a time: pages are handed out
lowest first, sequences are served in order, full pages are shared by a fork.
"""
from __future__ import annotations

import numpy as np


class Model:
    """The cache's state and what each call does to it. k and v [layers,
    n_pages, nkv, page, hd] hold the values of the cache's own type."""

    def __init__(self, layers, n_pages, nkv, page, hd, n_seqs, max_pages):
        self.dims = (layers, n_pages, nkv, page, hd)
        self.page, self.n_pages, self.n_seqs, self.max_pages = page, n_pages, n_seqs, max_pages
        self.k = np.zeros(self.dims)
        self.v = np.zeros(self.dims)
        self.table = np.full((n_seqs, max_pages), -1, np.int32)
        self.lens = np.zeros(n_seqs, np.int32)
        self.held = np.zeros(n_seqs, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        self.status = 0

    def free(self):
        f = np.flatnonzero(self.refs == 0)
        return int(f[0]) if len(f) else None

    def where(self, s, slot):
        """Page and place of a slot, or None."""
        return (int(self.table[s, slot // self.page]), slot % self.page) if slot < self.held[s] * self.page else None

    def reserve(self, entries):
        """entries: (sequence, rows)"""
        dry = False
        for s, n in entries:
            if not 0 <= s < self.n_seqs:
                continue
            want = -(-(int(self.lens[s]) + n) // self.page)
            if want > self.max_pages:
                self.status |= 1
                want = self.max_pages
            while self.held[s] < want:
                p = None if dry else self.free()
                if p is None:
                    dry = True
                    self.status |= 1
                    break
                self.table[s, self.held[s]] = p
                self.refs[p] = 1
                self.held[s] += 1

    def fork(self, pairs):
        made, seen = [], set()
        children = {d for s, d in pairs}
        lens, held = self.lens.copy(), self.held.copy()
        for s, d in pairs:
            ok = (0 <= s < self.n_seqs and 0 <= d < self.n_seqs and s != d and held[d] == 0 and lens[d] == 0
                  and d not in seen and not (s in children and self._claims(pairs, s, lens, held)))
            if 0 <= s < self.n_seqs and 0 <= d < self.n_seqs and s != d and held[d] == 0 and lens[d] == 0:
                seen.add(d)
            made.append(ok)
        for i, (s, d) in enumerate(pairs):
            if not made[i]:
                continue
            full, part = divmod(int(lens[s]), self.page)
            if part:
                p = self.free()
                if p is None:
                    made[i] = False
                    self.status |= 1
                    continue
                self.refs[p] = 1
                q = self.table[s, full]
                self.table[d, full] = p
                for c in (self.k, self.v):
                    c[:, p, :, :part] = c[:, q, :, :part]
            for j in range(full):
                self.table[d, j] = self.table[s, j]
                self.refs[self.table[s, j]] += 1
            self.lens[d], self.held[d] = lens[s], full + (part > 0)
        return [int(m) for m in made]

    def _claims(self, pairs, s, lens, held):
        """Whether some pair may make s a child (an empty sequence that a
        valid pair names)."""
        return any(d == s and 0 <= a < self.n_seqs and a != d and held[d] == 0 and lens[d] == 0 for a, d in pairs)

    def commit(self, entries, kept):
        """entries: (sequence, rows); kept: their lists (None: nothing moves,
        counts given as numbers)"""
        for (s, n), lst in zip(entries, kept):
            if not 0 <= s < self.n_seqs:
                continue
            count = lst if isinstance(lst, int) else len(lst)
            good = count <= n and (isinstance(lst, int) or (all(0 <= x < n for x in lst)
                                                            and all(b > a for a, b in zip(lst, lst[1:]))))
            if not good:
                self.status |= 2
                continue
            base = int(self.lens[s])
            if not isinstance(lst, int):
                for j, x in enumerate(lst):
                    a, b = self.where(s, base + x), self.where(s, base + j)
                    if a and b and x != j:
                        for c in (self.k, self.v):
                            c[:, b[0], :, b[1]] = c[:, a[0], :, a[1]]
            cap = int(self.held[s]) * self.page
            if base + count > cap:
                self.status |= 1
            self.lens[s] = min(base + count, cap)

    def release(self, seqs):
        for s in seqs:
            if not 0 <= s < self.n_seqs:
                continue
            for j in range(int(self.held[s])):
                self.refs[self.table[s, j]] -= 1
                self.table[s, j] = -1
            self.lens[s] = self.held[s] = 0


def norm_rope(x, gain, eps, cos, sin, pos):
    """x [heads, hd] in 64 bits: RMSNorm (gain None: none), then the rotation
    of the first 2 len(cos row) elements. Also what its absolute error scales
    with: the sum of the magnitudes that each result adds."""
    x = np.asarray(x, np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    size = np.abs(x)
    if cos is not None:
        half = cos.shape[1]
        c, s = cos[pos].astype(np.float64), sin[pos].astype(np.float64)
        a, b = x[..., :half].copy(), x[..., half:2 * half].copy()
        size = size.copy()
        size[..., :half] = np.abs(a * c) + np.abs(b * s)
        size[..., half:2 * half] = np.abs(b * c) + np.abs(a * s)
        x = x.copy()
        x[..., :half], x[..., half:2 * half] = a * c - b * s, b * c + a * s
    return x, size


def attention_row(q, k, v, see, scale):
    """One query [hd] over keys [n, hd] that `see` names, in 64 bits: the
    result, sum_j p_j |v_j|, and the largest sum_d |q_d k_d| scale."""
    idx = np.flatnonzero(see)
    if not len(idx):
        z = np.zeros(v.shape[1])
        return z, z, 0.0
    kk, vv = k[idx], v[idx]
    s = kk @ q * scale
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ vv, p @ np.abs(vv), float((np.abs(kk) @ np.abs(q)).max() * scale)
