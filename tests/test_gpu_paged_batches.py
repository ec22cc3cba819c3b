"""Attention over pages for batches of more entries than a wave has lanes, with
caches so long that a tile is shared by several workgroups: as a server of many
sequences calls it, padded or not, eager or captured. Tolerances and the plain
64-bit form are those of test_gpu_paged.py. Rows start out as NaN, so a row that
nobody writes shows.
"""
import numpy as np
import pytest
import torch

import test_gpu_paged as P
from test_gpu_paged import T16, T32, V  # noqa: F401  (V is the fixture)

pytestmark = pytest.mark.gpu


class Batch:
    """Sequences of lens slots, and the rows of a step over them. seqs: the
    entries' sequences (-1: padding, with its rows)."""

    def __init__(self, V, seed, T, hd, nq, nkv, lens, seqs, rows, page=64, kind=None):
        rng = np.random.default_rng(seed)
        grow = [0] * len(lens)
        for s, n in zip(seqs, rows):
            if s >= 0:
                grow[s] = n
        self.V, self.T, self.hd, self.nq, self.seqs, self.rows = V, T, hd, nq, list(seqs), list(rows)
        self.m = P.filled(rng, T, lens, grow, nkv=nkv, page=page, hd=hd)
        self.d = P.Dev(V, self.m, T)
        self.start = np.concatenate([[0], np.cumsum(rows)])
        self.n = int(self.start[-1])
        self.q = P.rounded(rng.standard_normal((self.n, nq, hd)), T)
        self.qd = torch.from_numpy(self.q).to(T).cuda()
        self.bits = self.mask = None
        if kind:
            words = (max(rows) + 31) // 32
            self.bits = np.concatenate([P.tree_mask(rng, c, words, kind) for c in rows])
            self.mask = torch.from_numpy(P.pack(self.bits)).cuda()
        self.seqs_d = P.i32(self.seqs)
        self.r = V.make_rows(P.i32(self.start), self.n, self.seqs_d)
        size = V.vla_tree_attention_scratch(self.d.p, self.r, nq)
        self.scratch = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        self.out = torch.full((self.n, nq, hd), float("nan"), dtype=T, device="cuda")

    def attend(self, stream=0):
        self.V.vla_tree_attention(self.d.p, 0, self.r, self.qd, self.out, self.scratch, mask=self.mask, stream=stream)

    def check(self, what=""):
        torch.cuda.synchronize()
        want, tol = P.expect(self.m, self.T, 0, self.seqs, self.start, self.rows, self.q, self.bits, self.hd ** -0.5,
                             self.n / len(self.seqs))
        got, live = P.vals(self.out), ~np.isnan(want)
        assert np.all(np.isnan(got[~live])), what  # (padding's rows are left as they were)
        assert not np.isnan(got[live]).any(), f"{what}: rows that nobody wrote"
        off = np.abs(got[live] - want[live]) / tol[live]
        assert np.all(off <= 1), (what, float(off.max()))


@pytest.mark.parametrize("T,hd,nq,nkv,lens,rows,kind", [
    (T16, 128, 8, 1, [4000] * 80, [1] * 80, None),                       # tokens, all caches alike
    (T16, 128, 8, 1, [200] * 64 + [6000] * 36, [1] * 100, None),         # the last 64 are the longer ones
    (T16, 128, 8, 1, [6000] * 36 + [200] * 64, [1] * 100, None),         # and the shorter ones
    (T16, 64, 4, 1, [2000] * 96, [40] * 96, "tree"),                     # tiles of 128 rows, half full
    (T16, 128, 4, 1, [2000] * 96, [40] * 96, "tree"),
    (T16, 256, 8, 1, [1500] * 70, [20] * 70, "tree"),
    (T16, 64, 4, 2, [30] * 30 + [9000] + [5] * 60, [1] * 91, None),
    (T32, 64, 6, 2, [1500] * 66, [1] * 66, None),
    (T32, 128, 3, 1, [100] * 64 + [5000] * 6, [3] * 70, "tree"),
    (T32, 64, 8, 1, [700] * 66, [33] * 66, None),
])
def test_more_entries_than_lanes(V, T, hd, nq, nkv, lens, rows, kind):
    P.say(f"attend {len(lens)} entries {T} hd={hd} nq={nq} nkv={nkv} lens {min(lens)}..{max(lens)} rows {max(rows)}")
    b = Batch(V, len(lens) + hd, T, hd, nq, nkv, lens, range(len(lens)), rows, kind=kind)
    b.attend()
    b.check()
    first = b.out.clone()
    b.scratch.fill_(7)
    b.out.fill_(3.0)
    b.attend()
    assert torch.equal(b.out, first)
    b.d.same()


@pytest.mark.parametrize("live", [range(0, 20), range(108, 128), range(50, 70), [0, 127], []])
@pytest.mark.parametrize("T,hd,rows", [(T16, 128, 1), (T16, 64, 40), (T32, 64, 2)])
def test_padded_batches(V, T, hd, rows, live):
    """128 entries of which few are sequences."""
    P.say(f"attend padded {T} hd={hd} rows={rows} live={list(live)}")
    seqs = [-1] * 128
    for i, e in enumerate(live):
        seqs[e] = i
    lens = [3000 - 130 * i for i in range(max(1, len(list(live))))]
    b = Batch(V, hd + rows, T, hd, 4, 1, lens, seqs, [rows] * 128)
    b.attend()
    b.check()


def test_a_captured_batch_takes_other_sequences(V):
    """One captured call of 96 entries, replayed while sequences come and go."""
    P.say("captured batch of 96 entries")
    lens = [50 + 61 * i for i in range(96)]
    b = Batch(V, 5, T16, 128, 8, 1, lens, range(96), [1] * 96)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        g.capture_begin()
        b.attend(side.cuda_stream)
        g.capture_end()
    torch.cuda.synchronize()
    rng = np.random.default_rng(2)
    for alive in (96, 7, 70, 1, 0, 96):
        b.seqs = [-1] * 96
        for i, e in enumerate(rng.permutation(96)[:alive]):
            b.seqs[e] = int(rng.permutation(96)[0]) if alive == 1 else i
        b.seqs_d.copy_(P.i32(b.seqs))
        b.out.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        b.check(f"{alive} alive")
        torch.ones(1000, device="cuda").sum().item()
