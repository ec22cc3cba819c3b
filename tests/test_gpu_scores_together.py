"""Attention with shaped scores, slot weights, eviction and draft verification
on the GPU in what a step of a serving loop does with them: large batches,
padding, holes in a table, values that are not finite, strided rows, caches past
32 bits, other streams, and whole steps captured into a graph and replayed."""
import numpy as np
import pytest
import torch

import scores_util as S
from test_gpu_paged import T16, T32, V, Dev, filled, i32, pack, rounded, say, vals  # noqa: F401

pytestmark = pytest.mark.gpu


class Call:
    """A batch over a model, its calls, and what they have to give."""

    def __init__(self, V, m, T, order, counts, q, sc, extra=0):
        self.V, self.m, self.T, self.sc, self.q = V, m, T, sc, q
        self.order, self.counts = order, counts
        self.start = np.concatenate([[0], np.cumsum(counts)])
        self.n = int(self.start[-1]) + extra
        assert q.shape[0] == self.n
        self.d = Dev(V, m, T)
        self.rows = V.make_rows(i32(self.start), self.n, i32(order))
        self.scores = sc.make(V, self.d.p, torch)
        self.mask = None if sc.bits is None else torch.from_numpy(pack(sc.bits)).cuda()
        self.qd = torch.from_numpy(q).to(T).cuda()
        nq = q.shape[1]
        size = max(16, V.vla_score_attention_scratch(self.d.p, self.rows, nq),
                   V.vla_attention_mass_scratch(self.d.p, self.rows, nq))
        self.scratch = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        self.out, self.lse = torch.zeros_like(self.qd), torch.zeros((self.n, nq), device="cuda")

    def attend(self, qd=None, layer=0):
        self.V.vla_score_attention(self.d.p, layer, self.rows, self.scores, self.qd if qd is None else qd, self.out,
                                   self.scratch, lse=self.lse, mask=self.mask)

    def weigh(self, mass, qd=None, lse=None, layer=0):
        self.V.vla_attention_mass(self.d.p, layer, self.rows, self.scores, self.qd if qd is None else qd,
                                  self.lse if lse is None else lse, mass, self.scratch, mask=self.mask)

    def check(self):
        """Both calls against 64 bits."""
        f32 = self.T is T32
        self.attend()
        mean = self.n / len(self.order)
        want, tol, ln, ltol = S.attention(self.m, f32, 0, self.order, self.start, self.counts, self.q, self.sc, mean)
        live = ~np.isnan(want)
        off = np.abs(vals(self.out)[live] - want[live]) / tol[live]
        assert np.all(off <= 1), float(np.nanmax(off))
        ok = np.isfinite(ln)
        off = np.abs(vals(self.lse)[ok] - ln[ok]) / ltol[ok]
        assert np.all(off <= 1), float(np.nanmax(off))
        lse = self.lse.cpu().numpy()
        shape = (self.m.dims[0], self.m.n_seqs, self.m.dims[2], self.m.max_pages * self.m.page)
        before = np.random.default_rng(1).random(shape).astype(np.float32)
        mass = torch.from_numpy(before).cuda()
        self.weigh(mass)
        want, tol = S.mass(self.m, f32, 0, self.order, self.start, self.counts, self.q, self.sc, lse, before[0])
        got = mass.cpu().numpy()
        assert np.array_equal(got[0][tol == 0], before[0][tol == 0]) and np.array_equal(got[1:], before[1:])
        at = tol > 0
        off = np.abs(got[0][at].astype(np.float64) - want[at]) / tol[at]
        assert np.all(off <= 1), float(np.nanmax(off))


@pytest.mark.parametrize("T,rows,window,cap", [(T16, [1], 0, 0.0), (T16, [1, 2, 3], 30, 9.0), (T16, [40, 0, 70], 20, 0.0),
                                               (T32, [1, 0, 30], 50, 3.0), (T16, [1] * 8 + [40], 25, 0.0),
                                               (T32, [1] * 8 + [30], 0, 5.0)])
def test_more_entries_than_lanes(V, T, rows, window, cap):
    say(f"scores many entries {T} rows={rows} window={window}")
    rng = np.random.default_rng(sum(rows) + window)
    n = 150
    lens = [int(x) for x in rng.integers(0, 90, n)]
    counts = [int(rng.choice(rows)) for _ in range(n)]
    m = filled(rng, T, lens, counts, nkv=2, page=16, hd=64)
    # every third entry is padding, with rows that are nobody's
    order, cnt = [], []
    for s in rng.permutation(n):
        order.append(int(s)), cnt.append(counts[s])
        if len(order) % 3 == 0:
            order.append(-1), cnt.append(1)
    q = rounded(rng.standard_normal((sum(cnt), 4, 64)) * 2, T)
    Call(V, m, T, order, cnt, q, S.Scores(0.125, cap, rng.uniform(0, 0.3, 4).astype(np.float32), window)).check()


@pytest.mark.parametrize("T,rows", [(T16, 1), (T16, 90), (T32, 1), (T32, 100)])
def test_holes_in_a_table(V, T, rows):
    """Slots whose table entry is no page are not seen and receive nothing."""
    say(f"scores holes {T} rows={rows}")
    rng = np.random.default_rng(rows)
    m = filled(rng, T, [300, 64], [rows, rows], page=16, hd=64)
    m.table[0, [0, 3, 7]] = -1
    m.table[1, 1:4] = [-1, -5, m.n_pages]  # (out of the pool as well)
    model = m.table.copy()
    m.table = np.where((model < 0) | (model >= m.n_pages), -1, model)
    q = rounded(rng.standard_normal((2 * rows, 4, 64)) * 2, T)
    c = Call(V, m, T, [0, 1], [rows, rows], q, S.Scores(0.125, 4.0))
    c.d.table.copy_(i32(model))
    c.check()


@pytest.mark.parametrize("T,rows", [(T16, 2), (T16, 70), (T32, 3), (T32, 90)])
def test_values_that_are_not_finite(V, T, rows):
    """Masked slots may hold anything; a key that is not a number makes its rows
    NaN, and those give no slot anything."""
    say(f"scores odd values {T} rows={rows}")
    rng = np.random.default_rng(rows)
    lens = [100, 40]
    m = filled(rng, T, lens, [rows, rows], page=16, hd=64)
    q = rounded(rng.standard_normal((2 * rows, 4, 64)) * 2, T)
    span = np.array([(20, lens[s] + i + 1) for s in (0, 1) for i in range(rows)])
    sc = S.Scores(0.125, 0.0, None, 0, None, span)
    for s in (0, 1):  # nobody sees the first 20 slots
        for i in range(20):
            p, at = m.where(s, i)
            m.k[:, p, :, at], m.v[:, p, :, at] = np.nan, np.inf if i % 2 else np.nan
    Call(V, m, T, [0, 1], [rows, rows], q, sc).check()
    p, at = m.where(1, 25)
    m.k[0, p, 0, at, 3] = np.nan
    c = Call(V, m, T, [0, 1], [rows, rows], q, sc)
    c.attend()
    torch.cuda.synchronize()
    assert torch.isfinite(c.out[:rows].float()).all() and torch.isfinite(c.lse[:rows]).all()
    assert torch.isnan(c.out[rows:].float()).all() and torch.isnan(c.lse[rows:]).all()
    mass = torch.full((1, 2, 1, m.max_pages * 16), 0.5, device="cuda")
    c.weigh(mass)
    assert torch.isfinite(mass).all() and torch.all(mass[0, 1, 0, :40] == 0.5)
    assert torch.all(mass[0, 1, 0, 40:40 + rows] == 0)


@pytest.mark.parametrize("T,rows", [(T16, 1), (T16, 60), (T32, 40)])
def test_strided_queries(V, T, rows):
    """Queries sliced out of a fused product, and rows tens of MB apart, give
    what contiguous ones give (far ones take another kernel: to its tolerance)."""
    say(f"scores strided {T} rows={rows}")
    rng = np.random.default_rng(rows)
    m = filled(rng, T, [200], [rows], page=16, hd=64)
    q = rounded(rng.standard_normal((rows, 4, 64)) * 2, T)
    c = Call(V, m, T, [0], [rows], q, S.Scores(0.125, 0.0))
    wide = torch.randn((rows, 9, 64), device="cuda").to(T)
    wide[:, 2:6] = c.qd
    c.attend()
    out, lse = c.out.clone(), c.lse.clone()
    a, b = (torch.zeros((1, 1, 1, m.max_pages * 16), device="cuda") for _ in range(2))
    c.weigh(a)
    c.out.zero_(), c.lse.zero_()
    c.attend(wide[:, 2:6])
    c.weigh(b, wide[:, 2:6])
    assert torch.equal(out, c.out) and torch.equal(lse, c.lse) and torch.equal(a, b)
    if rows > 1:
        step = 36 * 2 ** 20 // wide.element_size()
        far = torch.zeros(rows * step, dtype=T, device="cuda").view(rows, step)[:, :256].view(rows, 4, 64)
        far.copy_(c.qd)
        c.attend(far)
        b.zero_()
        c.weigh(b, far)
        assert torch.equal(out, c.out) and torch.equal(lse, c.lse)
        # (each slot's 4 rows summands of both sums, at most n 2^-24 of the sum apart each)
        assert torch.all((a - b).abs() <= 2 * (4 * rows + 16) * 2.0 ** -24 * a.abs())


def test_offsets_past_32_bits(V):
    """The same sequences in a pool of 5 GB a tensor, in its last pages: every
    call gives the same bits as in a small pool."""
    say("scores offsets past 32 bits")
    rng = np.random.default_rng(2)
    rows, page, hd, nkv = [1, 70], 256, 128, 2
    lens = [700, 300]
    m = filled(rng, T16, lens, rows, nkv=nkv, page=page, hd=hd, shuffle=False)
    big = 5 * 2 ** 30 // (nkv * page * hd * 2)
    q = rounded(rng.standard_normal((sum(rows), 4, hd)) * 2, T16)
    c = Call(V, m, T16, [0, 1], rows, q, S.Scores(hd ** -0.5, 20.0))
    k, v = (torch.zeros((1, big, nkv, page, hd), dtype=T16, device="cuda") for _ in range(2))
    k[:, big - m.n_pages:], v[:, big - m.n_pages:] = c.d.k, c.d.v
    moved = torch.where(c.d.table >= 0, c.d.table + (big - m.n_pages), c.d.table)
    refs = torch.zeros(big, dtype=torch.int32, device="cuda")
    refs[big - m.n_pages:] = c.d.refs
    far = V.make_pages(k, v, moved, c.d.lens.clone(), c.d.held.clone(), refs, c.d.status.clone())
    got = []
    mass = torch.rand((1, 2, nkv, m.max_pages * page), device="cuda")
    for p in (c.d.p, far):
        sc = c.sc.make(V, p, torch)
        out, lse, w = torch.zeros_like(c.qd), torch.zeros_like(c.lse), mass.clone()
        V.vla_score_attention(p, 0, c.rows, sc, c.qd, out, c.scratch, lse=lse)
        V.vla_attention_mass(p, 0, c.rows, sc, c.qd, lse, w, c.scratch)
        kept = torch.full((2, m.max_pages * page), -1, dtype=torch.int32, device="cuda")
        work = torch.zeros(V.vla_pages_evict_scratch(p, 2), dtype=torch.uint8, device="cuda")
        V.vla_pages_evict(p, i32([0, 1]), i32([333, 20]), w, w, kept, work, first=3, last=9)
        torch.cuda.synchronize()
        got.append((out, lse, w, kept))
    assert all(torch.equal(x, y) for x, y in zip(*got))
    assert torch.equal(k[:, big - m.n_pages:], c.d.k) and torch.equal(v[:, big - m.n_pages:], c.d.v)
    assert torch.count_nonzero(k[:, :big - m.n_pages]) == 0


class Step:
    """A serving step: room for the drafts, attention and slot weights of every
    layer, verification, commit, eviction."""

    def __init__(self, V, seed, T=T16):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.V, layers, nkv, hd, page, rows, vocab = V, 2, 2, 64, 16, 6, 300
        m = filled(rng, T, [40, 100, 7], [0, 0, 0], layers=layers, nkv=nkv, page=page, hd=hd, spare=20)
        m.table = np.concatenate([m.table, np.full((3, 6), -1, np.int32)], 1)
        m.max_pages += 6
        self.d, self.layers = Dev(V, m, T), layers
        self.rows = V.make_rows(i32([0, 6, 12, 18]), 18)
        parent = [[-1, 0, 0, 1, 1, 2]] * 3
        bits = np.zeros((18, 32), bool)
        for e in range(3):
            for j in range(rows):
                k = j
                while k >= 0:
                    bits[6 * e + j, k] = True
                    k = parent[e][k]
        self.mask = torch.from_numpy(pack(bits)).cuda()
        self.parent = i32(sum(parent, []))
        depth = i32([0, 1, 1, 2, 2, 2] * 3)
        self.scores = V.make_scores(self.d.p, cap=20.0, slopes=torch.full((4,), 0.01, device="cuda"), window=90, depth=depth)
        self.q = torch.randn((layers, 18, 4, hd), device="cuda", generator=gen).to(T)
        self.out = torch.zeros_like(self.q)
        self.lse = torch.zeros((layers, 18, 4), device="cuda")
        self.mass = torch.zeros((layers, 3, nkv, m.max_pages * page), device="cuda")
        self.probs = torch.softmax(torch.randn((18, vocab), device="cuda", generator=gen), -1)
        self.drafted = torch.softmax(torch.randn((18, vocab), device="cuda", generator=gen), -1)
        self.tokens = torch.randint(vocab, (18,), device="cuda", generator=gen).int()
        self.uniform = torch.rand(18, device="cuda", generator=gen)
        self.kept, self.n_kept, self.next = i32([0] * 18), i32([0] * 3), i32([0] * 3)
        self.seqs, self.keep = i32([2, 0, 1]), i32([30, 39, 64])
        self.stay = torch.full((3, m.max_pages * page), -1, dtype=torch.int32, device="cuda")
        size = [V.vla_score_attention_scratch(self.d.p, self.rows, 4), V.vla_attention_mass_scratch(self.d.p, self.rows, 4),
                V.vla_verify_drafts_scratch(self.d.p, self.rows, vocab), V.vla_pages_evict_scratch(self.d.p, 3)]
        self.scratch = torch.zeros(max(size), dtype=torch.uint8, device="cuda")

    def run(self, stream=0):
        V, p, r = self.V, self.d.p, self.rows
        V.vla_pages_reserve(p, r, stream=stream)
        for l in range(self.layers):
            V.vla_score_attention(p, l, r, self.scores, self.q[l], self.out[l], self.scratch, lse=self.lse[l],
                                  mask=self.mask, stream=stream)
            V.vla_attention_mass(p, l, r, self.scores, self.q[l], self.lse[l], self.mass, self.scratch, mask=self.mask,
                                 stream=stream)
        V.vla_verify_drafts(p, r, self.tokens, self.probs, self.kept, self.n_kept, self.next, self.scratch,
                            parent=self.parent, drafted=self.drafted, uniform=self.uniform, stream=stream)
        V.vla_pages_commit(p, r, self.kept, self.n_kept, stream=stream)
        V.vla_pages_evict(p, self.seqs, self.keep, self.mass, self.mass, self.stay, self.scratch, first=2, last=10,
                          stream=stream)

    def state(self):
        d = self.d
        return [self.out, self.lse, self.mass, self.kept, self.n_kept, self.next, self.stay, d.k, d.v, d.table, d.lens,
                d.held, d.refs, d.status]

    def change(self, i):
        """What the model and the sampler would bring to step i."""
        gen = torch.Generator(device="cuda")
        gen.manual_seed(100 + i)
        self.q.copy_(torch.randn(self.q.shape, device="cuda", generator=gen))
        self.uniform.copy_(torch.rand(18, device="cuda", generator=gen))
        self.tokens.copy_(torch.randint(300, (18,), device="cuda", generator=gen).int())


def same(a, b):
    for x, y in zip(a.state(), b.state()):
        assert torch.equal(x, y)


def test_captured_steps_replay(V):
    """Steps replayed from a graph, with eager steps of another cache and
    synchronizations between, leave the same bits as eager ones."""
    say("scores captured step")
    a, b, other = Step(V, 1), Step(V, 1), Step(V, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.run(torch.cuda.current_stream().cuda_stream)
    for i in range(6):
        a.change(i), b.change(i)
        a.run(torch.cuda.current_stream().cuda_stream)
        graph.replay()
        other.run(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        same(a, b)
    assert a.d.lens.cpu().tolist() == [39, 64, min(30, int(a.d.lens[2]))] and int(a.d.status) == 0


def test_steps_on_two_streams(V):
    """Two caches' steps on two streams at once, scratch of their own each."""
    say("scores two streams")
    alone, both = [Step(V, s) for s in (3, 4)], [Step(V, s) for s in (3, 4)]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for i in range(5):
        for x, st in zip(both, streams):
            x.run(st.cuda_stream)
    for x in alone:
        for i in range(5):
            x.run()
    torch.cuda.synchronize()
    for x, y in zip(alone, both):
        same(x, y)
