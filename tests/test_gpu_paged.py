"""The paged KV cache on the GPU, through the binding, against a plain model in
64 bits (paged_util): norms, rotation and store; attention over pages with
causal and tree masks; pages handed out, shared, copied, moved and freed.

Tolerances count roundings. A bf16 value is off by at most half a step, 2^-8
of it; fp32 sums of n terms by n 2^-24 of the sum of their magnitudes.

* store: the rotated value adds two products of normed values. The norm takes
  a mean of squares (head_dim terms), a square root, a division and two
  products: under (head_dim / 2 + 8) 2^-24 relative, and the rotation 3 2^-24
  more of |a c| + |b s|; then one rounding to the cache's type.
* attention: a score is off by hd 2^-24 sum |q k| scale =: ds (and by 4 2^-24
  of its magnitude in the exponent), so a weight by a factor of e^(2 ds); the
  two sums over n keys add (n + 16) 2^-24. Every such error moves the result by
  at most itself times sum p |v| (numerator) and |o| <= sum p |v|
  (denominator). bf16 with more than 128 rows of a KV head to a sequence (on
  average; head dims up to 64: 192) rounds the probabilities once: 2^-8 in both
  sums; with fewer they are kept to 2^-16.
  Then one rounding of the output.
"""
import numpy as np
import pytest
import torch

import paged_util as U

pytestmark = pytest.mark.gpu

T32, T16 = torch.float32, torch.bfloat16
HALF = {T32: 2.0 ** -24, T16: 2.0 ** -8}


@pytest.fixture(scope="module")
def V():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_22335_amd as V
    return V


def say(msg):
    print(f"[gpu] {msg}", flush=True)


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), dtype=torch.int32, device="cuda")


def vals(t):
    return t.detach().cpu().to(torch.float64).numpy()


class Dev:
    """Device tensors of a model's state, and its descriptor."""

    def __init__(self, V, m, T, k=None, v=None):
        self.V, self.m, self.T = V, m, T
        self.k = torch.from_numpy(m.k).to(T).cuda() if k is None else k
        self.v = torch.from_numpy(m.v).to(T).cuda() if v is None else v
        self.table, self.lens, self.held, self.refs = i32(m.table), i32(m.lens), i32(m.held), i32(m.refs)
        self.status = i32([m.status])
        self.p = V.make_pages(self.k, self.v, self.table, self.lens, self.held, self.refs, self.status)

    def same(self, contents=True):
        m = self.m
        torch.cuda.synchronize()
        for name in ("lens", "held", "refs", "table"):
            got, want = getattr(self, name).cpu().numpy(), getattr(m, name)
            assert np.array_equal(got, want), (name, got, want)
        assert int(self.status.item()) == m.status
        if contents:
            assert np.array_equal(vals(self.k), m.k, equal_nan=True)
            assert np.array_equal(vals(self.v), m.v, equal_nan=True)


def rounded(x, T):
    return torch.from_numpy(np.ascontiguousarray(x)).to(T).to(torch.float64).numpy()


def filled(rng, T, lens, rows, layers=1, nkv=1, page=16, hd=64, spare=3, extra_seqs=0, shuffle=True):
    """A model whose sequences hold lens committed slots and pages for rows
    more, in scattered pages, every slot of the pool with a value."""
    need = [-(-(n + r) // page) for n, r in zip(lens, rows)]
    n_pages, n_seqs = sum(need) + spare, len(lens) + extra_seqs
    m = U.Model(layers, n_pages, nkv, page, hd, n_seqs, max(need + [1]) + 2)
    order = rng.permutation(n_pages) if shuffle else np.arange(n_pages)
    at = 0
    for s, n in enumerate(need):
        m.table[s, :n] = order[at:at + n]
        m.refs[order[at:at + n]] = 1
        m.held[s], m.lens[s] = n, lens[s]
        at += n
    m.k = rounded(rng.standard_normal(m.dims), T)
    m.v = rounded(rng.standard_normal(m.dims), T)
    return m


# --------------------------------------------------------------------------
# Norm, rotation, store
# --------------------------------------------------------------------------

STORE = [
    # T, hd, nq, nkv, rot, page, gains, plus_one, given positions, lens, rows
    (T16, 64, 4, 1, 64, 16, "qk", 0, False, [0, 15, 16], [1, 1, 1]),
    (T16, 256, 8, 1, 256, 32, "qk", 1, False, [305, 0], [1, 40]),
    (T16, 128, 6, 2, 128, 64, "qk", 0, True, [63, 64, 1], [2, 0, 65]),
    (T16, 96, 3, 3, 64, 16, "q", 0, True, [7], [33]),
    (T16, 160, 10, 2, 16, 128, "k", 0, False, [127, 129], [3, 130]),
    (T16, 32, 2, 1, 0, 16, "", 0, False, [5], [19]),
    (T16, 224, 5, 1, 112, 256, "qk", 0, True, [250], [9]),
    (T32, 32, 16, 16, 32, 16, "qk", 0, False, [0, 3], [17, 2]),
    (T32, 96, 6, 2, 64, 16, "qk", 1, True, [30, 100], [61, 17]),
    (T32, 128, 7, 7, 128, 32, "qk", 0, False, [31, 33], [1, 1]),
    (T32, 64, 8, 1, 48, 64, "", 0, False, [10], [70]),
]


@pytest.mark.parametrize("T,hd,nq,nkv,rot,page,gains,one,given,lens,rows", STORE)
def test_norm_rope_store(V, T, hd, nq, nkv, rot, page, gains, one, given, lens, rows):
    say(f"store {T} hd={hd} nq={nq} nkv={nkv} rot={rot} page={page} lens={lens} rows={rows}")
    rng = np.random.default_rng(hd * 7 + nq)
    m = filled(rng, T, lens, rows, layers=2, nkv=nkv, page=page, hd=hd, extra_seqs=1)
    d = Dev(V, m, T)
    n = sum(rows)
    n_rows = n + 3  # the last rows belong to nobody
    heads = nq + 2 * nkv
    # entries in another order than the sequences, one of them padding
    order = list(rng.permutation(len(lens))) + [-1]
    counts = [rows[s] for s in order[:-1]] + [2]
    start = np.concatenate([[0], np.cumsum(counts)])
    x = rounded(rng.standard_normal((n_rows, heads, hd)) * 2 ** rng.uniform(-3, 3, (1, heads, 1)), T)
    qkv = torch.from_numpy(x).to(T).cuda()
    q_out = torch.full((n_rows, nq + 1, hd), 7.0, dtype=T, device="cuda")  # rows with a gap between them
    qg = rng.standard_normal(hd).astype(np.float32) if "q" in gains else None
    kg = rng.standard_normal(hd).astype(np.float32) if "k" in gains else None
    n_pos = max(l + r for l, r in zip(lens, rows)) + 40
    cos = sin = None
    if rot:
        ang = np.arange(n_pos)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
        cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    pos = np.concatenate([np.arange(c) // 2 + (m.lens[s] if s >= 0 else 0) + 3 for s, c in zip(order, counts)]
                         + [np.zeros(1)]).astype(np.int32) if given else None
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    rope = V.make_rope_norm(dev(cos), dev(sin), dev(qg), dev(kg), one, 1e-6)
    r = V.make_rows(i32(start), n_rows, i32(order))
    V.vla_qk_norm_rope(d.p, 1, r, rope, qkv[:, :nq], qkv[:, nq:nq + nkv], qkv[:, nq + nkv:], q_out[:, :nq],
                       pos=None if pos is None else i32(pos))
    want_q, tol_q = np.full((n_rows, nq + 1, hd), 7.0), np.zeros((n_rows, nq + 1, hd))
    want_k, tol_k = m.k.copy(), np.zeros_like(m.k)
    rel = (hd / 2 + 12) * 2.0 ** -24
    for s, a, c in zip(order, start, counts):
        if s < 0:
            continue
        for i in range(c):
            t, slot = a + i, int(m.lens[s]) + i
            ps = slot if pos is None else int(pos[t])
            g = lambda v: None if v is None else (1 if one else 0) + v.astype(np.float64)  # noqa: E731
            qv, qs = U.norm_rope(x[t, :nq], g(qg), 1e-6, cos, sin, ps)
            kv, ks = U.norm_rope(x[t, nq:nq + nkv], g(kg), 1e-6, cos, sin, ps)
            want_q[t, :nq], tol_q[t, :nq] = qv, rel * qs + HALF[T] * np.abs(qv)
            p, at = m.where(s, slot)
            want_k[1, p, :, at], tol_k[1, p, :, at] = kv, rel * ks + HALF[T] * np.abs(kv)
            m.v[1, p, :, at] = x[t, nq + nkv:]
    torch.cuda.synchronize()
    assert np.all(np.abs(vals(q_out) - want_q) <= tol_q)
    assert np.all(np.abs(vals(d.k) - want_k) <= tol_k)
    m.k = vals(d.k)
    d.same()  # V bit for bit, and nothing else changed


def test_store_in_place_and_left_out_rows(V):
    """q_out may be q; a row whose position is outside the table is left out, a
    slot without a page keeps q but stores nothing, and status says so."""
    say("store in place, bad positions, missing pages")
    rng = np.random.default_rng(3)
    T, hd, nq, nkv = T16, 64, 4, 2
    m = filled(rng, T, [14, 20], [2, 12], nkv=nkv, hd=hd)
    m.held[0] = 1  # 16 slots; rows 2 and 3 of entry 0 have no page
    d = Dev(V, m, T)
    x = rounded(rng.standard_normal((7, nq + 2 * nkv, hd)), T)
    qkv = torch.from_numpy(x).to(T).cuda()
    cos, sin = np.ones((30, 32), np.float32), np.zeros((30, 32), np.float32)  # no turn
    rope = V.make_rope_norm(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    pos = [0, 1, 2, 3, 29, 30, -1]
    V.vla_qk_norm_rope(d.p, 0, V.make_rows(i32([0, 4, 7]), 7), rope, qkv[:, :nq], qkv[:, nq:nq + nkv],
                       qkv[:, nq + nkv:], qkv[:, :nq], pos=i32(pos))
    for t, (s, i) in enumerate([(0, 0), (0, 1), (0, 2), (0, 3), (1, 0), (1, 1), (1, 2)]):
        w = m.where(s, int(m.lens[s]) + i)
        if w is not None and 0 <= pos[t] < 30:
            m.k[0, w[0], :, w[1]], m.v[0, w[0], :, w[1]] = x[t, nq:nq + nkv], x[t, nq + nkv:]
    m.status = V.PAGES_OUT | V.PAGES_BAD
    d.same()
    assert np.array_equal(vals(qkv), x)  # without norm and turn, q is what it was


# --------------------------------------------------------------------------
# Attention
# --------------------------------------------------------------------------

def tree_mask(rng, n, words, kind):
    """Bits [n][32 words]: a random tree's ancestors and self, or random bits
    (rows may see nothing)."""
    b = np.zeros((n, 32 * words), bool)
    for j in range(n):
        if kind == "tree":
            p = rng.integers(-1, j) if j else -1
            if p >= 0:
                b[j] = b[p]
            if j < 32 * words:
                b[j, j] = True
        elif kind == "random":
            b[j] = rng.random(32 * words) < 0.4
            if j % 3 == 0:
                b[j] = False
    return b


def pack(bits):
    w = bits.reshape(bits.shape[0], -1, 32).astype(np.uint64) @ (1 << np.arange(32, dtype=np.uint64))
    return w.astype(np.uint32).view(np.int32)


def expect(m, T, layer, order, start, counts, q, bits, scale, mean_rows):
    """Results and tolerances of every row (rows of nobody: nan), in 64 bits."""
    nq, hd = q.shape[1:]
    nkv = m.dims[2]
    group = nq // nkv
    want, tol = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for s, a, c in zip(order, start, counts):
        if s < 0 or c == 0:
            continue
        L, cap = int(m.lens[s]), int(m.held[s]) * m.page
        end = min(L + c, cap)
        pages, places = m.table[s][np.arange(end) // m.page], np.arange(end) % m.page
        see = np.zeros((c, end), bool)
        see[:, :min(L, end)] = True
        j = np.arange(L, end) - L
        if bits is None:
            see[:, L:] = j[None, :] <= np.arange(c)[:, None]
        else:
            see[:, L:] = (j < bits.shape[1]) & bits[a:a + c][:, np.minimum(j, bits.shape[1] - 1)]
        any_seen = see.any(1)[:, None, None]
        see = see[:, None, :]  # [rows, heads of the group, keys]
        for h in range(nkv):
            k, v = m.k[layer, pages, h, places], m.v[layer, pages, h, places]
            x = q[a:a + c, h * group:(h + 1) * group]
            # hidden keys' and values' contents do not count
            shown = see[:, 0].any(0)
            k, v = np.where(shown[:, None], k, 0), np.where(shown[:, None], v, 0)
            score = np.where(see, np.matmul(x, k.T) * scale, -np.inf)
            top = np.where(any_seen, score.max(-1, keepdims=True, initial=-np.inf), 0)
            p = np.exp(score - top)
            p /= np.where(any_seen, p.sum(-1, keepdims=True), 1)
            o, mag = np.matmul(p, v), np.matmul(p, np.abs(v))
            ds = np.where(see, np.matmul(np.abs(x), np.abs(k).T), 0).max(-1, initial=0)[..., None] * scale
            ds = ds * (hd + 4) * 2.0 ** -24
            one = 0.0 if T is T32 else 2.0 ** -8 if mean_rows * group > (128 if hd > 64 else 192) else 2.0 ** -16
            rel = np.expm1(2 * ds) + (end + 16) * 2.0 ** -24 + one
            want[a:a + c, h * group:(h + 1) * group] = o
            tol[a:a + c, h * group:(h + 1) * group] = rel * (mag + np.abs(o)) + HALF[T] * np.abs(o) * (1 + rel) + 1e-38
    return want, tol


ATTEND = [
    # T, hd, nq, nkv, page, mask, lens, rows
    (T16, 64, 1, 1, 16, None, [0], [1]),
    (T16, 64, 4, 1, 16, None, [0, 1, 15, 16, 17, 31, 32, 33], [1] * 8),
    (T16, 256, 8, 1, 32, None, [305, 420, 31, 0], [1, 1, 1, 1]),
    (T16, 128, 8, 2, 16, None, [1000, 3, 130], [1, 2, 0]),
    (T16, 128, 32, 8, 64, None, [127, 128, 129], [1, 1, 1]),
    (T16, 256, 8, 1, 32, "tree", [300, 64, 0], [40, 33, 7]),
    (T16, 128, 6, 2, 16, "tree", [50, 0, 9], [61, 31, 1]),
    (T16, 64, 2, 2, 256, "random", [5, 0, 256], [70, 20, 33]),
    (T16, 32, 4, 4, 16, "random", [0, 40], [9, 12]),
    (T16, 96, 5, 1, 16, None, [0, 70], [150, 33]),
    (T16, 160, 4, 2, 64, None, [10], [90]),
    (T16, 224, 3, 1, 16, "tree", [100], [30]),
    (T16, 256, 16, 1, 128, None, [200], [70]),
    (T16, 128, 16, 2, 16, None, [0, 300], [260, 17]),
    (T32, 64, 4, 1, 16, None, [0, 33, 17], [1, 1, 1]),
    (T32, 128, 8, 2, 32, "tree", [77, 0], [40, 12]),
    (T32, 96, 6, 2, 16, "random", [30, 0, 50], [61, 17, 3]),
    (T32, 32, 2, 1, 16, None, [60], [100]),
    (T32, 128, 8, 1, 64, None, [5, 200], [64, 1]),
    (T32, 64, 8, 1, 16, "tree", [70, 0], [50, 41]),
    (T32, 96, 6, 1, 16, "random", [33], [61]),
    (T32, 128, 8, 1, 32, "tree", [77, 300], [45, 40]),
    (T16, 128, 8, 1, 16, "tree", [700, 0], [50, 40]),
    (T16, 64, 8, 1, 16, "random", [1100], [60]),
]


@pytest.mark.parametrize("T,hd,nq,nkv,page,kind,lens,rows", ATTEND)
def test_tree_attention(V, T, hd, nq, nkv, page, kind, lens, rows):
    say(f"attend {T} hd={hd} nq={nq} nkv={nkv} page={page} mask={kind} lens={lens} rows={rows}")
    rng = np.random.default_rng(hd * 5 + nq * 3 + len(lens) + sum(lens))
    m = filled(rng, T, lens, rows, layers=2, nkv=nkv, page=page, hd=hd)
    # whatever lies in slots that nobody has written must not show
    used = np.zeros(m.dims[:4], bool)
    for s in range(len(lens)):
        for i in range(lens[s] + rows[s]):
            p, at = m.where(s, i)
            used[:, p, :, at] = True
    m.k[~used], m.v[~used] = np.nan, np.inf
    d = Dev(V, m, T)
    order = list(rng.permutation(len(lens))) + [-1]
    counts = [rows[s] for s in order[:-1]] + [2]
    start = np.concatenate([[0], np.cumsum(counts)])
    n_rows = int(start[-1]) + 2
    q = rounded(rng.standard_normal((n_rows, nq, hd)) * 1.5, T)
    qd = torch.from_numpy(q).to(T).cuda()
    out = torch.full((n_rows, nq + 1, hd), 5.0, dtype=T, device="cuda")
    bits, mask = None, None
    if kind:
        words = (max(rows) + 31) // 32 if kind == "tree" else 2
        bits = np.concatenate([tree_mask(rng, c, words, kind) for c in counts] + [np.ones((2, 32 * words), bool)])
        mask = torch.from_numpy(pack(bits)).cuda()
    r = V.make_rows(i32(start), n_rows, i32(order))
    scratch = torch.full((V.vla_tree_attention_scratch(d.p, r, nq),), 255, dtype=torch.uint8, device="cuda")
    for scale in (hd ** -0.5, 0.31):
        V.vla_tree_attention(d.p, 1, r, qd, out[:, :nq], scratch, mask=mask, scale=scale)
        want, tol = expect(m, T, 1, order, start, counts, q, bits, scale, n_rows / len(order))
        torch.cuda.synchronize()
        got = vals(out)
        assert np.all(got[:, nq] == 5.0)
        live = ~np.isnan(want)
        assert np.all(got[:, :nq][~live] == 5.0)
        off = np.abs(got[:, :nq][live] - want[live]) / tol[live]
        assert np.all(off <= 1), float(np.nanmax(off))
    d.same()


@pytest.mark.parametrize("T,rows,nq", [(T16, 20, 4), (T16, 90, 4), (T32, 20, 2), (T32, 90, 4)])
def test_masked_drafts_may_hold_anything(V, T, rows, nq):
    """NaN and infinities in K and V of drafts show in the rows that see them
    and in no other, and a row of large scores stays finite."""
    say(f"attend with odd drafts {T} rows={rows}")
    rng = np.random.default_rng(rows)
    hd = 64
    m = filled(rng, T, [37], [rows], hd=hd)
    bad = {3: (np.nan, None), 7: (None, np.inf), 11: (None, np.nan), 12: (np.inf, None)}
    for j, (a, b) in bad.items():
        p, at = m.where(0, 37 + j)
        if a is not None:
            m.k[0, p, 0, at, 5] = a
        if b is not None:
            m.v[0, p, 0, at, 9] = b
    d = Dev(V, m, T)
    q = rounded(rng.standard_normal((rows, nq, hd)), T)
    q[1] *= 64  # scores far apart
    r = V.make_rows(i32([0, rows]), rows)
    out = torch.empty((rows, nq, hd), dtype=T, device="cuda")
    scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, nq), dtype=torch.uint8, device="cuda")
    words = (rows + 31) // 32
    bits = np.zeros((rows, 32 * words), bool)
    for j in range(rows):
        bits[j, j] = j not in bad
        bits[j, 0] = True
    bits[5, 7] = True   # these see an odd draft
    bits[6, 11] = True
    V.vla_tree_attention(d.p, 0, r, torch.from_numpy(q).to(T).cuda(), out, scratch,
                         mask=torch.from_numpy(pack(bits)).cuda())
    torch.cuda.synchronize()
    got = vals(out)
    clean = [j for j in range(rows) if j not in (5, 6)]
    plain = m.k.copy(), m.v.copy()
    m.k, m.v = np.nan_to_num(m.k, nan=0, posinf=0), np.nan_to_num(m.v, nan=0, posinf=0)
    want, tol = expect(m, T, 0, [0], [0], [rows], q, bits, hd ** -0.5, rows)
    assert np.all(np.abs(got[clean] - want[clean]) <= tol[clean])
    assert np.all(np.isposinf(got[5, :, 9])) and np.all(np.isnan(got[6, :, 9]))
    for j in (5, 6):
        rest = [c for c in range(hd) if c != 9]
        assert np.all(np.abs(got[j][:, rest] - want[j][:, rest]) <= tol[j][:, rest])
    # causal: rows before the first odd draft are clean, later ones see it
    m.k, m.v = plain
    V.vla_tree_attention(d.p, 0, r, torch.from_numpy(q).to(T).cuda(), out, scratch)
    torch.cuda.synchronize()
    got = vals(out)
    assert np.all(np.isfinite(got[:3])) and np.all(np.isnan(got[3]))


def test_long_uneven_sequences_are_shared_out(V):
    """Keys of one sequence split over many workgroups and joined, next to
    short sequences; the same bits on every call."""
    say("attend long")
    rng = np.random.default_rng(11)
    for T, hd, nq, nkv, lens, rows in [(T16, 128, 8, 1, [20000, 5, 700], [1, 1, 1]),
                                       (T16, 256, 2, 1, [9000], [3]), (T16, 64, 8, 2, [12000, 100], [64, 2]),
                                       (T32, 64, 2, 1, [7000, 1], [1, 1])]:
        m = filled(rng, T, lens, rows, nkv=nkv, page=64, hd=hd)
        d = Dev(V, m, T)
        start = np.concatenate([[0], np.cumsum(rows)])
        n = int(start[-1])
        q = rounded(rng.standard_normal((n, nq, hd)) * 2, T)
        qd = torch.from_numpy(q).to(T).cuda()
        r = V.make_rows(i32(start), n)
        outs = []
        scratch = torch.zeros(V.vla_tree_attention_scratch(d.p, r, nq), dtype=torch.uint8, device="cuda")
        for fill in (0, 255, 77):
            scratch.fill_(fill)
            out = torch.empty((n, nq, hd), dtype=T, device="cuda")
            V.vla_tree_attention(d.p, 0, r, qd, out, scratch)
            outs.append(out)
        torch.cuda.synchronize()
        want, tol = expect(m, T, 0, list(range(len(lens))), start, rows, q, None, hd ** -0.5, n / len(rows))
        assert np.all(np.abs(vals(outs[0]) - want) <= tol)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("T,hd,nq,nkv,lens,rows", [
    (T16, 64, 28, 4, [500, 3, 70], [1100, 900, 40]),    # seven heads to a KV head: tiles that part tokens
    (T16, 128, 32, 8, [0, 900], [1100, 60]),
    (T16, 256, 24, 8, [100, 0], [500, 700]),
    (T32, 64, 16, 16, [40, 600], [900, 1100]),
    (T16, 64, 8, 8, [int(x) for x in range(90)], [1 + x % 3 for x in range(90)])])
def test_more_tiles_than_workgroups(V, T, hd, nq, nkv, lens, rows):
    """Runs that begin and end inside tiles, causal tiles of growing length."""
    say(f"attend many tiles {T} hd={hd} nq={nq} nkv={nkv}")
    rng = np.random.default_rng(nq + hd)
    m = filled(rng, T, lens, rows, nkv=nkv, page=64, hd=hd)
    d = Dev(V, m, T)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = int(start[-1])
    q = rounded(rng.standard_normal((n, nq, hd)), T)
    qd = torch.from_numpy(q).to(T).cuda()
    r = V.make_rows(i32(start), n)
    out = torch.full((n, nq, hd), float("nan"), dtype=T, device="cuda")
    scratch = torch.full((V.vla_tree_attention_scratch(d.p, r, nq),), 255, dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(d.p, 0, r, qd, out, scratch)
    torch.cuda.synchronize()
    want, tol = expect(m, T, 0, list(range(len(lens))), start, rows, q, None, hd ** -0.5, n / len(rows))
    off = np.abs(vals(out) - want) / tol
    assert np.all(off <= 1), float(np.nanmax(off))


@pytest.mark.parametrize("T,hd,nq,nkv,page,lens,rows", [
    (T16, 64, 32, 8, 16, [3001, 2040, 1500, 2999], [300, 299, 31, 257]),
    (T16, 128, 32, 8, 256, [2500, 3100], [300, 260]),
    (T16, 256, 16, 8, 32, [1025, 2400], [400, 333])])
def test_long_runs(V, T, hd, nq, nkv, page, lens, rows):
    """Runs of more blocks of keys than a wave looks up at once."""
    say(f"attend long runs {T} hd={hd} page={page}")
    rng = np.random.default_rng(hd + page)
    m = filled(rng, T, lens, rows, nkv=nkv, page=page, hd=hd)
    d = Dev(V, m, T)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = int(start[-1])
    q = rounded(rng.standard_normal((n, nq, hd)), T)
    r = V.make_rows(i32(start), n)
    out = torch.full((n, nq, hd), float("nan"), dtype=T, device="cuda")
    scratch = torch.full((V.vla_tree_attention_scratch(d.p, r, nq),), 255, dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(d.p, 0, r, torch.from_numpy(q).to(T).cuda(), out, scratch)
    torch.cuda.synchronize()
    want, tol = expect(m, T, 0, list(range(len(lens))), start, rows, q, None, hd ** -0.5, n / len(rows))
    off = np.abs(vals(out) - want) / tol
    assert np.all(off <= 1), float(np.nanmax(off))


@pytest.mark.parametrize("T,rows,nq", [(T16, 3, 4), (T16, 70, 4), (T32, 5, 2), (T32, 80, 4)])
def test_odd_queries_stay_alone(V, T, rows, nq):
    """A query that holds NaN or infinities spoils its own row and head only."""
    say(f"attend with odd queries {T} rows={rows}")
    rng = np.random.default_rng(rows + 7)
    hd = 128
    m = filled(rng, T, [300], [rows], hd=hd, page=32)
    d = Dev(V, m, T)
    q = rounded(rng.standard_normal((rows, nq, hd)), T)
    odd = q.copy()
    odd[1, 0, 5], odd[2, 1, 9], odd[rows - 1, nq - 1, 0] = np.nan, np.inf, -np.inf
    r = V.make_rows(i32([0, rows]), rows)
    out = torch.empty((rows, nq, hd), dtype=T, device="cuda")
    scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, nq), dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(d.p, 0, r, torch.from_numpy(odd).to(T).cuda(), out, scratch)
    torch.cuda.synchronize()
    got = vals(out)
    want, tol = expect(m, T, 0, [0], [0], [rows], q, None, hd ** -0.5, rows)
    spoilt = ~np.isfinite(odd).all(-1)
    assert spoilt.sum() == 3 and np.all(np.isnan(got[1, 0]))
    assert np.all(np.abs(got - want)[~spoilt] <= tol[~spoilt])


@pytest.mark.parametrize("T,hd,nq", [(T16, 64, 2), (T16, 128, 24), (T32, 96, 2)])
def test_rows_outside_the_entries(V, T, hd, nq):
    """Rows in front of the first entry and behind the last are left alone, and
    an entry that passes the buffers ends with them."""
    say(f"rows outside the entries {T} hd={hd}")
    rng = np.random.default_rng(hd)
    page, n_rows = 16, 40
    m = filled(rng, T, [21, 40, 3], [14, 20, 90], hd=hd, page=page)
    m.k[:], m.v[:] = rounded(m.k, T), rounded(m.v, T)
    d = Dev(V, m, T)
    x = rounded(rng.standard_normal((n_rows, nq + 2, hd)), T)
    qkv = torch.from_numpy(x).to(T).cuda()
    # entry 0: rows 4 .. 17, entry 1: none, entry 2 (n_rows behind its start 30): rows 30 .. 39
    for start, live in (([4, 18, 18, 18], {0: (4, 18)}), ([30, 30, 30, 120], {2: (30, 40)}),
                        ([5, 12, 31, 36], {0: (5, 12), 1: (12, 31), 2: (31, 36)})):
        r = V.make_rows(i32(start), n_rows)
        out = torch.full((n_rows, nq, hd), 7.0, dtype=T, device="cuda")
        scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, nq), dtype=torch.uint8, device="cuda")
        V.vla_qk_norm_rope(d.p, 0, r, V.make_rope_norm(), qkv[:, :nq], qkv[:, nq:nq + 1], qkv[:, nq + 1:],
                           qkv[:, :nq])
        V.vla_tree_attention(d.p, 0, r, qkv[:, :nq], out, scratch)
        want = np.full((n_rows, nq, hd), 7.0)
        tol = np.zeros_like(want)
        for s, (a, b) in live.items():
            for t in range(a, b):
                p, at = m.where(s, int(m.lens[s]) + t - a)
                m.k[0, p, :, at], m.v[0, p, :, at] = x[t, nq:nq + 1], x[t, nq + 1:]
        for s, (a, b) in live.items():
            w, e = expect(m, T, 0, [s], [a], [b - a], x[:, :nq], None, hd ** -0.5, n_rows / 3)
            want[a:b], tol[a:b] = w[a:b], e[a:b]
        d.same()
        assert np.all(np.abs(vals(out) - want) <= tol), start


def test_drafts_without_pages_are_not_seen(V):
    """A pool that ran dry: rows see the slots that have pages; a row that has
    none is zero."""
    say("attend without pages")
    rng = np.random.default_rng(15)
    for rows in ([20, 3, 40], [300, 5, 200]):
        m = filled(rng, T16, [30, 0, 10], rows, hd=64)
        m.held[:] = [2, 0, 2]  # 32 slots, none, 32 slots
        d = Dev(V, m, T16)
        start = np.concatenate([[0], np.cumsum(rows)])
        n = int(start[-1])
        q = rounded(rng.standard_normal((n, 2, 64)), T16)
        r = V.make_rows(i32(start), n)
        out = torch.full((n, 2, 64), float("nan"), dtype=T16, device="cuda")
        scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, 2), dtype=torch.uint8, device="cuda")
        V.vla_tree_attention(d.p, 0, r, torch.from_numpy(q).to(T16).cuda(), out, scratch)
        torch.cuda.synchronize()
        want, tol = expect(m, T16, 0, [0, 1, 2], start, rows, q, None, 0.125, n / 3)
        assert np.all(np.abs(vals(out) - want) <= tol)
        assert not vals(out)[start[1]:start[2]].any()


def test_thousands_of_entries(V):
    """Two steps of the search for a row's sequence, many chunks of entries."""
    say("5,000 entries")
    rng = np.random.default_rng(16)
    lens, rows = [int(x) for x in rng.integers(0, 20, 5000)], [int(x) for x in rng.integers(0, 3, 5000)]
    m = filled(rng, T16, lens, rows, hd=32)
    d = Dev(V, m, T16)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = int(start[-1])
    x = rounded(rng.standard_normal((n, 3, 32)), T16)
    xd = torch.from_numpy(x).to(T16).cuda()
    r = V.make_rows(i32(start), n)
    q, out = torch.empty((n, 1, 32), dtype=T16, device="cuda"), torch.empty((n, 1, 32), dtype=T16, device="cuda")
    V.vla_qk_norm_rope(d.p, 0, r, V.make_rope_norm(), xd[:, :1], xd[:, 1:2], xd[:, 2:], q)
    scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, 1), dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(d.p, 0, r, q, out, scratch)
    V.vla_pages_commit(d.p, r)
    torch.cuda.synchronize()
    assert np.array_equal(vals(q), x[:, :1])
    for s in range(5000):
        for i in range(rows[s]):
            p, at = m.where(s, lens[s] + i)
            m.k[0, p, :, at], m.v[0, p, :, at] = x[start[s] + i, 1:2], x[start[s] + i, 2:]
    want, tol = expect(m, T16, 0, list(range(5000)), start, rows, x[:, :1], None, 32 ** -0.5, n / 5000)
    assert np.all(np.abs(vals(out) - want) <= tol)
    m.lens += np.array(rows, np.int32)
    d.same()


def test_many_entries(V):
    """More entries than a wave has lanes, most of them short or empty."""
    say("attend many entries")
    rng = np.random.default_rng(12)
    lens = [int(x) for x in rng.integers(0, 40, 300)]
    rows = [int(x) for x in rng.integers(0, 3, 300)]
    m = filled(rng, T16, lens, rows, hd=64)
    d = Dev(V, m, T16)
    start = np.concatenate([[0], np.cumsum(rows)])
    n = int(start[-1])
    q = rounded(rng.standard_normal((n, 2, 64)), T16)
    r = V.make_rows(i32(start), n)
    out = torch.empty((n, 2, 64), dtype=T16, device="cuda")
    scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, 2), dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(d.p, 0, r, torch.from_numpy(q).to(T16).cuda(), out, scratch)
    torch.cuda.synchronize()
    want, tol = expect(m, T16, 0, list(range(300)), start, rows, q, None, 0.125, n / 300)
    assert np.all(np.abs(vals(out) - want) <= tol)
    # and their store: every row's K is where its sequence's slot is
    x = torch.from_numpy(rounded(rng.standard_normal((n, 4, 64)), T16)).to(T16).cuda()
    V.vla_qk_norm_rope(d.p, 0, r, V.make_rope_norm(), x[:, :2], x[:, 2:3], x[:, 3:], out)
    for s in range(300):
        for i in range(rows[s]):
            p, at = m.where(s, lens[s] + i)
            m.k[0, p, :, at], m.v[0, p, :, at] = vals(x[start[s] + i, 2:3]), vals(x[start[s] + i, 3:])
    d.same()


def test_offsets_past_32_bits(V):
    """Pages more than 4 GiB into K and V."""
    say("offsets past 32 bits")
    rng = np.random.default_rng(13)
    page, hd, nkv, n_pages = 256, 128, 8, 9000  # 512 KiB a page: 4.7 GB each
    k = torch.zeros((1, n_pages, nkv, page, hd), dtype=T16, device="cuda")
    v = torch.zeros_like(k)
    table, lens, held = i32([[n_pages - 1, 3, n_pages - 2, -1]]), i32([600]), i32([3])
    refs, status = torch.zeros(n_pages, dtype=torch.int32, device="cuda"), i32([0])
    refs[[n_pages - 1, 3, n_pages - 2]] = 1
    p = V.make_pages(k, v, table, lens, held, refs, status)
    vv = rounded(rng.standard_normal((600, nkv, hd)), T16)
    kk = rounded(rng.standard_normal((600, nkv, hd)), T16)
    for i, pg in enumerate([n_pages - 1, 3, n_pages - 2]):
        part = slice(256 * i, min(256 * i + 256, 600))
        n = part.stop - part.start
        k[0, pg, :, :n] = torch.from_numpy(kk[part]).to(T16).cuda().transpose(0, 1)
        v[0, pg, :, :n] = torch.from_numpy(vv[part]).to(T16).cuda().transpose(0, 1)
    x = rounded(rng.standard_normal((2, 3 * nkv, hd)), T16)
    xd = torch.from_numpy(x).to(T16).cuda()
    r = V.make_rows(i32([0, 2]), 2)
    q_out = torch.empty((2, nkv, hd), dtype=T16, device="cuda")
    V.vla_qk_norm_rope(p, 0, r, V.make_rope_norm(), xd[:, :nkv], xd[:, nkv:2 * nkv], xd[:, 2 * nkv:], q_out)
    assert np.array_equal(vals(k[0, n_pages - 2, :, 88:90]), x[:, nkv:2 * nkv].transpose(1, 0, 2))
    out = torch.empty_like(q_out)
    scratch = torch.empty(V.vla_tree_attention_scratch(p, r, nkv), dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(p, 0, r, q_out, out, scratch)
    ka, va = np.concatenate([kk, x[:, nkv:2 * nkv]]), np.concatenate([vv, x[:, 2 * nkv:]])
    for i in range(2):
        for h in range(nkv):
            see = np.arange(602) <= 600 + i
            o, mag, ds = U.attention_row(x[i, h], ka[:, h], va[:, h], see, hd ** -0.5)
            rel = np.expm1(2 * ds * (hd + 4) * 2.0 ** -24) + 618 * 2.0 ** -24 + 2.0 ** -16
            assert np.all(np.abs(vals(out[i, h]) - o) <= 2 * rel * mag + 2.0 ** -8 * np.abs(o) * (1 + rel))
    made = i32([0])
    table2, lens2, held2 = torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), i32([602, 0]), i32([3, 0])
    table2[0] = table[0]
    refs[:] = 1
    refs[n_pages - 3] = 0  # the only free page
    p2 = V.make_pages(k, v, table2, lens2, held2, refs, status)
    V.vla_pages_fork(p2, i32([0]), i32([1]), made)
    torch.cuda.synchronize()
    assert made.item() == 1 and table2[1].tolist() == [n_pages - 1, 3, n_pages - 3, -1]
    assert torch.equal(k[0, n_pages - 3, :, :90], k[0, n_pages - 2, :, :90])
    assert torch.equal(v[0, n_pages - 3, :, :90], v[0, n_pages - 2, :, :90]) and not v[0, n_pages - 3, :, 90:].any()
    kept = i32([1, -1])
    V.vla_pages_commit(V.make_pages(k, v, table, lens, held, refs, status), r, kept, i32([1]))
    torch.cuda.synchronize()
    assert torch.equal(k[0, n_pages - 2, :, 88], k[0, n_pages - 2, :, 89]) and lens.item() == 601


# --------------------------------------------------------------------------
# Book-keeping
# --------------------------------------------------------------------------

@pytest.mark.parametrize("seed,T,layers,nkv,hd,page,n_pages", [
    (0, T16, 3, 1, 64, 16, 60), (1, T16, 2, 3, 96, 32, 24), (2, T32, 1, 2, 32, 16, 40), (3, T16, 5, 2, 256, 16, 90),
    (4, T32, 2, 1, 128, 64, 12)])
def test_calls_follow_the_model(V, seed, T, layers, nkv, hd, page, n_pages):
    """A random run of calls, the pool running dry now and then: tables,
    counts, lengths, status and every value of the pool as the model has them."""
    say(f"book-keeping seed={seed}")
    rng = np.random.default_rng(seed)
    n_seqs = 9
    m = U.Model(layers, n_pages, nkv, page, hd, n_seqs, 9)
    m.k, m.v = rounded(rng.standard_normal(m.dims), T), rounded(rng.standard_normal(m.dims), T)
    d = Dev(V, m, T)
    d.table.fill_(3)
    V.vla_pages_init(d.p)
    d.same()
    for step in range(40):
        kind = rng.choice(["grow", "grow", "grow", "fork", "release"])
        if kind == "grow":
            seqs = [int(x) for x in rng.permutation(n_seqs)[:rng.integers(1, 6)]]
            if rng.random() < 0.3:
                seqs[0] = -1
            rows = [int(x) for x in rng.integers(0, 2 * page, len(seqs))]
            start = np.concatenate([[0], np.cumsum(rows)])
            n_rows = int(start[-1]) + 1
            r = V.make_rows(i32(start), n_rows, i32(seqs))
            entries = list(zip(seqs, rows))
            V.vla_pages_reserve(d.p, r)
            m.reserve(entries)
            d.same(contents=False)
            form = rng.integers(0, 3)
            if form == 0:
                V.vla_pages_commit(d.p, r)
                m.commit(entries, rows)
            elif form == 1:
                counts = [int(rng.integers(0, n + 1)) for n in rows]
                V.vla_pages_commit(d.p, r, n_kept=i32(counts))
                m.commit(entries, counts)
            else:
                lists = [sorted(int(x) for x in rng.permutation(n)[:rng.integers(0, n + 1)]) for n in rows]
                if rng.random() < 0.3 and rows[-1] >= 2:
                    lists[-1] = [1, 1] if rng.random() < 0.5 else [rows[-1]]  # not a list of its drafts
                kept = np.full(n_rows, -5)
                for a, lst in zip(start, lists):
                    kept[a:a + len(lst)] = lst
                V.vla_pages_commit(d.p, r, i32(kept), i32([len(x) for x in lists]))
                m.commit(entries, lists)
        elif kind == "fork":
            n = int(rng.integers(1, 7))
            pairs = [(int(a), int(b)) for a, b in zip(rng.integers(-1, n_seqs + 1, n), rng.integers(-1, n_seqs + 1, n))]
            made = i32([9] * n)
            V.vla_pages_fork(d.p, i32([a for a, _ in pairs]), i32([b for _, b in pairs]), made)
            assert made.tolist() == m.fork(pairs)
        else:
            seqs = [int(x) for x in rng.integers(-1, n_seqs + 1, rng.integers(1, 4))]
            V.vla_pages_release(d.p, i32(seqs))
            m.release(seqs)
        d.same()


def test_large_pool_and_batches(V):
    """Counts beyond one round of the dealing workgroup: 1,500 sequences, a
    pool of 40,000 pages, one sequence of 3,000 pages."""
    say("large pool")
    rng = np.random.default_rng(5)
    m = U.Model(1, 40000, 1, 16, 32, 3100, 3000)
    T = T16
    k = torch.zeros(m.dims, dtype=T, device="cuda")
    d = Dev(V, m, T, k, k.clone())
    rows = [int(x) for x in rng.integers(0, 60, 1500)]
    rows[700] = 48000
    m.refs[rng.permutation(40000)[:20000]] = 1  # held elsewhere
    d.refs.copy_(i32(m.refs))
    start = np.concatenate([[0], np.cumsum(rows)])
    r = V.make_rows(i32(start), int(start[-1]))
    V.vla_pages_reserve(d.p, r)
    m.reserve(list(enumerate(rows)))
    V.vla_pages_commit(d.p, r)
    m.commit(list(enumerate(rows)), rows)
    m.k = m.v = vals(k)
    d.same()
    pairs = [(i, 1500 + i) for i in range(1500)] + [(0, 1500), (1500, 3050), (700, 3051)]
    made = i32([9] * len(pairs))
    V.vla_pages_fork(d.p, i32([a for a, _ in pairs]), i32([b for _, b in pairs]), made)
    assert made.tolist() == m.fork(pairs)
    d.same()
    V.vla_pages_release(d.p, i32(list(range(3100)) + [4, 4]))
    m.release(range(3100))
    d.same()


# --------------------------------------------------------------------------
# Together
# --------------------------------------------------------------------------

class Lm:
    """The attention part of a small LM: fixed projections, two layers, its
    values in 64 bits and its calls on the device."""

    def __init__(self, V, T, nq=4, nkv=2, hd=64, layers=2, seed=0):
        self.V, self.T, self.nq, self.nkv, self.hd, self.layers = V, T, nq, nkv, hd, layers
        rng = np.random.default_rng(seed)
        self.emb = rng.standard_normal((97, layers, nq + 2 * nkv, hd))
        half = hd // 2
        ang = np.arange(400)[:, None] * 10000.0 ** (-np.arange(half) / half)
        self.cos, self.sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
        self.qg = (1 + 0.1 * rng.standard_normal(hd)).astype(np.float32)
        self.kg = (1 + 0.1 * rng.standard_normal(hd)).astype(np.float32)
        dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        self.rope = V.make_rope_norm(dev(self.cos), dev(self.sin), dev(self.qg), dev(self.kg))

    def rows(self, toks, layer):
        return rounded(self.emb[toks, layer], self.T)

    def step(self, d, r, toks, pos, mask, stream=0):
        """Every layer's rows of the step's tokens; [layers][n][nq][hd]."""
        outs = []
        n_rows = r.n_rows
        for l in range(self.layers):
            x = torch.from_numpy(self.rows(toks, l)).to(self.T).cuda()
            q = torch.empty((n_rows, self.nq, self.hd), dtype=self.T, device="cuda")
            self.V.vla_qk_norm_rope(d.p, l, r, self.rope, x[:, :self.nq], x[:, self.nq:self.nq + self.nkv],
                                    x[:, self.nq + self.nkv:], q, pos=pos, stream=stream)
            scratch = torch.empty(self.V.vla_tree_attention_scratch(d.p, r, self.nq), dtype=torch.uint8, device="cuda")
            out = torch.empty_like(q)
            self.V.vla_tree_attention(d.p, l, r, q, out, scratch, mask=mask, stream=stream)
            outs.append(out)
        return outs

    def dense(self, path, layer):
        """The last token of a path of tokens at positions 0 .. in 64 bits,
        its keys and queries rounded as the cache rounds them; with the sum of
        p |v| that its error scales with."""
        x = self.rows(path, layer)
        q, _ = U.norm_rope(x[-1, :self.nq], self.qg.astype(np.float64), 1e-6, self.cos, self.sin, len(path) - 1)
        ks = np.stack([U.norm_rope(x[i, self.nq:self.nq + self.nkv], self.kg.astype(np.float64), 1e-6, self.cos,
                                   self.sin, i)[0] for i in range(len(path))])
        out, size = np.zeros((self.nq, self.hd)), np.zeros((self.nq, self.hd))
        dq = np.zeros(self.nq)
        g = self.nq // self.nkv
        for h in range(self.nq):
            out[h], size[h], dq[h] = U.attention_row(q[h], ks[:, h // g], x[:, self.nq + self.nkv + h // g],
                                                     np.ones(len(path), bool), self.hd ** -0.5)
        return out, size, dq


@pytest.mark.parametrize("T", [T16, T32])
def test_prompt_drafts_commit_fork_decode(V, T):
    """As a serving program uses them together: prompts enter in two chunks,
    a tree of drafts is scored, a path of it accepted, the sequence forked, and
    both branches decode on. Every row equals dense attention over its own
    path of tokens.

    Queries and keys are rounded once (2 half steps in a score, of sum |q k|),
    so a weight is off by e^(4 half ds); then as in the attention test."""
    say(f"together {T}")
    rng = np.random.default_rng(21)
    lm = Lm(V, T)
    m = U.Model(lm.layers, 40, lm.nkv, 16, lm.hd, 4, 8)
    m.k[:], m.v[:] = np.nan, np.nan  # nobody has written the pool yet
    d = Dev(V, m, T)
    V.vla_pages_init(d.p)

    def check(outs, row, path):
        for l in range(lm.layers):
            want, size, dq = lm.dense(path, l)
            rel = np.expm1(dq * (4.2 * HALF[T] + 2.0 ** -16))[:, None] + 2.0 ** -8 * (T is T16) + 200 * 2.0 ** -24
            off = np.abs(vals(outs[l][row]) - want)
            assert np.all(off <= 2 * rel * size + HALF[T] * np.abs(want)), (l, row, path)

    prompts = [list(rng.integers(0, 97, 45)), list(rng.integers(0, 97, 16))]
    for a, b in ((0, 30), (30, 45)):
        parts = [p[a:b] for p in prompts]
        start = np.concatenate([[0], np.cumsum([len(p) for p in parts])])
        r = V.make_rows(i32(start), int(start[-1]), i32([2, 0]))
        V.vla_pages_reserve(d.p, r)
        outs = lm.step(d, r, np.array(parts[0] + parts[1], int), None, None)
        torch.cuda.synchronize()
        for e in range(2):
            for i in range(len(parts[e])):
                check(outs, start[e] + i, prompts[e][:a + i + 1])
        V.vla_pages_commit(d.p, r)
    assert d.lens.tolist() == [16, 0, 45, 0]
    # trees
    n = [11, 7]
    parents = [[-1 if j < 3 else int(rng.integers(max(0, j - 5), j)) for j in range(c)] for c in n]
    toks = [list(rng.integers(0, 97, c)) for c in n]
    paths, pos, bits = [], [], []
    for e in range(2):
        ps = []
        for j, p in enumerate(parents[e]):
            ps.append((ps[p] if p >= 0 else []) + [j])
            pos.append(len(prompts[e]) + len(ps[j]) - 1)
            b = np.zeros(32, bool)
            b[ps[j]] = True
            bits.append(b)
        paths.append(ps)
    start = np.concatenate([[0], np.cumsum(n)])
    r = V.make_rows(i32(start), 18, i32([2, 0]))
    V.vla_pages_reserve(d.p, r)
    outs = lm.step(d, r, np.array(toks[0] + toks[1], int), i32(pos), torch.from_numpy(pack(np.array(bits))).cuda())
    torch.cuda.synchronize()
    for e in range(2):
        for j in range(n[e]):
            check(outs, start[e] + j, prompts[e] + [toks[e][i] for i in paths[e][j]])
    # accept the longest path of each
    acc = [max(ps, key=len) for ps in paths]
    kept = np.full(18, -1)
    for a, lst in zip(start, acc):
        kept[a:a + len(lst)] = lst
    V.vla_pages_commit(d.p, r, i32(kept), i32([len(x) for x in acc]))
    seqs = [prompts[e] + [toks[e][i] for i in acc[e]] for e in range(2)]
    made = i32([0, 0])
    V.vla_pages_fork(d.p, i32([2, 0]), i32([3, 1]), made)
    assert made.tolist() == [1, 1]
    # four branches decode three tokens of their own
    branch = {2: list(seqs[0]), 3: list(seqs[0]), 0: list(seqs[1]), 1: list(seqs[1])}
    for step in range(3):
        order = [3, 0, 2, 1]
        r = V.make_rows(i32([0, 1, 2, 3, 4]), 4, i32(order))
        new = [int(rng.integers(0, 97)) for _ in order]
        V.vla_pages_reserve(d.p, r)
        outs = lm.step(d, r, np.array(new), None, None)
        torch.cuda.synchronize()
        for i, s in enumerate(order):
            branch[s].append(new[i])
            check(outs, i, branch[s])
        V.vla_pages_commit(d.p, r)
    V.vla_pages_release(d.p, i32([0, 1, 2, 3]))
    torch.cuda.synchronize()
    assert not d.refs.any() and d.status.item() == 0 and (d.table == -1).all()


def test_a_captured_step_replays_on_what_the_arrays_hold(V):
    """Reserve, store, attention and commit of two sequences in one graph,
    replayed with eager work between: each replay decodes the next token."""
    say("graph")
    T, lm = T16, Lm(V, T16, seed=4)
    rng = np.random.default_rng(6)
    lens = [30, 5]

    def setup():
        m = filled(np.random.default_rng(9), T, lens, [0, 0], layers=2, nkv=lm.nkv, hd=lm.hd, spare=12)
        m.max_pages = m.table.shape[1]
        return Dev(V, m, T)

    toks = rng.integers(0, 97, (6, 2))
    eager, graph = setup(), setup()
    start = i32([0, 1, 2])
    bufs = [torch.empty((2, lm.nq + 2 * lm.nkv, lm.hd), dtype=T, device="cuda") for _ in range(lm.layers)]
    qs = [torch.empty((2, lm.nq, lm.hd), dtype=T, device="cuda") for _ in range(lm.layers)]
    outs = [torch.empty_like(q) for q in qs]

    def step(d, r, scratch, stream):
        V.vla_pages_reserve(d.p, r, stream=stream)
        for l in range(lm.layers):
            x = bufs[l]
            V.vla_qk_norm_rope(d.p, l, r, lm.rope, x[:, :lm.nq], x[:, lm.nq:lm.nq + lm.nkv], x[:, lm.nq + lm.nkv:],
                               qs[l], stream=stream)
            V.vla_tree_attention(d.p, l, r, qs[l], outs[l], scratch, stream=stream)
        V.vla_pages_commit(d.p, r, stream=stream)

    r = V.make_rows(start, 2)
    scratch = torch.zeros(V.vla_tree_attention_scratch(eager.p, r, lm.nq), dtype=torch.uint8, device="cuda")
    want = []
    for t in range(6):
        for l in range(lm.layers):
            bufs[l].copy_(torch.from_numpy(lm.rows(toks[t], l)).to(T))
        step(eager, r, scratch, 0)
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        g.capture_begin()
        step(graph, r, scratch, side.cuda_stream)
        g.capture_end()
    torch.cuda.synchronize()
    for t in range(6):
        for l in range(lm.layers):
            bufs[l].copy_(torch.from_numpy(lm.rows(toks[t], l)).to(T))
        scratch.fill_(t * 40)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for l in range(lm.layers):
            assert torch.equal(outs[l], want[t][l]), (t, l)
        torch.ones(1000, device="cuda").sum().item()
    assert graph.lens.tolist() == [36, 11] == eager.lens.tolist()
    assert torch.equal(graph.k, eager.k) and torch.equal(graph.table, eager.table)


def test_two_caches_on_two_streams(V):
    """Calls on different caches overlap freely; each equals its own run."""
    say("two streams")
    lm = Lm(V, T16, seed=5)
    toks = np.random.default_rng(8).integers(0, 97, 64)
    r = [V.make_rows(i32([0, 40]), 40), V.make_rows(i32([0, 64]), 64)]

    def fresh():
        out = []
        for n in (40, 64):
            m = filled(np.random.default_rng(n), T16, [100], [n], layers=2, nkv=lm.nkv, hd=lm.hd)
            out.append(Dev(V, m, T16))
        return out

    alone = []
    for i, d in enumerate(fresh()):
        alone.append(lm.step(d, r[i], toks[:r[i].n_rows], None, None))
        torch.cuda.synchronize()
    both = fresh()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for i, d in enumerate(both):
        with torch.cuda.stream(streams[i]):
            got.append(lm.step(d, r[i], toks[:r[i].n_rows], None, None, stream=streams[i].cuda_stream))
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


@pytest.mark.parametrize("cfg", ["micro-f32", "micro-bf16", "tiny", "micro_dit"])
def test_a_prefill_goes_on_in_pages(V, cfg):
    """A frame's prefix moves from its context into a sequence's pages (bit for
    bit what vla_ctx_export_kv gives, in every layer), behind slots that are
    there, and a new token attends to it."""
    import gpu_util as g
    import synth
    say(f"context to pages {cfg}")
    c = {"micro-f32": synth.micro(0), "micro-bf16": synth.micro(1), "tiny": synth.TINY,
         "micro_dit": synth.micro_dit(1)}[cfg]
    T = T16 if c["dtype"] == V.VLA_BF16 else T32
    P, nkv, hd, L = synth.derived(c)["prefix"], c["lm_kv_heads"], c["head_dim"], c["lm_layers"]
    rng = np.random.default_rng(1)
    m = filled(rng, T, [5, 18], [P + 1, P + 1], layers=L, nkv=nkv, page=16, hd=hd)
    d = Dev(V, m, T)
    with g.model(c) as model, g.context(model) as ctx:
        f = g.DevFrame(synth.make_frame(c, 0, 0))
        V.vla_vlm_prefill(model, f.c, ctx)
        for s in (1, 0):
            assert V.vla_ctx_to_pages(model, ctx, d.p, s) == P
        torch.cuda.synchronize()
        kv = [V.vla_ctx_export_kv(model, ctx, l, P * nkv * hd) for l in range(L)]
        for s in (0, 1):
            for i in range(P):
                p, at = m.where(s, int(m.lens[s]) + i)
                for l in range(L):
                    m.k[l, p, :, at] = kv[l][0].reshape(P, nkv, hd)[i]
                    m.v[l, p, :, at] = kv[l][1].reshape(P, nkv, hd)[i]
        d.same()
        for what, bad in (("layers", L + 1), ("kv_heads", nkv + 1), ("head_dim", hd + 32), ("dtype", 1 - c["dtype"])):
            p = V.make_pages(d.k, d.v, d.table, d.lens, d.held, d.refs, d.status)
            setattr(p, what, bad)
            with pytest.raises(V.VlaError) as e:
                V.vla_ctx_to_pages(model, ctx, p, 0)
            assert e.value.code == -1
        with pytest.raises(V.VlaError):
            V.vla_ctx_to_pages(model, ctx, d.p, 2)
    V.vla_pages_commit(d.p, V.make_rows(i32([0, P, 2 * P]), 2 * P))
    m.commit([(0, P), (1, P)], [P, P])
    nq = c["lm_heads"]
    q = rounded(rng.standard_normal((2, nq, hd)), T)
    r = V.make_rows(i32([0, 1, 2]), 2)
    out = torch.empty((2, nq, hd), dtype=T, device="cuda")
    scratch = torch.empty(V.vla_tree_attention_scratch(d.p, r, nq), dtype=torch.uint8, device="cuda")
    V.vla_tree_attention(d.p, L - 1, r, torch.from_numpy(q).to(T).cuda(), out, scratch)
    d.same()
    want, tol = expect(m, T, L - 1, [0, 1], [0, 1, 2], [1, 1], q, None, hd ** -0.5, 1)
    assert np.all(np.abs(vals(out) - want) <= tol)
