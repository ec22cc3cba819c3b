"""Verification of drafted tokens on the GPU, through the binding, against the
definition in 64-bit NumPy, one entry at a time. What is compared with a random
number is computed in 64 bits on both sides, so the answers are equal: a draft's
comparison is off by a few 2^-53, a running sum over n tokens by n 2^-53 of the
total, and no case below has a number that close to a border (asserted)."""
import numpy as np
import pytest
import torch

from test_gpu_paged import T16, T32, V, i32, say  # noqa: F401

pytestmark = pytest.mark.gpu


def walk(p, q, tokens, parent, u, near=None):
    """kept, next, bad of one entry: p and q [rows, vocab] in 64 bits (q None:
    chosen without chance), u None: greedy."""
    n, vocab = p.shape
    p = np.where(p > 0, p, 0)
    bad = False
    par = []
    for i in range(n):
        x = parent[i] if parent is not None else i - 1
        ok = i > 0 and 0 <= x < i and 0 <= tokens[i] < vocab
        bad = bad or (i > 0 and not ok)
        par.append(x if ok else None)
    node, path = 0, [0]
    kids = lambda k: [i for i in range(1, n) if par[i] == k]  # noqa: E731
    while True:
        step = None
        if u is None:
            best = int(np.argmax(p[node]))
            step = next((i for i in kids(node) if tokens[i] == best), None)
        else:
            s, z, left = 0.0, 1.0, p[node].copy()
            for i in kids(node):
                x = tokens[i]
                a, b = u[i] * (q[node, x] if q is not None else 1.0) * z, left[x]
                if near is not None and a != b:
                    near.append(abs(a - b) / max(a, b))
                if a < b:
                    step = i
                    break
                if q is not None:
                    s += z
                    left = np.maximum(p[node] - s * q[node], 0)
                    z = left.sum()
                else:
                    z -= left[x]
                    left[x] = 0
        if step is None:
            break
        node = step
        path.append(step)
    if u is None:
        return path, best, bad
    if not left.sum() > 0:
        left = p[node]
    cum = np.cumsum(left)
    if not 0 < cum[-1] < np.inf:
        return path, -1, True
    if near is not None:
        near.append(np.abs(cum - u[0] * cum[-1])[left > 0].min() / cum[-1] * 1e3)
    over = np.flatnonzero(cum > u[0] * cum[-1])
    return path, int(over[0] if len(over) else np.flatnonzero(left)[-1]), bad


def tree(rng, n, width):
    return [-1] + [int(rng.integers(max(0, i - 2 * width), max(1, i - width + 1))) if i > width else 0 for i in range(1, n)]


def run(V, T, probs, drafted, tokens, parent, u, start, seqs, n_seqs, pad=0, skew=0):
    """The call on whole arrays (numpy), its rows `pad` values apart from one
    another (the drafts' distributions' `skew` more)."""
    n, vocab = probs.shape

    def wide(x, pad=pad):
        if x is None:
            return None
        t = torch.full((n, vocab + pad), float("nan"), dtype=T, device="cuda")
        t[:, :vocab] = torch.from_numpy(np.array(x)).to(T).cuda()
        return t[:, :vocab]

    z = torch.zeros((1, 1, 1, 16, 32), dtype=T16, device="cuda")
    status = i32([0])
    pages = V.make_pages(z, z.clone(), i32([[-1]] * n_seqs), i32([0] * n_seqs), i32([0] * n_seqs), i32([0]), status)
    r = V.make_rows(i32(start), n, i32(seqs))
    kept = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    count, after = (torch.full((len(seqs),), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    scratch = torch.full((V.vla_verify_drafts_scratch(pages, r, vocab),), 255, dtype=torch.uint8, device="cuda")
    V.vla_verify_drafts(pages, r, i32(tokens), wide(probs), kept, count, after, scratch,
                        parent=None if parent is None else i32(parent), drafted=wide(drafted, pad + skew),
                        uniform=None if u is None else torch.from_numpy(u).cuda())
    torch.cuda.synchronize()
    return kept.cpu().numpy(), count.cpu().numpy(), after.cpu().numpy(), int(status.item())


def softmax(x):
    x = np.exp(x - x.max(-1, keepdims=True))
    return x / x.sum(-1, keepdims=True)


CASES = [
    # T, vocab, entries' rows, tree width (0: chains), drafted, greedy, row padding
    (T32, 1024, [4] * 8, 0, False, True, 0),
    (T32, 1000, [1, 5, 0, 9], 0, True, False, 0),
    (T32, 7, [9, 3, 12], 2, True, False, 0),
    (T32, 5003, [24, 40, 2], 4, True, False, 0),
    (T32, 5003, [24, 40, 2], 4, False, False, 3),
    (T16, 2050, [17, 30], 3, True, False, 1),
    (T16, 999, [20, 6, 8], 2, False, False, 0),
    (T16, 513, [12, 30, 1], 3, False, True, 5),
    (T32, 1, [3, 1], 0, True, False, 0),
    (T32, 40000, [8, 6], 0, True, False, 0),
    (T32, 70001, [5], 2, False, False, 0),
    (T32, 64, [700, 3], 30, False, False, 0),
    (T32, 64, [700, 3], 600, False, False, 0),
    (T32, 64, [600], 90, True, False, 2),
    # rows that several workgroups begin with
    (T32, 66001, [9, 4, 1, 0, 30], 3, True, False, 0),
    (T32, 65536, [8, 8, 3], 0, True, False, 0),
    (T32, 65537, [100], 90, False, False, 1),
    (T16, 80003, [7, 12], 2, True, False, 0),
    (T16, 65540, [5], 0, False, False, 4),
]


@pytest.mark.parametrize("T,vocab,rows,width,drafted,greedy,pad", CASES)
def test_verify(V, T, vocab, rows, width, drafted, greedy, pad):
    say(f"verify {T} vocab={vocab} rows={rows} width={width} drafted={drafted} greedy={greedy}")
    taken = 0
    for seed in range(4):
        rng = np.random.default_rng(vocab + sum(rows) + 1000 * seed)
        # entries in any order of sequences, one of them padding, rows of nobody behind
        counts = rows + [2]
        seqs = list(rng.permutation(len(rows))) + [-1]
        start = np.concatenate([[0], np.cumsum(counts)])
        n = int(start[-1]) + 2
        logits = rng.standard_normal((n, vocab)) * 2
        probs = torch.from_numpy(softmax(logits)).to(T).to(torch.float64).numpy()
        q = torch.from_numpy(softmax(0.8 * logits + 0.6 * rng.standard_normal((n, vocab)))).to(T).to(torch.float64).numpy()
        parent = np.full(n, -3, np.int64)
        tokens = rng.integers(0, vocab, n)
        for a, c in zip(start, counts):
            par = tree(rng, c, width) if width else list(range(-1, c - 1))
            parent[a:a + c] = par[:c]
            for i in range(1, c):
                w = q[a + par[i]] / q[a + par[i]].sum()
                tokens[a + i] = int(np.argmax(probs[a + par[i]])) if greedy and rng.random() < 0.7 else rng.choice(vocab, p=w)
        u = None if greedy else rng.random(n).astype(np.float32)
        got = run(V, T, probs, q if drafted else None, tokens, parent if width else None, u, start, seqs, len(rows), pad)
        near = []
        kept, count, after = np.full(n, -7), np.full(len(seqs), -7), np.full(len(seqs), -7)
        for e, (s, a, c) in enumerate(zip(seqs, start, counts)):
            if s < 0:
                continue
            if c == 0:
                count[e], after[e] = 0, -1
                continue
            path, after[e], bad = walk(probs[a:a + c], q[a:a + c] if drafted else None, tokens[a:a + c],
                                       parent[a:a + c] if width else None,
                                       None if u is None else u[a:a + c].astype(np.float64), near)
            assert not bad
            kept[a:a + c] = path + [-1] * (c - len(path))
            count[e] = len(path)
            taken += len(path) - 1
        assert all(x > 1e-11 for x in near)
        assert np.array_equal(got[1], count), (got[1], count)
        assert np.array_equal(got[0], kept)
        assert np.array_equal(got[2], after), (got[2], after)
        assert got[3] == 0
    # (the test tries something; drafts chosen without chance from a flat target are seldom kept)
    assert taken > 0 or not (drafted or greedy)


@pytest.mark.parametrize("T,vocab", [(T32, 4001), (T16, 4001), (T32, 70000), (T16, 65541)])
def test_rows_of_two_alignments(V, T, vocab):
    """The draft's rows need not lie as the target's do."""
    say(f"verify alignments {T} vocab={vocab}")
    rng = np.random.default_rng(vocab)
    n = 24
    p, q = (torch.from_numpy(softmax(2 * rng.standard_normal((n, vocab)))).to(T).to(torch.float64).numpy() for _ in range(2))
    parent = [-1, 0, 0, 0, 1, 2, 3, 3] * 3
    tokens, u = rng.integers(0, vocab, n), rng.random(n).astype(np.float32)
    got = [run(V, T, p, q, tokens, parent, u, [0, 8, 16, 24], [0, 1, 2], 3, pad, skew)
           for pad, skew in ((0, 0), (0, 1), (3, 2), (1, 7))]
    for g in got[1:]:
        assert all(np.array_equal(x, y) for x, y in zip(g, got[0]))
    for e in range(3):
        path, after, _ = walk(p[8 * e:8 * e + 8], q[8 * e:8 * e + 8], tokens[8 * e:8 * e + 8], parent[:8],
                              u[8 * e:8 * e + 8].astype(np.float64))
        assert got[0][1][e] == len(path) and got[0][2][e] == after


def test_edges(V):
    """Ties, drafts that cannot be tried, nothing left of a target, no target."""
    say("verify edges")
    f = lambda *x: np.array(x, np.float64)  # noqa: E731
    nan, inf = float("nan"), float("inf")
    one = f(0.25, 0.25, 0.25, 0.25)
    # greedy: the lowest of several; NaN is nothing; a row of nothing has no likeliest
    P = np.array([f(0.1, 0.4, 0.4, 0.1), f(nan, 0.2, 0.7, 0.1), f(0, 0, 0, 0.5), f(nan, nan, nan, nan)])
    got = run(V, T32, P, None, [0, 1, 2, 3], None, None, [0, 4], [0], 1)
    assert list(got[0]) == [0, 1, 2, 3] and got[1][0] == 4 and got[2][0] == -1 and got[3] == V.PAGES_BAD
    got = run(V, T32, P[:2], None, [0, 2], None, None, [0, 2], [0], 1)
    assert list(got[0]) == [0, -1] and got[1][0] == 1 and got[2][0] == 1 and got[3] == 0
    # tokens outside the vocabulary, parents that do not stand before: passed over
    P = np.array([one] * 5)
    u = np.array([0.6, 0, 0, 0, 0], np.float32)
    got = run(V, T32, P, None, [0, 4, -1, 2, 3], [-1, 0, 0, 3, 0], u, [0, 5], [0], 1)
    assert list(got[0]) == [0, 4, -1, -1, -1] and got[1][0] == 2 and got[2][0] == 2 and got[3] == V.PAGES_BAD
    # numbers on the border: u q Z < r is strict, the sum has to pass u times the total
    for u1, k in ((0.25, 1), (np.nextafter(np.float32(0.25), np.float32(0)), 2)):
        got = run(V, T32, P[:2], None, [0, 3], None, np.array([0.0, u1], np.float32), [0, 2], [0], 1)
        assert got[1][0] == k and got[2][0] == 0
    for u0, t in ((0.0, 0), (0.25, 1), (0.75, 3), (1.0, 3)):
        got = run(V, T32, P[:1], None, [0], None, np.array([u0], np.float32), [0, 1], [0], 1)
        assert got[2][0] == t
    # the draft's distribution is the target's: a refused one leaves nothing, so all of the target counts
    got = run(V, T32, P[:2], P[:2], [0, 1], None, np.array([0.5, 1.0], np.float32), [0, 2], [0], 1)
    assert got[1][0] == 1 and got[2][0] == 2 and got[3] == 0
    # the same without chance: every token was drafted and refused
    got = run(V, T32, P, None, [0, 0, 1, 2, 3], [-1, 0, 0, 0, 0], np.array([0.9, 1, 1, 1, 1], np.float32), [0, 5], [0], 1)
    assert got[1][0] == 1 and got[2][0] == 3 and got[3] == 0
    # the same token twice: refused once, it is not there any more
    got = run(V, T32, P[:3], None, [0, 1, 1], [-1, 0, 0], np.array([0.4, 0.9, 0.0], np.float32), [0, 3], [0], 1)
    assert got[1][0] == 1 and got[2][0] == 2 and got[3] == 0
    # no target to draw from
    for row in (f(0, 0, 0, 0), f(nan, -1, 0, nan), f(0, inf, 0, 0)):
        got = run(V, T32, row[None], None, [0], None, np.array([0.5], np.float32), [0, 1], [0], 1)
        assert got[1][0] == 1 and got[2][0] == -1 and got[3] == V.PAGES_BAD


def test_answers_are_distributed_as_the_target(V):
    """Over many entries with numbers of their own the first token behind the
    decided one is distributed as the target: 60,000 answers over 5 tokens are
    within 5 standard deviations, sqrt(p (1 - p) / n) each."""
    say("verify distribution")
    n, vocab = 60000, 5
    rng = np.random.default_rng(4)
    p, q = softmax(rng.standard_normal((2, vocab)) * 1.3)
    p, q = p.astype(np.float32).astype(np.float64), q.astype(np.float32).astype(np.float64)
    for drafted in (True, False):
        # three drafts of one parent each: drawn from q, or the first three tokens
        tokens = np.zeros((n, 4), np.int64)
        tokens[:, 1:] = rng.choice(vocab, (n, 3), p=q / q.sum()) if drafted else [[0, 1, 2]]
        u = rng.random((n, 4)).astype(np.float32)
        probs = np.broadcast_to(p, (4 * n, vocab))
        got = run(V, T32, probs, np.broadcast_to(q, (4 * n, vocab)) if drafted else None, tokens.reshape(-1),
                  np.tile([-1, 0, 0, 0], n), u.reshape(-1), np.arange(n + 1) * 4, np.arange(n), n)
        kept = got[0].reshape(n, 4)[:, 1]
        first = np.where(kept > 0, tokens[np.arange(n), np.maximum(kept, 0)], got[2])
        share = np.bincount(first, minlength=vocab) / n
        assert np.all(np.abs(share - p / p.sum()) < 5 * np.sqrt(p * (1 - p) / n)), (share, p)
        assert got[3] == 0


ODD = [
    # T, vocab, rows, tree width: one workgroup an entry, and several at first
    (T32, 5, 40, 6), (T32, 3001, 24, 4), (T16, 2050, 17, 3), (T32, 300, 9, 0), (T32, 66001, 30, 4), (T16, 80003, 12, 2),
]


@pytest.mark.parametrize("T,vocab,rows,width", ODD)
def test_odd_values_of_the_drafts(V, T, vocab, rows, width):
    """Negative probabilities and NaN count as 0 in the drafts' distributions as
    in the target's: the answers are those of the clean ones."""
    say(f"verify odd drafted {T} vocab={vocab} rows={rows}")
    for seed in range(4):
        rng = np.random.default_rng(vocab + rows + 1000 * seed)
        n = 3 * rows
        p, q = (torch.from_numpy(softmax(2 * rng.standard_normal((n, vocab)))).to(T).to(torch.float64).numpy() for _ in range(2))
        for x in (p, q):
            at = rng.random(x.shape)
            at[:, 0] = 0.5  # (something is left of every row)
            x[at < 0.15] = np.nan
            x[(at >= 0.15) & (at < 0.35)] *= -1
            x[at > 0.9] = 0
        clean = np.where(q > 0, q, 0)
        parent = np.concatenate([tree(rng, rows, width) if width else np.arange(-1, rows - 1) for _ in range(3)])
        tokens, u = rng.integers(0, vocab, n), rng.random(n).astype(np.float32)
        u[rng.random(n) < 0.2] = 0
        # (tokens whose q is odd among those that are tried)
        for i in range(n):
            row = i // rows * rows + max(0, int(parent[i]))
            odd = np.flatnonzero(~(q[row] >= 0))
            if len(odd) and rng.random() < 0.5:
                tokens[i] = rng.choice(odd)
        start = [0, rows, 2 * rows, n]
        got = run(V, T, p, q, tokens, parent if width else None, u, start, [0, 1, 2], 3)
        near = []
        for e in range(3):
            s = slice(e * rows, (e + 1) * rows)
            path, after, bad = walk(p[s], clean[s], tokens[s], parent[s] if width else None, u[s].astype(np.float64), near)
            assert got[1][e] == len(path) and got[2][e] == after and not bad
            assert list(got[0][s]) == path + [-1] * (rows - len(path))
        assert all(x > 1e-11 for x in near)
        assert got[3] == 0


@pytest.mark.parametrize("T", [T32, T16])
def test_odd_drafted_one_by_one(V, T):
    """A token whose target is 0 is not kept for a negative q, nor refused for a
    NaN; what is left of a target never passes it."""
    say(f"verify odd drafted one by one {T}")
    nan = float("nan")
    P = np.array([[0.0, 0.5, 0.25, 0.25]] * 2)
    half = np.array([0.5, 0.5], np.float32)

    def answer(q, token, u=half):
        got = run(V, T, P, np.array([q] * 2, np.float64), [0, token], None, u, [0, 2], [0], 1)
        assert got[3] == 0
        return int(got[1][0]), int(got[2][0])

    # p = 0: refused whatever q is; all of the target is left (q is 0 elsewhere): sums 0.5, 0.75, 1
    for x in (-0.5, nan, 0.0):
        assert answer([x, 0, 0, 0], 0, np.array([0.6, 0.5], np.float32)) == (1, 2)
    # p > 0 and q 0: kept
    for x in (-0.5, nan, 0.0):
        assert answer([0, x, 0, 0], 1)[0] == 2
    # token 2 is refused (u q = 0.5 > 0.25) and leaves max(p - q, 0) = 0, 0.5, 0, 0.25 beside a q of 0, negative or NaN
    for x in (-1.0, nan, 0.0):
        for u0, want in ((0.3, 1), (0.9, 3)):
            assert answer([x, x, 1, x], 2, np.array([u0, 0.5], np.float32)) == (1, want)


@pytest.mark.parametrize("T,vocab", [(T32, 9), (T16, 4001), (T32, 70001)])
def test_infinite_drafted(V, T, vocab):
    """All of a target is left where no draft of it was refused, whatever q holds;
    of a token whose q is infinite nothing is left where one was."""
    say(f"verify infinite drafted {T} vocab={vocab}")
    P = np.zeros((3, vocab))
    P[:, [1, vocab - 2, vocab - 1]] = 0.5, 0.25, 0.25
    q = np.zeros((3, vocab))
    q[:, 1] = np.inf
    for u0, want in ((0.25, 1), (0.625, vocab - 2), (0.875, vocab - 1)):
        u = np.array([u0, 0.5, 0.5], np.float32)
        # no draft; one that is kept (its q is 0)
        got = run(V, T, P[:1], q[:1], [0], None, u[:1], [0, 1], [0], 1)
        assert got[1][0] == 1 and got[2][0] == want and got[3] == 0
        got = run(V, T, P[:2], q[:2], [0, vocab - 1], None, u[:2], [0, 2], [0], 1)
        assert got[1][0] == 2 and got[2][0] == want and got[3] == 0
        # token 0 (p = 0) is refused first: half of the rest to each of the last two
        got = run(V, T, P, q, [0, 0, 1], [-1, 0, 0], u, [0, 3], [0], 1)
        assert got[1][0] == 1 and got[2][0] == (vocab - 2 if u0 < 0.5 else vocab - 1) and got[3] == 0


@pytest.mark.parametrize("kind", ["greedy", "chosen", "drawn"])
@pytest.mark.parametrize("vocab", [50, 70000])
def test_a_batch_without_rows(V, kind, vocab):
    """Entries without rows are answered where the whole batch has none, too;
    padding is left as it was."""
    say(f"verify no rows {kind} vocab={vocab}")
    probs = np.zeros((0, vocab))
    none = np.zeros(0, np.float32)
    got = run(V, T32, probs, probs if kind == "drawn" else None, none, None, None if kind == "greedy" else none,
              [0, 0, 0, 0, 0], [1, -1, 0, 7], 2)
    assert list(got[1]) == [0, -7, 0, -7] and list(got[2]) == [-1, -7, -1, -7] and got[3] == 0


def test_likeliest_of_odd_rows(V):
    """The likeliest token is looked for among the values as they are, NaN left
    out, so that logits will do."""
    say("verify likeliest of odd rows")
    nan, inf = float("nan"), float("inf")
    rows = [([-3, -1, -2, nan], 1), ([-1, 0, -1, 0], 1), ([nan, -inf, -5, -5], 2), ([-inf] * 4, -1), ([nan] * 4, -1),
            ([0, inf, 1, inf], 1), ([nan, 0, 0, 0], 1)]
    for T in (T32, T16):
        for row, best in rows:
            got = run(V, T, np.array([row, [0, 0, 0, 1]], np.float64), None, [0, max(best, 0)], None, None, [0, 2], [0], 1)
            assert got[1][0] == (2 if best >= 0 else 1) and got[2][0] == (3 if best >= 0 else -1)
            assert got[3] == (0 if best >= 0 else V.PAGES_BAD)
