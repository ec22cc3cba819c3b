"""Measured cases of the paged cache's further operators: attention whose
scores are capped, biased by distance, windowed or held in documents; the
weight that slots receive; the cache's slimming by that weight; and the
verification of drafted tokens.

Kinds of case:

* ``attend``  ``vla_score_attention``: as ``vla_tree_attention``, with a tanh
              cap, slopes over the distance, a window, and spans of slots; its
              log-sum-exp beside the result;
* ``weigh``   ``vla_attention_mass``: the attention weight that each slot
              receives from the rows' queries, added to what it has;
* ``evict``   ``vla_pages_evict``: long sequences keep their first slots, their
              last ones and the heaviest of the others, and close ranks;
* ``verify``  ``vla_verify_drafts``: which drafted tokens the target's
              probabilities keep, and the token behind them.

The plain forms compute with elementary torch operations, in 32 bits, sums of
slot weights and what is compared with a random number in 64, and round once at
the end. Lengths, row counts, trees and documents come from the case (its
``mix``), so that the work of a case is known; values, the order of the pages
in the pool, tokens and random numbers come from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"


# --------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------

def listed():
    return [
        # one token of each of eight robots over its prefix, capped scores:
        # the smallest call, all latency (head layout of the PaliGemma-shaped LM)
        dict(name="attend_cap_decode8", kind="attend", dtype="bf16", seqs=8, len_lo=305, len_hi=420, rows_lo=1, rows_hi=1,
             nq=8, nkv=1, hd=256, page=32, tree=0, cap=50.0, bias=False, window=0, span="", mix=21),
        # single tokens over long, uneven caches, slopes over the distance:
        # the cache's bandwidth
        dict(name="attend_bias_long", kind="attend", dtype="bf16", seqs=16, len_lo=8000, len_hi=65000, rows_lo=1,
             rows_hi=1, nq=32, nkv=8, hd=128, page=64, tree=0, cap=0.0, bias=True, window=0, span="", mix=22),
        # chunks of two long prompts, capped scores in a sliding window: matrix
        # products and exponentials
        dict(name="attend_cap_chunk", kind="attend", dtype="bf16", seqs=2, len_lo=2000, len_hi=6000, rows_lo=2000,
             rows_hi=2048, nq=32, nkv=8, hd=128, page=64, tree=0, cap=30.0, bias=False, window=4096, span="", mix=23),
        # fp32 chunks of several documents with a prefix that sees all of
        # itself, three queries to a key head, odd head dim
        dict(name="attend_f32_spans", kind="attend", dtype="f32", seqs=5, len_lo=30, len_hi=700, rows_lo=17, rows_hi=301,
             nq=6, nkv=2, hd=96, page=16, tree=0, cap=0.0, bias=True, window=0, span="docs", mix=24),
        # the weight that slots receive from single tokens
        dict(name="weigh_long", kind="weigh", dtype="bf16", seqs=16, len_lo=8000, len_hi=65000, rows_lo=1, rows_hi=1,
             nq=32, nkv=8, hd=128, page=64, tree=0, cap=0.0, bias=False, window=0, span="", mix=25),
        # and from the chunk of a prompt
        dict(name="weigh_chunk", kind="weigh", dtype="bf16", seqs=2, len_lo=2000, len_hi=6000, rows_lo=2000, rows_hi=2048,
             nq=32, nkv=8, hd=128, page=64, tree=0, cap=0.0, bias=False, window=0, span="", mix=26),
        # from fp32 trees with capped scores
        dict(name="weigh_f32_trees", kind="weigh", dtype="f32", seqs=5, len_lo=30, len_hi=700, rows_lo=17, rows_hi=61,
             nq=6, nkv=2, hd=96, page=16, tree=6, cap=20.0, bias=False, window=0, span="", mix=27),
        # eight robots' histories cut back to 600 slots (18 layers, one KV head)
        dict(name="evict8", kind="evict", dtype="bf16", seqs=8, len_lo=700, len_hi=1500, keep=600, first=4, last=128,
             nkv=1, hd=256, page=32, layers=18, mix=28),
        # sixteen longer sequences, grouped heads: bandwidth
        dict(name="evict16", kind="evict", dtype="bf16", seqs=16, len_lo=1800, len_hi=4000, keep=1600, first=4, last=256,
             nkv=8, hd=128, page=64, layers=28, mix=29),
        # chains of three greedy drafts over the preset's vocabulary
        dict(name="verify_greedy8", kind="verify", dtype="f32", entries=8, rows_lo=4, rows_hi=4, vocab=1024, tree=0,
             drafted=False, greedy=True, mix=30),
        # sixty-four chains of seven sampled drafts, a large vocabulary
        dict(name="verify_chain64", kind="verify", dtype="f32", entries=64, rows_lo=8, rows_hi=8, vocab=131072, tree=0,
             drafted=True, greedy=False, mix=31),
        # eight trees of 24 to 40 drafts, an odd vocabulary
        dict(name="verify_tree8", kind="verify", dtype="f32", entries=8, rows_lo=24, rows_hi=40, vocab=50001, tree=4,
             drafted=True, greedy=False, mix=32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "weigh", "evict", "verify"])
    mix = rng.randrange(1 << 20)
    if kind == "verify":
        drafted = rng.random() < 0.6
        c = dict(kind=kind, dtype=rng.choice(["f32", "f32", "bf16"]), entries=_log_int(rng, 1, 64), rows_lo=1,
                 rows_hi=_log_int(rng, 2, 48), vocab=_log_int(rng, 500, 131072), tree=rng.choice([0, 0, 1, 2, 3, 6]),
                 drafted=drafted, greedy=not drafted and rng.random() < 0.4, mix=mix)
        # at most the probabilities of 512 rows of 131,072
        c["entries"] = max(1, min(c["entries"], 2 ** 26 // (c["rows_hi"] * c["vocab"])))
        c["rows_lo"] = rng.randint(1, c["rows_hi"])
        return c
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    esz = 2 if dtype == "bf16" else 4
    hd = rng.choice([32, 64, 96, 128] if dtype == "f32" else [32, 64, 96, 128, 160, 256])
    nkv = rng.choice([1, 1, 2, 4, 8])
    page = rng.choice([16, 32, 64, 128, 256])
    c = dict(kind=kind, dtype=dtype, hd=hd, nkv=nkv, page=page, mix=mix)
    if kind == "evict":
        hi = _log_int(rng, 40, 4000)
        c.update(seqs=_log_int(rng, 1, 32), len_lo=max(2, hi // rng.choice([1, 2, 4])), len_hi=hi)
        c["keep"] = rng.randint(max(1, hi // 8), hi)
        c["first"] = min(rng.choice([0, 1, 4, 7]), c["keep"] // 2)
        c["last"] = rng.randint(0, c["keep"] - c["first"])
        # at most 2^30 values of K in the pool
        c["layers"] = max(1, min(rng.randint(1, 28), 2 ** 30 // (c["seqs"] * (hi + page) * nkv * hd)))
        return c
    c["nq"] = nq = nkv * rng.choice([1, 2, 3, 4, 5, 8])
    form = rng.choice(["one", "tree", "chunk"])
    c["seqs"] = _log_int(rng, 1, 48)
    if form == "one":
        lo = hi = 1
    elif form == "tree":
        lo, hi = 2, _log_int(rng, 3, 90)
    else:
        hi = _log_int(rng, 32, 2048)
        lo = rng.randint(1, hi)
    ctx = _log_int(rng, 8, 60000)
    c.update(rows_lo=lo, rows_hi=hi, tree=rng.randint(1, 12) if form == "tree" else 0, len_hi=ctx,
             len_lo=max(1, ctx // rng.choice([1, 2, 8, 30])), cap=rng.choice([0.0, 0.0, 15.0, 30.0, 50.0]),
             bias=rng.random() < 0.4, window=rng.choice([0, 0, _log_int(rng, 8, 8000)]),
             span=rng.choice(["", "docs", "prefix"]) if form == "chunk" else "")
    # at most 512 MiB of K, 2^29 scores and 2^36 products (fp32: half as many)
    for _ in range(40):
        keys = c["seqs"] * (c["len_hi"] + c["rows_hi"])
        if keys * nkv * hd * esz <= 2 ** 29 and keys * c["rows_hi"] * nq * max(hd, 64) * esz <= 2 ** 37 \
                and keys * c["rows_hi"] * nq <= 2 ** 29:
            break
        if c["seqs"] > 1:
            c["seqs"] = (c["seqs"] + 1) // 2
        else:
            c["len_hi"] = max(8, c["len_hi"] * 2 // 3)
            c["rows_hi"] = max(1, c["rows_hi"] * 2 // 3)
    c["len_lo"], c["rows_lo"] = min(c["len_lo"], c["len_hi"]), min(c["rows_lo"], c["rows_hi"])
    return c


# --------------------------------------------------------------------------
# Shapes of a case
# --------------------------------------------------------------------------

def _parents(rng, n, w, first):
    """Parents of n drafts in levels of about w; `first` stands for the token
    above the first level."""
    return [first if j < w else rng.randint(max(0, j - 2 * w + 1), max(0, j - w)) for j in range(n)]


def _layout(case):
    """Lengths and row counts of the case's sequences, the parents of drafted
    tokens (-1: a child of the cache's last token), and spans."""
    rng = random.Random(case["mix"])
    lens = [_log_int(rng, case["len_lo"], case["len_hi"]) for _ in range(case["seqs"])]
    if case["kind"] == "evict":
        return lens, None, None, None
    rows = [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in lens]
    parents = spans = None
    if case["tree"]:
        parents = [_parents(rng, r, case["tree"], -1) for r in rows]
    if case["span"] == "docs":
        # documents of some tens to some hundreds of slots: a row sees its own
        # from its first slot on, the first half of the chunk's first document
        # as a prefix that sees all of itself
        spans = []
        for n, r in zip(lens, rows):
            cuts = [0]
            while cuts[-1] < n + r:
                cuts.append(cuts[-1] + rng.randint(20, 400))
            for i in range(r):
                lo = max(x for x in cuts if x <= n + i)
                end = min(x for x in cuts if x > n)
                pre = min(n + r, n + (end - n) // 2)
                spans.append((lo, max(n + i + 1, pre) if n + i < end else n + i + 1))
    elif case["span"] == "prefix":
        spans = []
        for n, r in zip(lens, rows):
            pre = rng.randint(0, r)
            spans += [(0, n + max(pre, i + 1)) for i in range(r)]
    return lens, rows, parents, spans


def _pages(n, page):
    return (n + page - 1) // page


def _depths(par):
    d = []
    for p in par:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _seen(case):
    """Keys that some row of a sequence sees, summed over the sequences, and
    pairs of a row and a key that it sees."""
    lens, rows, parents, spans = _layout(case)
    w = case["window"] or 1 << 30
    keys = pairs = at = 0
    for b, (n, r) in enumerate(zip(lens, rows)):
        if parents:
            d = _depths(parents[b])
            pairs += sum(min(n, w - 1 - x) if w > x else 0 for x in d) + sum(min(x + 1, w) for x in d)
            keys += min(n, w - 1) + r
            continue
        lo = [max(0, n + i + 1 - w, spans[at + i][0] if spans else 0) for i in range(r)]
        hi = [spans[at + i][1] if spans else n + i + 1 for i in range(r)]
        pairs += sum(max(0, y - x) for x, y in zip(lo, hi))
        keys += max(hi) - min(lo)
        at += r
    return keys, pairs, sum(rows)


def work(case):
    esz = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind == "verify":
        rows, _ = _trees(case)
        # a row of the target's (and the draft's) for each entry's next token
        read = case["entries"] * case["vocab"] * (2 if case["drafted"] else 1)
        return {"bytes": read * esz + sum(rows) * 16 + case["entries"] * 8, "flops": 0}
    hd, nkv = case["hd"], case["nkv"]
    if kind == "evict":
        lens = _layout(case)[0]
        moved = sum(case["keep"] - case["first"] for n in lens if n > case["keep"])
        weights = case["layers"] * nkv * 4 * (sum(lens) + sum(min(n, case["keep"]) for n in lens))
        return {"bytes": 4 * moved * case["layers"] * nkv * hd * esz + weights, "flops": 0}
    keys, pairs, n = _seen(case)
    q = n * case["nq"] * hd
    extra = n * 4 * ((case["rows_hi"] + 31) // 32) if case["tree"] else 8 * n if case["span"] else 0
    if kind == "attend":
        return {"bytes": 2 * keys * nkv * hd * esz + 2 * q * esz + n * case["nq"] * 4 + extra,
                "flops": 4.0 * pairs * case["nq"] * hd}
    return {"bytes": keys * nkv * (hd * esz + 8) + q * esz + n * case["nq"] * 4 + extra,
            "flops": 2.0 * pairs * case["nq"] * hd}


def _trees(case):
    """Rows of a case's entries (the token that is decided, then its drafts)
    and the parents of all but the first (None: chains)."""
    rng = random.Random(case["mix"])
    rows = [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["entries"])]
    if not case["tree"]:
        return rows, None
    return rows, [[-1] + [p + 1 for p in _parents(rng, r - 1, case["tree"], -1)] for r in rows]


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = _prepare_drafts(case, gen) if case["kind"] == "verify" else _prepare_cache(case, seed, gen)
    s["kind"] = case["kind"]
    if own:
        import paper_2609_22335_amd as V
        _own_state(case, s, V)
    return s


def _prepare_cache(case, seed, gen):
    rng = random.Random(seed * 2 + 1)
    T = _type(case)
    lens, rows, parents, spans = _layout(case)
    page, kind, nkv, hd = case["page"], case["kind"], case["nkv"], case["hd"]
    layers = case.get("layers", 1)
    # the pool: sequences' pages in random order, as after some time of use
    need = [_pages(n + r, page) for n, r in zip(lens, rows or [0] * len(lens))]
    n_pages, wide = sum(need) + 8, max(need) + 1
    order = list(range(n_pages))
    rng.shuffle(order)
    table, refs, at = [[-1] * wide for _ in lens], [0] * n_pages, 0
    for s, n in enumerate(need):
        table[s][:n] = order[at:at + n]
        for p in order[at:at + n]:
            refs[p] = 1
        at += n
    shape = (layers, n_pages, nkv, page, hd)
    s = dict(page=page, hd=hd, nkv=nkv, layer=layers - 1,
             k=torch.randn(shape, dtype=T, device=DEV, generator=gen),
             v=torch.randn(shape, dtype=T, device=DEV, generator=gen),
             table=_i32(table), lens=_i32(lens), held=_i32(need), refs=_i32(refs), status=_i32([0]))
    # what slots have received so far: few have much
    weights = (layers, len(lens), nkv, wide * page)
    s["mass"] = torch.rand(weights, device=DEV, generator=gen).pow_(6)
    if kind == "evict":
        # (behind the committed slots there is nothing)
        s["mass"] *= torch.arange(wide * page, device=DEV) < s["lens"][:, None, None]
        s["mass_out"] = torch.zeros_like(s["mass"])
        s["seqs"] = _i32(list(range(len(lens))))
        s["keep"] = _i32([case["keep"]] * len(lens))
        s["first"], s["last"], s["most"] = case["first"], case["last"], max(min(n, case["keep"]) for n in lens)
        s["kept"] = torch.full((len(lens), wide * page), -1, dtype=torch.int32, device=DEV)
        s["before"] = [s[x].clone() for x in ("table", "lens", "held", "refs")]
        return s
    start = [0]
    for r in rows:
        start.append(start[-1] + r)
    s["start"], s["n_rows"], s["max_rows"], s["nq"] = _i32(start), start[-1], max(rows), case["nq"]
    s["mask"] = s["depth"] = s["span"] = s["slopes"] = None
    if parents:
        s["depth"] = _i32([d for p in parents for d in _depths(p)])
        words = (max(rows) + 31) // 32
        bits = []
        for p in parents:
            seen = []
            for j, q in enumerate(p):
                seen.append((1 << j) | (seen[q] if q >= 0 else 0))
            bits += [[(b >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for b in seen]
        s["mask"] = torch.tensor(bits, dtype=torch.int64, device=DEV).to(torch.int32)  # the low 32 bits
    if spans:
        s["span"] = _i32(spans)
    s["cap"], s["window"] = case["cap"], case["window"]
    if case["bias"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / case["nq"]) for h in range(case["nq"])],
                                   dtype=torch.float32, device=DEV)
    # scores of a few units, so that a cap of some tens bends the large ones
    s["q"] = (4 * torch.randn((s["n_rows"], case["nq"], hd), device=DEV, generator=gen)).to(T)
    s["lse"] = torch.empty((s["n_rows"], case["nq"]), device=DEV)
    if kind == "attend":
        s["out"] = torch.empty_like(s["q"])
    else:
        s["lse"].copy_(_by_row(s, _log_sum(_scores(s))))
    return s


def _prepare_drafts(case, gen):
    rows, parents = _trees(case)
    start = [0]
    for r in rows:
        start.append(start[-1] + r)
    n, V, T = start[-1], case["vocab"], _type(case)
    s = dict(entries=case["entries"], n_rows=n, vocab=V, max_rows=max(rows), greedy=case["greedy"], start=_i32(start))
    flat = [p for i, r in enumerate(rows) for p in (parents[i] if parents else range(-1, r - 1))]
    s["parent"] = _i32(flat) if parents else None
    # a sharp target and a draft model that is close to it
    logits = 3 * torch.randn((n, V), device=DEV, generator=gen)
    s["probs"] = torch.softmax(logits, -1).to(T)
    logits = 0.9 * logits + 0.7 * torch.randn((n, V), device=DEV, generator=gen)
    draft = torch.softmax(logits, -1).to(T)
    s["drafted"] = draft if case["drafted"] else None
    # a draft is drawn from its parent's distribution (greedy: mostly the
    # target's likeliest token)
    above = [start[i] + max(0, flat[start[i] + j]) for i, r in enumerate(rows) for j in range(r)]
    if case["greedy"]:
        best = _likeliest(s["probs"])[above]
        miss = torch.rand(n, device=DEV, generator=gen) < 0.2
        s["tokens"] = torch.where(miss, torch.randint(V, (n,), device=DEV, generator=gen), best).int()
        s["uniform"] = None
    else:
        kids, which = {}, []  # a row's place among its parent's children
        for i, a in enumerate(above):
            which.append(kids.get(a, 0))
            kids[a] = which[-1] + (i not in start)
        drawn = torch.multinomial(draft.float(), max(which) + 1, replacement=True, generator=gen)
        s["tokens"] = drawn[above, which].int()
        s["uniform"] = torch.rand(n, device=DEV, generator=gen)
    s["kept"], s["n_kept"], s["next"] = _i32([-1] * n), _i32([0] * len(rows)), _i32([0] * len(rows))
    # the cache whose sequences the entries are: its status is what the call writes of it
    one = (1, 1, 1, 16, 32)
    s.update(k=torch.zeros(one, dtype=torch.bfloat16, device=DEV), v=torch.zeros(one, dtype=torch.bfloat16, device=DEV),
             table=_i32([[-1]] * len(rows)), lens=_i32([0] * len(rows)), held=_i32([0] * len(rows)), refs=_i32([0]),
             status=_i32([0]))
    return s




def _own_state(case, s, V):
    s["V"] = V
    s["pages"] = V.make_pages(s["k"], s["v"], s["table"], s["lens"], s["held"], s["refs"], s["status"])
    kind = case["kind"]
    if kind == "evict":
        n = V.vla_pages_evict_scratch(s["pages"], case["seqs"])
    else:
        s["rows"] = V.make_rows(s["start"], s["n_rows"])
        if kind == "verify":
            n = V.vla_verify_drafts_scratch(s["pages"], s["rows"], case["vocab"])
        else:
            s["scores"] = V.make_scores(s["pages"], cap=s["cap"], slopes=s["slopes"], window=s["window"],
                                        depth=s["depth"], span=s["span"])
            size = V.vla_score_attention_scratch if kind == "attend" else V.vla_attention_mass_scratch
            n = size(s["pages"], s["rows"], s["nq"])
    s["scratch"] = torch.zeros(max(n, 16), dtype=torch.uint8, device=DEV)


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _own_attend(s):
    s["V"].vla_score_attention(s["pages"], s["layer"], s["rows"], s["scores"], s["q"], s["out"], s["scratch"],
                               lse=s["lse"], mask=s["mask"])
    return s["out"], s["lse"]


def _own_weigh(s):
    s["V"].vla_attention_mass(s["pages"], s["layer"], s["rows"], s["scores"], s["q"], s["lse"], s["mass"],
                              s["scratch"], mask=s["mask"])
    return s["mass"]


def _restore(s):
    s["table"].copy_(s["before"][0])
    s["lens"].copy_(s["before"][1])
    s["held"].copy_(s["before"][2])
    s["refs"].copy_(s["before"][3])


def _own_evict(s):
    _restore(s)
    s["V"].vla_pages_evict(s["pages"], s["seqs"], s["keep"], s["mass"], s["mass_out"], s["kept"], s["scratch"],
                           first=s["first"], last=s["last"])
    return s["k"], s["v"], s["mass_out"], s["kept"], s["table"], s["lens"], s["held"], s["refs"]


def _own_verify(s):
    s["V"].vla_verify_drafts(s["pages"], s["rows"], s["tokens"], s["probs"], s["kept"], s["n_kept"], s["next"],
                             s["scratch"], parent=s["parent"], drafted=s["drafted"], uniform=s["uniform"])
    return s["kept"], s["n_kept"], s["next"]


def _row_index(s):
    """The sequence and the index in it of every row."""
    t = torch.arange(s["n_rows"], device=DEV)
    seq = torch.searchsorted(s["start"][1:].long(), t, right=True)
    return seq, t - s["start"][seq].long()


def _by_row(s, x):
    """[B, nkv, R, group] of padded sequences as [n_rows, nq]."""
    seq, i = _row_index(s)
    return x.permute(0, 2, 1, 3).reshape(x.shape[0], x.shape[2], -1)[seq, i]


def _keys(s, c):
    """The slots of every sequence, [B, nkv, K, hd]."""
    x = c[s["layer"]][s["table"].long().clamp(min=0)]
    return x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], s["nkv"], -1, s["hd"]).float()


def _scores(s):
    """Scores of all rows of padded sequences, [B, nkv, R, group, K], minus
    infinity where a row does not see a slot."""
    nq, nkv, hd, group = s["nq"], s["nkv"], s["hd"], s["nq"] // s["nkv"]
    seq, i = _row_index(s)
    B, R, K = s["lens"].shape[0], s["max_rows"], s["table"].shape[1] * s["page"]
    q = torch.zeros((B, R, nq, hd), device=DEV)
    q[seq, i] = s["q"].float()
    q = q.view(B, R, nkv, group, hd).permute(0, 2, 1, 3, 4).reshape(B, nkv, R * group, hd)
    p = torch.matmul(q, _keys(s, s["k"]).transpose(-1, -2)).mul_(hd ** -0.5).view(B, nkv, R, group, K)
    if s["cap"] > 0:
        p = p.div_(s["cap"]).tanh_().mul_(s["cap"])
    slot = torch.arange(K, device=DEV)[None, :]
    j = slot - s["lens"][:, None].long()  # draft index, negative: the cache
    rows = s["start"][1:] - s["start"][:-1]
    depth = torch.arange(R, device=DEV).expand(B, R).clone()
    if s["depth"] is not None:
        depth[seq, i] = s["depth"].long()
    place = s["lens"][:, None].long() + depth
    key = torch.where(j < 0, slot, place.gather(1, j.clamp(0, R - 1)))
    gap = place[:, :, None] - key[:, None, :]  # [B, R, K]
    if s["slopes"] is not None:
        p = p - s["slopes"].view(nkv, 1, group, 1) * gap.abs()[:, None, :, None, :]
    see = (j < rows[:, None])[:, None, :]
    if s["mask"] is not None:
        bits = torch.zeros((B, R, s["mask"].shape[1]), dtype=torch.int64, device=DEV)
        bits[seq, i] = s["mask"].long() & 0xFFFFFFFF
        most = 32 * s["mask"].shape[1]
        bit = (bits.gather(2, (j.clamp(0, most - 1) // 32)[:, None, :].expand(B, R, K)) >> (j.clamp(min=0) % 32)[:, None]) & 1
        see = see & ((j[:, None, :] < 0) | ((bit == 1) & (j[:, None, :] < most)))
    elif s["span"] is None:
        see = see & (j[:, None, :] <= torch.arange(R, device=DEV)[None, :, None])
    if s["span"] is not None:
        span = torch.zeros((B, R, 2), dtype=torch.int64, device=DEV)
        span[seq, i] = s["span"].long()
        see = see & (slot[:, None] >= span[:, :, :1]) & (slot[:, None] < span[:, :, 1:])
    if s["window"]:
        see = see & (gap < s["window"])
    return p.masked_fill_(~see[:, None, :, None, :], -math.inf)


def _likeliest(p):
    """The largest value's index (the lowest, where several are)."""
    return (p < p.amax(-1, keepdim=True)).int().cummin(-1).values.sum(-1)


def _log_sum(p):
    top = p.amax(-1, keepdim=True).clamp(min=-3e38)
    return ((p - top).exp_().sum(-1).log() + top[..., 0])


def _plain_attend(s):
    nq, nkv, hd, group = s["nq"], s["nkv"], s["hd"], s["nq"] // s["nkv"]
    seq, i = _row_index(s)
    p = _scores(s)
    B, R, K = p.shape[0], p.shape[2], p.shape[4]
    top = p.amax(-1, keepdim=True).clamp(min=-3e38)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, nkv, R * group, K), _keys(s, s["v"])).view(B, nkv, R, group, hd)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    s["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(B, R, nq, hd)[seq, i])
    s["lse"].copy_(_by_row(s, total.log()[..., 0] + top[..., 0]))
    return s["out"], s["lse"]


def _plain_weigh(s):
    nkv, group = s["nkv"], s["nq"] // s["nkv"]
    seq, i = _row_index(s)
    p = _scores(s)
    B, R, K = p.shape[0], p.shape[2], p.shape[4]
    lse = torch.full((B, R, nkv * group), math.inf, device=DEV)
    lse[seq, i] = s["lse"].masked_fill(s["lse"].isinf(), math.inf)  # (a row that sees nothing gives nothing)
    lse = lse.view(B, R, nkv, group).permute(0, 2, 1, 3)
    got = p.sub_(lse[..., None]).exp_().sum((2, 3))  # [B, nkv, K]
    j = torch.arange(K, device=DEV)[None, :] - s["lens"][:, None].long()
    rows = (s["start"][1:] - s["start"][:-1])[:, None]
    # committed slots add up; this step's drafts begin anew (those of a tree at nothing)
    m = s["mass"][s["layer"]]
    new = torch.zeros_like(got) if s["mask"] is not None else got
    m.copy_(torch.where((j < 0)[:, None], m + got, torch.where((j < rows)[:, None], new, m)))
    return s["mass"]


def _plain_evict(s):
    _restore(s)
    seqs, page = s["seqs"].long(), s["page"]
    lens, keep = s["lens"][seqs].long(), s["keep"].long()
    mass = s["mass"][:, seqs]
    n, K = seqs.shape[0], mass.shape[-1]
    slot = torch.arange(K, device=DEV)[None, :]
    score = mass.double().sum((0, 2))
    safe = (slot < s["first"]) | (slot >= lens[:, None] - s["last"])
    score = torch.where(safe, math.inf, score).masked_fill(slot >= lens[:, None], -1.0)
    rank = torch.empty_like(slot.expand(n, K))
    rank.scatter_(1, torch.argsort(score, dim=1, descending=True, stable=True), slot.expand(n, K).contiguous())
    stay = torch.minimum(lens, keep)
    kept = (rank < stay[:, None]) & (slot < lens[:, None])
    A = s["most"]
    frm = torch.argsort((~kept).int(), dim=1, stable=True)[:, :A]  # kept slots, ascending
    live = torch.arange(A, device=DEV)[None, :] < stay[:, None]
    s["kept"][:, :A] = torch.where(live, frm.int(), s["kept"][:, :A])
    # (places behind a sequence's last kept slot write its first one again)
    to = slot[:, :A].expand(n, A)
    t = s["table"][seqs].long().clamp(min=0)
    pf, pt = t.gather(1, frm // page), t.gather(1, to // page)
    pt, at = torch.where(live, pt, pt[:, :1]), torch.where(live, to % page, 0)
    pf, af = torch.where(live, pf, pf[:, :1]), torch.where(live, frm % page, frm[:, :1] % page)
    for c in (s["k"], s["v"]):
        c[:, pt, :, at] = c[:, pf, :, af]
    idx = frm[None, :, None].expand(mass.shape[0], n, mass.shape[2], A)
    out = torch.zeros_like(mass)
    out[..., :A] = torch.where(live[None, :, None], mass.gather(3, idx), 0)
    s["mass_out"][:, seqs] = out
    cut = lens > keep
    held = torch.where(cut, (stay + page - 1) // page, s["held"][seqs].long())
    col = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    gone = (col >= held[:, None]) & (s["table"][seqs] >= 0)
    s["refs"].scatter_add_(0, t.reshape(-1), -gone.int().reshape(-1))
    s["table"][seqs] = torch.where(col < held[:, None], s["table"][seqs], -1)
    s["held"][seqs] = held.int()
    s["lens"][seqs] = stay.int()
    return s["k"], s["v"], s["mass_out"], s["kept"], s["table"], s["lens"], s["held"], s["refs"]


def _plain_verify(s):
    E, n = s["entries"], s["n_rows"]
    start = s["start"].long()
    first, rows = start[:-1], (start[1:] - start[:-1])
    at = torch.zeros_like(first)  # the node that the walk is at
    count = torch.ones_like(first)
    kept = s["kept"].fill_(-1)
    kept[first] = 0
    if s["greedy"]:
        best = _likeliest(s["probs"])
    else:
        rest = s["probs"][first].double()  # what is left of the node's target
        z = torch.ones(E, dtype=torch.float64, device=DEV)
        u = s["uniform"].double()
    for i in range(1, s["max_rows"]):
        row = (first + i).clamp(max=n - 1)
        par = s["parent"][row].long() if s["parent"] is not None else torch.full_like(at, i - 1)
        mine = (i < rows) & (par == at)
        x = s["tokens"][row].long()
        if s["greedy"]:
            yes = mine & (best[first + at] == x)
        else:
            left = rest.gather(1, x[:, None])[:, 0]
            if s["drafted"] is not None:
                d = s["drafted"][first + at].double()
                yes = mine & (u[row] * d.gather(1, x[:, None])[:, 0] * z < left)
                less = (rest - z[:, None] * d).clamp(min=0)
                zl = less.sum(-1)
            else:
                yes = mine & (u[row] * z < left)
                less = rest.scatter(1, x[:, None], 0.0)
                zl = z - left
            no = mine & ~yes
            rest = torch.where(no[:, None], less, torch.where(yes[:, None], s["probs"][row].double(), rest))
            z = torch.where(no, zl, torch.where(yes, torch.ones_like(z), z))
        at = torch.where(yes, i, at)
        to = torch.where(yes, first + count, first)
        kept[to] = torch.where(yes, torch.full_like(kept[to], i), kept[first])
        count = count + yes
    s["n_kept"].copy_(count)
    if s["greedy"]:
        s["next"].copy_(best[first + at])
    else:
        # nothing left of a target: all of it
        rest = torch.where((rest.sum(-1) > 0)[:, None], rest, s["probs"][first + at].double())
        cum = rest.cumsum(-1)
        s["next"].copy_((cum <= u[first][:, None] * cum[:, -1:]).sum(-1))
    return s["kept"], s["n_kept"], s["next"]


_own = {"attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict, "verify": _own_verify}
_plain = {"attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict, "verify": _plain_verify}


# --------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "weigh": _exact_weigh, "evict": _exact_evict, "verify": _exact_verify}[s["kind"]](s)


def _exact_rows(s):
    """For every sequence: its number, first row, rows, keys and values in 64
    bits, and the scores of each KV head."""
    nkv, hd, group = s["nkv"], s["hd"], s["nq"] // s["nkv"]
    start, lens = s["start"].tolist(), s["lens"].tolist()
    for b, n in enumerate(lens):
        r0, r = start[b], start[b + 1] - start[b]
        slot = torch.arange(n + r, device=DEV)
        page = s["table"][b][torch.div(slot, s["page"], rounding_mode="floor")].long()
        k = s["k"][s["layer"], page, :, slot % s["page"]].double()  # [n + r, nkv, hd]
        v = s["v"][s["layer"], page, :, slot % s["page"]].double()
        q = s["q"][r0:r0 + r].double().view(r, nkv, group, hd)
        depth = torch.arange(r, device=DEV) if s["depth"] is None else s["depth"][r0:r0 + r].long()
        key = torch.cat([slot[:n], n + depth])
        gap = (n + depth)[:, None] - key[None, :]
        hide = torch.zeros((r, n + r), dtype=torch.bool, device=DEV)
        if s["mask"] is not None:
            for j in range(r):
                hide[:, n + j] = (s["mask"][r0:r0 + r, j // 32] >> (j % 32)) & 1 == 0
        elif s["span"] is None:
            hide[:, n:] = torch.ones((r, r), dtype=torch.bool, device=DEV).triu(1)
        if s["span"] is not None:
            lo, hi = s["span"][r0:r0 + r].long().unbind(1)
            hide |= (slot < lo[:, None]) | (slot >= hi[:, None])
        if s["window"]:
            hide |= gap >= s["window"]

        def score(h):
            x = torch.matmul(q[:, h].reshape(r * group, hd), k[:, h].t().contiguous()) / math.sqrt(hd)
            if s["cap"]:
                x = s["cap"] * torch.tanh(x / s["cap"])
            x = x.view(r, group, n + r)
            if s["slopes"] is not None:
                x = x - s["slopes"][h * group:(h + 1) * group].double()[:, None] * gap.abs()[:, None].double()
            return x.masked_fill(hide[:, None], -math.inf)

        yield b, n, r0, r, v, score


def _exact_attend(s):
    nkv, hd, group = s["nkv"], s["hd"], s["nq"] // s["nkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for b, n, r0, r, v, score in _exact_rows(s):
        for h in range(nkv):
            x = score(h)
            p = torch.softmax(x, -1).nan_to_num(0.0).view(r * group, n + r)
            out[r0:r0 + r, h * group:(h + 1) * group] = torch.matmul(p, v[:, h].contiguous()).view(r, group, hd)
            lse[r0:r0 + r, h * group:(h + 1) * group] = torch.logsumexp(x, -1)
    return out, lse


def _exact_weigh(s):
    nkv, group = s["nkv"], s["nq"] // s["nkv"]
    mass = s["mass"].double()
    for b, n, r0, r, v, score in _exact_rows(s):
        for h in range(nkv):
            lse = s["lse"][r0:r0 + r, h * group:(h + 1) * group].double()
            got = torch.exp(score(h) - lse[..., None]).masked_fill(lse.isinf()[..., None], 0.0).sum((0, 1))
            row = mass[s["layer"], b, h]
            row[:n] += got[:n]
            row[n:n + r] = 0.0 if s["mask"] is not None else got[n:]
    return mass


def _exact_evict(s):
    page = s["page"]
    k, v, out = s["k"].clone(), s["v"].clone(), torch.zeros_like(s["mass"], dtype=torch.float64)
    kept, table, lens, held, refs = (s[x].tolist() for x in ("kept", "table", "lens", "held", "refs"))
    weight = s["mass"].double().sum((0, 2)).tolist()
    for b, most in zip(s["seqs"].tolist(), s["keep"].tolist()):
        n = lens[b]
        if n > most:
            safe = [i for i in range(n) if i < s["first"] or i >= n - s["last"]]
            rest = sorted((i for i in range(s["first"], n - s["last"])), key=lambda i: (-weight[b][i], i))
            stay = sorted(safe + rest[:most - len(safe)])
        else:
            stay = list(range(n))
        kept[b][:len(stay)] = stay
        frm = torch.tensor(stay, device=DEV)
        to = torch.arange(len(stay), device=DEV)
        t = s["table"][b].long()
        for c, old in ((k, s["k"]), (v, s["v"])):
            c[:, t[to // page], :, to % page] = old[:, t[frm // page], :, frm % page]
        out[:, b, :, :len(stay)] = s["mass"][:, b][..., frm].double()
        if n > most:
            lens[b] = most
            while (held[b] - 1) * page >= most:
                held[b] -= 1
                refs[table[b][held[b]]] -= 1
                table[b][held[b]] = -1
    return (k.double(), v.double(), out, *[_i32(x) for x in (kept, table, lens, held, refs)])


def _exact_verify(s):
    start, tokens = s["start"].tolist(), s["tokens"].tolist()
    parent = s["parent"].tolist() if s["parent"] is not None else None
    uniform = s["uniform"].tolist() if s["uniform"] is not None else None
    kept, counts, after = [-1] * s["n_rows"], [], []
    for b in range(s["entries"]):
        r0, r = start[b], start[b + 1] - start[b]
        node, path = 0, [0]
        while True:
            p = s["probs"][r0 + node].double()
            kids = [i for i in range(1, r) if (parent[r0 + i] if parent else i - 1) == node]
            if uniform is None:
                token = int((p == p.max()).nonzero()[0])
                step = next((i for i in kids if tokens[r0 + i] == token), None)
            else:
                step, total = None, 1.0
                if s["drafted"] is not None:
                    d = s["drafted"][r0 + node].double()
                    sub = 0.0  # the target is left with what passes this many of the draft's
                    for i in kids:
                        x = tokens[r0 + i]
                        if uniform[r0 + i] * float(d[x]) * total < max(0.0, float(p[x]) - sub * float(d[x])):
                            step = i
                            break
                        sub += total
                        total = float(torch.relu(p - sub * d).sum())
                    left = torch.relu(p - sub * d)
                else:
                    left = p.clone()
                    for i in kids:
                        x = tokens[r0 + i]
                        if uniform[r0 + i] * total < float(left[x]):
                            step = i
                            break
                        total -= float(left[x])
                        left[x] = 0.0
                if step is None:
                    if not float(left.sum()) > 0:
                        left = p
                    cum = torch.cumsum(left, 0)
                    token = int(torch.searchsorted(cum, cum[-1:] * uniform[r0], right=True)[0])
            if step is None:
                break
            node = step
            path.append(step)
        kept[r0:r0 + len(path)] = path
        counts.append(len(path))
        after.append(token)
    return _i32(kept), _i32(counts), _i32(after)
