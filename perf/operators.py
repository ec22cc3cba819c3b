"""Measured cases of the paged cache's operators: what a language model that
answers token by token, or by drafted trees of tokens, runs around its GEMMs.

Kinds of case:

* ``store``   ``vla_qk_norm_rope``: per-head RMSNorm of queries and keys,
              rotation, and the store of K and V into the cache's pages;
* ``attend``  ``vla_tree_attention``: queries of drafted tokens (one token, a
              tree, or a causal chunk) over a sequence's pages;
* ``fork``    ``vla_pages_release`` of the last step's children, then
              ``vla_pages_fork`` into new ones (full pages shared, the last one
              copied in every layer) and ``vla_pages_reserve`` of room for
              their drafts;
* ``commit``  ``vla_pages_commit``: the accepted drafts' K and V move together
              in every layer.

The plain forms compute in 32 bits with elementary torch operations and round
once at the end. Sequence lengths, row counts and trees come from the case
(its ``mix``), so that the work of a case is known; values, the order of the
pages in the pool and the accepted drafts come from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-6
ROPE_BASE = 10000.0


# --------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------

def listed():
    return [
        # one token of each of eight robots: the smallest call, all latency
        # (head layout of the PaliGemma-shaped LM)
        dict(name="store_decode8", kind="store", dtype="bf16", seqs=8, len_lo=305, len_hi=420, rows_lo=1, rows_hi=1,
             nq=8, nkv=1, hd=256, rot=256, page=32, layers=2, tree=0, mix=1),
        # two long prompts entering the cache (grouped heads): bandwidth
        dict(name="store_prompts", kind="store", dtype="bf16", seqs=2, len_lo=1, len_hi=900, rows_lo=7900, rows_hi=8300,
             nq=32, nkv=8, hd=128, rot=128, page=64, layers=1, tree=0, mix=2),
        # ragged trees in fp32, part of each head rotated
        dict(name="store_f32_trees", kind="store", dtype="f32", seqs=5, len_lo=30, len_hi=700, rows_lo=17, rows_hi=61,
             nq=6, nkv=2, hd=96, rot=64, page=16, layers=2, tree=6, mix=3),
        # one token of each of eight robots over its prefix
        dict(name="attend_decode8", kind="attend", dtype="bf16", seqs=8, len_lo=305, len_hi=420, rows_lo=1, rows_hi=1,
             nq=8, nkv=1, hd=256, page=32, tree=0, mix=4),
        # drafted trees of 40 to 64 tokens of eight robots with some history
        dict(name="attend_tree8", kind="attend", dtype="bf16", seqs=8, len_lo=305, len_hi=4000, rows_lo=40, rows_hi=64,
             nq=8, nkv=1, hd=256, page=32, tree=8, mix=5),
        # single tokens over long, uneven caches: the cache's bandwidth
        dict(name="attend_long", kind="attend", dtype="bf16", seqs=16, len_lo=8000, len_hi=65000, rows_lo=1, rows_hi=1,
             nq=32, nkv=8, hd=128, page=64, tree=0, mix=6),
        # chunks of two long prompts, causal: matrix products
        dict(name="attend_chunk", kind="attend", dtype="bf16", seqs=2, len_lo=2000, len_hi=6000, rows_lo=2000,
             rows_hi=2048, nq=32, nkv=8, hd=128, page=64, tree=0, mix=7),
        # ragged trees in fp32, three queries to a key head, odd head dim
        dict(name="attend_f32_trees", kind="attend", dtype="f32", seqs=5, len_lo=30, len_hi=700, rows_lo=17, rows_hi=61,
             nq=6, nkv=2, hd=96, page=16, tree=6, mix=8),
        # eight answers sampled from one prompt
        dict(name="fork_answers8", kind="fork", dtype="bf16", parents=1, seqs=8, len_lo=305, len_hi=420, rows_lo=8,
             rows_hi=8, nkv=1, hd=256, page=32, layers=18, mix=9),
        # four branches of each of sixteen sequences, grouped heads
        dict(name="fork_beams64", kind="fork", dtype="bf16", parents=16, seqs=64, len_lo=300, len_hi=3000, rows_lo=8,
             rows_hi=64, nkv=8, hd=128, page=64, layers=28, mix=10),
        # eight robots' accepted drafts
        dict(name="commit8", kind="commit", dtype="bf16", seqs=8, len_lo=305, len_hi=420, rows_lo=40, rows_hi=64,
             nkv=1, hd=256, page=32, layers=18, accept_hi=6, mix=11),
        # sixty-four sequences' accepted drafts, grouped heads
        dict(name="commit64", kind="commit", dtype="bf16", seqs=64, len_lo=300, len_hi=3000, rows_lo=32, rows_hi=64,
             nkv=8, hd=128, page=64, layers=28, accept_hi=12, mix=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["store", "attend", "attend", "fork", "commit"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    esz = 2 if dtype == "bf16" else 4
    hd = rng.choice([32, 64, 96, 128] if dtype == "f32" else [32, 64, 96, 128, 160, 256])
    nkv = rng.choice([1, 1, 2, 4, 8])
    nq = nkv * rng.choice([1, 2, 3, 4, 5, 8])
    page = rng.choice([16, 32, 64, 128, 256])
    c = dict(kind=kind, dtype=dtype, hd=hd, nkv=nkv, page=page, mix=rng.randrange(1 << 20))
    if kind in ("store", "attend"):
        form = rng.choice(["one", "tree", "chunk"])
        seqs = _log_int(rng, 1, 48)
        if form == "one":
            lo = hi = 1
        elif form == "tree":
            lo, hi = 2, _log_int(rng, 3, 90)
        else:
            hi = _log_int(rng, 32, 4000)
            lo = rng.randint(1, hi)
        c.update(nq=nq, seqs=seqs, rows_lo=lo, rows_hi=hi, tree=rng.randint(1, 12) if form == "tree" else 0)
        ctx = _log_int(rng, 8, 60000)
        if kind == "store":
            c.update(len_lo=1, len_hi=min(ctx, 20000), layers=rng.choice([1, 2, 3]), rot=hd // 32 * rng.choice([16, 32]))
            # at most the values of 8,000 rows of 48 heads of 128
            c["seqs"] = max(1, min(seqs, int(8000 * 48 * 128 / (hi * (nq + 2 * nkv) * hd))))
            c["rows_hi"] = min(hi, int(8000 * 48 * 128 / ((nq + 2 * nkv) * hd)))
        else:
            c.update(len_lo=max(1, ctx // rng.choice([1, 2, 8, 30])), len_hi=ctx)
            # at most 512 MiB of K, 2^30 scores and 2^36 products (fp32: half as many)
            for _ in range(40):
                keys = c["seqs"] * (c["len_hi"] + c["rows_hi"])
                if keys * nkv * hd * esz <= 2 ** 29 and keys * c["rows_hi"] * nq * max(hd, 64) * esz <= 2 ** 37 \
                        and keys * c["rows_hi"] * nq <= 2 ** 30:
                    break
                if c["seqs"] > 1:
                    c["seqs"] = (c["seqs"] + 1) // 2
                else:
                    c["len_hi"] = max(8, c["len_hi"] * 2 // 3)
                    c["rows_hi"] = max(1, c["rows_hi"] * 2 // 3)
            c["len_lo"] = min(c["len_lo"], c["len_hi"])
        c["rows_lo"] = min(c["rows_lo"], c["rows_hi"])
    else:
        c.update(seqs=_log_int(rng, 1, 64), len_lo=1, len_hi=_log_int(rng, 20, 3000), layers=rng.randint(1, 28),
                 rows_lo=1, rows_hi=_log_int(rng, 2, 64))
        if kind == "fork":
            c["parents"] = rng.randint(1, min(16, c["seqs"]))
        else:
            c["accept_hi"] = rng.randint(1, 12)
        # at most 2^30 values of K in the pool
        keys = (c["seqs"] if kind == "commit" else c["parents"]) * (c["len_hi"] + 64) + c["seqs"] * (2 * page + 64)
        c["layers"] = max(1, min(c["layers"], int(2 ** 30 / (keys * nkv * hd))))
    return c


# --------------------------------------------------------------------------
# Shapes of a case
# --------------------------------------------------------------------------

def _layout(case):
    """Lengths and row counts of the case's sequences, and the parents of the
    drafted tokens (-1: a child of the cache's last token)."""
    rng = random.Random(case["mix"])
    n = case["parents"] if case["kind"] == "fork" else case["seqs"]
    lens = [_log_int(rng, case["len_lo"], case["len_hi"]) for _ in range(n)]
    rows = [rng.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["seqs"])]
    parents = None
    if case.get("tree"):
        # levels of about `tree` tokens: a token's parent is one of the
        # `tree` tokens before its level, or the cache's last token
        w = case["tree"]
        parents = [[-1 if j < w else rng.randint(max(0, j - 2 * w + 1), max(0, j - w)) for j in range(r)] for r in rows]
    return lens, rows, parents


def _pages(n, page):
    return (n + page - 1) // page


def _depths(par):
    d = []
    for j, p in enumerate(par):
        d.append(0 if p < 0 else d[p] + 1)
    return d


def work(case):
    lens, rows, parents = _layout(case)
    esz = 2 if case["dtype"] == "bf16" else 4
    hd, nkv = case["hd"], case["nkv"]
    if case["kind"] == "store":
        heads = case["nq"] + 2 * nkv
        if parents:
            pos = {n + d for n, p in zip(lens, parents) for d in _depths(p)}
        else:
            pos = {n + i for n, r in zip(lens, rows) for i in range(r)}
        values = sum(rows) * heads * hd
        turned = sum(rows) * (case["nq"] + nkv) * hd
        return {"bytes": 2 * values * esz + len(pos) * case["rot"] * 4 + 8 * hd + 8 * sum(rows),
                "flops": turned * 4 + turned * case["rot"] / hd * 3}
    if case["kind"] == "attend":
        q = sum(rows) * case["nq"] * hd
        keys = sum(n + r for n, r in zip(lens, rows))
        if parents:
            pairs = sum(n * r + sum(d + 1 for d in _depths(p)) for n, r, p in zip(lens, rows, parents))
        else:
            pairs = sum(n * r + r * (r + 1) // 2 for n, r in zip(lens, rows))
        bits = sum(rows) * 4 * ((max(rows) + 31) // 32) if parents else 0
        return {"bytes": 2 * keys * nkv * hd * esz + 2 * q * esz + bits, "flops": 4.0 * pairs * case["nq"] * hd}
    row = 2 * case["layers"] * nkv * hd * esz  # K and V of one token
    if case["kind"] == "fork":
        par = _families(case)
        part = [lens[p] % case["page"] for p in par]
        reads = sum(n % case["page"] for n in lens)
        table = sum(_pages(lens[p] + r, case["page"]) for p, r in zip(par, rows))
        return {"bytes": (reads + sum(part)) * row + 12 * table, "flops": 0}
    # all but the first accepted draft move
    moved = sum(a - 1 for a in _accepts(case, rows))
    return {"bytes": 2 * moved * row + 8 * case["seqs"], "flops": 0}


def _families(case):
    """The parent of each child."""
    return [i * case["parents"] // case["seqs"] for i in range(case["seqs"])]


def _accepts(case, rows):
    rng = random.Random(case["mix"] + 1)
    return [rng.randint(1, max(1, min(case["accept_hi"], (r + 1) // 2))) for r in rows]


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    rng = random.Random(seed * 2 + 1)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    T = _type(case)
    lens, rows, parents = _layout(case)
    page, kind, nkv, hd = case["page"], case["kind"], case["nkv"], case["hd"]
    layers = case.get("layers", 1)

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)

    # the pool: sequences' pages in random order, as after some time of use
    if kind == "fork":
        slots = len(lens) + case["seqs"]
        need = [_pages(n, page) for n in lens]
        spare = sum(_pages(max(lens) % page + r + page, page) for r in rows) + 8
        wide = max(_pages(n + max(rows), page) for n in lens) + 1
    else:
        slots = len(lens)
        need = [_pages(n + r, page) for n, r in zip(lens, rows)]
        spare = 8
        wide = max(need) + 1
    n_pages = sum(need) + spare
    order = list(range(n_pages))
    rng.shuffle(order)
    table = [[-1] * wide for _ in range(slots)]
    refs = [0] * n_pages
    at = 0
    for s, n in enumerate(need):
        table[s][:n] = order[at:at + n]
        for p in order[at:at + n]:
            refs[p] = 1
        at += n
    shape = (layers, n_pages, nkv, page, hd)
    s = dict(case=case, kind=kind, page=page, hd=hd, nkv=nkv, lens0=lens, layer=layers - 1,
             k=torch.randn(shape, dtype=T, device=DEV, generator=gen),
             v=torch.randn(shape, dtype=T, device=DEV, generator=gen),
             table=i32(table), lens=i32(lens + [0] * (slots - len(lens))),
             held=i32(need + [0] * (slots - len(lens))), refs=i32(refs), status=i32([0]))
    start = [0]
    for r in rows:
        start.append(start[-1] + r)
    s["start"], s["n_rows"], s["max_rows"] = i32(start), start[-1], max(rows)

    if kind in ("store", "attend"):
        s["nq"] = case["nq"]
        if parents:
            s["pos"] = i32([n + d for n, p in zip(lens, parents) for d in _depths(p)])
            words = (max(rows) + 31) // 32
            bits = []
            for p in parents:
                seen = []
                for j, q in enumerate(p):
                    seen.append((1 << j) | (seen[q] if q >= 0 else 0))
                bits += [[(b >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for b in seen]
            s["mask"] = torch.tensor(bits, dtype=torch.int64, device=DEV).to(torch.int32)  # the low 32 bits
        else:
            s["pos"], s["mask"] = None, None
    if kind == "store":
        heads = case["nq"] + 2 * nkv
        # the QKV projection's rows: heads of different magnitude
        s["qkv"] = (torch.randn((s["n_rows"], heads, hd), device=DEV, generator=gen)
                    * (0.25 + 2 * torch.rand((1, heads, 1), device=DEV, generator=gen))).to(T)
        s["q_out"] = torch.empty((s["n_rows"], case["nq"], hd), dtype=T, device=DEV)
        s["q_gain"] = 1 + 0.1 * torch.randn(hd, device=DEV, generator=gen)
        s["k_gain"] = 1 + 0.1 * torch.randn(hd, device=DEV, generator=gen)
        half = case["rot"] // 2
        freq = ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        angle = torch.arange(max(lens) + max(rows) + 1, dtype=torch.float64, device=DEV)[:, None] * freq
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    if kind == "attend":
        s["q"] = torch.randn((s["n_rows"], case["nq"], hd), device=DEV, generator=gen).to(T)
        s["out"] = torch.empty_like(s["q"])
    if kind == "fork":
        par = _families(case)
        s["src"], s["dst"] = i32(par), i32([len(lens) + i for i in range(case["seqs"])])
        s["made"] = i32([0] * case["seqs"])
    if kind == "commit":
        # accepted paths: the first draft, which stays, then drafts from
        # behind the accepted count (levels of a tree are wider than its path
        # is long), so a pass can be repeated
        acc, kept = _accepts(case, rows), []
        for a, r in zip(acc, rows):
            kept += [0] + sorted(rng.sample(range(a, r), a - 1)) + [-1] * (r - a)
        s["kept"], s["n_kept"], s["max_kept"] = i32(kept), i32(acc), max(acc)
        s["lens_before"] = s["lens"].clone()
    if own:
        import paper_2609_22335_amd as V
        s["V"] = V
        s["pages"] = V.make_pages(s["k"], s["v"], s["table"], s["lens"], s["held"], s["refs"], s["status"])
        if kind == "fork":
            s["rows"] = V.make_rows(s["start"], s["n_rows"], s["dst"])
        else:
            s["rows"] = V.make_rows(s["start"], s["n_rows"])
        if kind == "store":
            s["rope"] = V.make_rope_norm(s["cos"], s["sin"], s["q_gain"], s["k_gain"], eps=EPS)
        if kind == "attend":
            n = V.vla_tree_attention_scratch(s["pages"], s["rows"], s["nq"])
            s["scratch"] = torch.zeros(n, dtype=torch.uint8, device=DEV)
    return s


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _own_store(s):
    nq, nkv, x = s["nq"], s["nkv"], s["qkv"]
    s["V"].vla_qk_norm_rope(s["pages"], s["layer"], s["rows"], s["rope"], x[:, :nq], x[:, nq:nq + nkv],
                            x[:, nq + nkv:], s["q_out"], pos=s["pos"])
    return s["q_out"], s["k"], s["v"]


def _own_attend(s):
    s["V"].vla_tree_attention(s["pages"], s["layer"], s["rows"], s["q"], s["out"], s["scratch"], mask=s["mask"])
    return s["out"]


def _own_fork(s):
    V = s["V"]
    V.vla_pages_release(s["pages"], s["dst"])
    V.vla_pages_fork(s["pages"], s["src"], s["dst"], s["made"])
    V.vla_pages_reserve(s["pages"], s["rows"])
    return s["k"], s["v"], s["table"], s["lens"], s["held"], s["refs"], s["made"]


def _own_commit(s):
    s["lens"].copy_(s["lens_before"])
    s["V"].vla_pages_commit(s["pages"], s["rows"], s["kept"], s["n_kept"])
    return s["k"], s["v"], s["lens"]


def _row_index(s):
    """The sequence and the index in it of every row."""
    t = torch.arange(s["n_rows"], device=DEV)
    seq = torch.searchsorted(s["start"][1:].long(), t, right=True)
    return seq, t - s["start"][seq].long()


def _plain_store(s):
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    seq, i = _row_index(s)
    slot = s["lens"][seq].long() + i
    pos = slot if s["pos"] is None else s["pos"].long()
    x = s["qkv"].float()
    qk = x[:, :nq + nkv]
    gain = torch.cat([s["q_gain"].expand(nq, hd), s["k_gain"].expand(nkv, hd)])
    qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS) * gain
    half = s["cos"].shape[1]
    c, n = s["cos"][pos][:, None], s["sin"][pos][:, None]
    a, b = qk[..., :half], qk[..., half:2 * half]
    qk = torch.cat([a * c - b * n, b * c + a * n, qk[..., 2 * half:]], -1).to(s["qkv"].dtype)
    s["q_out"].copy_(qk[:, :nq])
    page, at = s["table"][seq, slot // s["page"]].long(), slot % s["page"]
    s["k"][s["layer"]][page, :, at] = qk[:, nq:]
    s["v"][s["layer"]][page, :, at] = s["qkv"][:, nq + nkv:]
    return s["q_out"], s["k"], s["v"]


def _plain_attend(s):
    nq, nkv, hd, group = s["nq"], s["nkv"], s["hd"], s["nq"] // s["nkv"]
    seq, i = _row_index(s)
    B, R = s["lens"].shape[0], s["max_rows"]
    idx = s["table"].long().clamp(min=0)
    K = idx.shape[1] * s["page"]

    def keys(c):  # [B, nkv, K, hd]
        return c[s["layer"]][idx].permute(0, 2, 1, 3, 4).reshape(B, nkv, K, hd).float()

    q = torch.zeros((B, R, nq, hd), device=DEV)
    q[seq, i] = s["q"].float()
    q = q.view(B, R, nkv, group, hd).permute(0, 2, 1, 3, 4).reshape(B, nkv, R * group, hd)
    p = torch.matmul(q, keys(s["k"]).transpose(-1, -2)) * hd ** -0.5
    key = torch.arange(K, device=DEV)[None, :] - s["lens"][:, None].long()  # draft index, negative: the cache
    if s["mask"] is None:
        see = key[:, None, :] <= torch.arange(R, device=DEV)[None, :, None]
    else:
        bits = torch.zeros((B, R, s["mask"].shape[1]), dtype=torch.int64, device=DEV)
        bits[seq, i] = s["mask"].long() & 0xFFFFFFFF
        most = 32 * s["mask"].shape[1]
        word = (key.clamp(0, most - 1) // 32)[:, None, :].expand(B, R, K)
        see = (bits.gather(2, word) >> (key.clamp(min=0) % 32)[:, None, :]) & 1
        see = (key[:, None, :] < 0) | ((see == 1) & (key[:, None, :] < most))
    p = p.view(B, nkv, R, group, K).masked_fill(~see[:, None, :, None, :], -math.inf)
    p = p - p.amax(-1, keepdim=True).clamp(min=-3e38)
    p = p.exp()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, nkv, R * group, K), keys(s["v"])).view(B, nkv, R, group, hd)
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    s["out"].copy_(o.permute(0, 2, 1, 3, 4).reshape(B, R, nq, hd)[seq, i])
    return s["out"]


def _give(s, seq, first, count, most):
    """Deals free pages, lowest first, out to the sequences in order: `count`
    of them at table columns `first` and on. `most` bounds a count."""
    t, refs = s["table"], s["refs"]
    order = torch.argsort((refs != 0).int(), stable=True)
    col = torch.arange(most, device=DEV)[None, :]
    want = col < count[:, None]
    rank = (torch.cumsum(count, 0) - count)[:, None] + col
    page = order[rank.clamp(max=order.shape[0] - 1)]
    # columns past a sequence's count write the table's own value back
    at = (first[:, None] + col).clamp(max=t.shape[1] - 1)
    flat = torch.where(want, seq[:, None] * t.shape[1] + at, t.numel())
    both = torch.cat([t.reshape(-1), t.new_zeros(1)])
    both.scatter_(0, flat.reshape(-1), page.int().reshape(-1))
    t.copy_(both[:-1].view_as(t))
    refs.scatter_add_(0, page.reshape(-1), want.int().reshape(-1))
    return page[:, 0]


def _plain_fork(s):
    page, t, refs = s["page"], s["table"], s["refs"]
    src, dst = s["src"].long(), s["dst"].long()
    col = torch.arange(t.shape[1], device=DEV)[None, :]
    # release
    mine = col < s["held"][dst][:, None]
    refs.scatter_add_(0, t[dst].clamp(min=0).long().reshape(-1), -mine.int().reshape(-1))
    t[dst] = -1
    s["lens"][dst] = 0
    s["held"][dst] = 0
    # fork: share the full pages, copy the part of the last one
    n = s["lens"][src]
    full, part = n // page, n % page
    shared = torch.where(col < full[:, None], t[src], -1)
    refs.scatter_add_(0, shared.clamp(min=0).long().reshape(-1), (shared >= 0).int().reshape(-1))
    t[dst] = shared
    new = _give(s, dst, full.long(), (part > 0).long(), 1)
    last = t[src, full.long().clamp(max=t.shape[1] - 1)].clamp(min=0).long()
    last = torch.where(part > 0, last, t[src, 0].long())
    new = torch.where(part > 0, new, last)
    copied = (torch.arange(page, device=DEV)[None, :] < part[:, None])[None, :, None, :, None]
    for c in (s["k"], s["v"]):
        c[:, new] = torch.where(copied, c[:, last], c[:, new])
    s["lens"][dst] = n
    s["held"][dst] = (n + page - 1) // page
    s["made"].fill_(1)
    # reserve
    rows = s["start"][1:] - s["start"][:-1]
    held = s["held"][dst]
    need = ((n + rows + page - 1) // page - held).clamp(min=0)
    _give(s, dst, held.long(), need.long(), (s["max_rows"] + page - 1) // page + 1)
    s["held"][dst] = held + need
    return s["k"], s["v"], s["table"], s["lens"], s["held"], s["refs"], s["made"]


def _plain_commit(s):
    page = s["page"]
    s["lens"].copy_(s["lens_before"])
    B, A = s["lens"].shape[0], s["max_kept"]
    j = torch.arange(A, device=DEV)[None, :]
    moved = j < s["n_kept"][:, None]
    row = (s["start"][:-1, None] + j).clamp(max=s["n_rows"] - 1).long()
    frm = s["lens"][:, None] + torch.where(moved, s["kept"][row], j)
    to = s["lens"][:, None] + j
    # a path is never longer than its tree, so `to` has a page where it counts;
    # other places write their own value back
    seq = torch.arange(B, device=DEV)[:, None]
    most = s["table"].shape[1] * page - 1
    frm, to = frm.clamp(max=most).long(), to.clamp(max=most).long()
    pf, pt = s["table"][seq, frm // page].long(), s["table"][seq, to // page].long()
    pt = torch.where(moved, pt, pt[:, :1])
    to = torch.where(moved, to % page, (to % page)[:, :1])
    pf = torch.where(moved, pf, pf[:, :1])
    frm = torch.where(moved, frm % page, (frm % page)[:, :1])
    for c in (s["k"], s["v"]):
        c[:, pt, :, to] = c[:, pf, :, frm]
    s["lens"].add_(s["n_kept"])
    return s["k"], s["v"], s["lens"]


_own = {"store": _own_store, "attend": _own_attend, "fork": _own_fork, "commit": _own_commit}
_plain = {"store": _plain_store, "attend": _plain_attend, "fork": _plain_fork, "commit": _plain_commit}


# --------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"store": _exact_store, "attend": _exact_attend, "fork": _exact_fork, "commit": _exact_commit}[s["kind"]](s)


def _of_sequences(s):
    """Host lists: (sequence, its committed length, its first row, its rows)."""
    start, lens = s["start"].tolist(), s["lens"].tolist()
    return [(b, lens[b], start[b], start[b + 1] - start[b]) for b in range(len(start) - 1)]


def _slots(s, b, first, count):
    """Page and place of `count` slots of sequence b, from `first` on."""
    slot = torch.arange(first, first + count, device=DEV)
    return s["table"][b][torch.div(slot, s["page"], rounding_mode="floor")].long(), slot % s["page"]


def _exact_store(s):
    nq, nkv = s["nq"], s["nkv"]
    half = s["cos"].shape[1]
    q_out = torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEV)
    k, v = s["k"].double(), s["v"].double()
    for b, n, r0, r in _of_sequences(s):
        x = s["qkv"][r0:r0 + r].double()
        pos = (torch.arange(n, n + r, device=DEV) if s["pos"] is None else s["pos"][r0:r0 + r]).long()
        turn = torch.complex(s["cos"][pos].double(), s["sin"][pos].double())[:, None]

        def norm_turn(h, gain):
            h = h / torch.sqrt(h.square().sum(-1, keepdim=True) / h.shape[-1] + EPS) * gain.double()
            z = torch.complex(h[..., :half].contiguous(), h[..., half:2 * half].contiguous()) * turn
            return torch.cat([z.real, z.imag, h[..., 2 * half:]], -1)

        q_out[r0:r0 + r] = norm_turn(x[:, :nq], s["q_gain"])
        page, at = _slots(s, b, n, r)
        k[s["layer"], page, :, at] = norm_turn(x[:, nq:nq + nkv], s["k_gain"])
        v[s["layer"], page, :, at] = x[:, nq + nkv:]
    return q_out, k, v


def _exact_attend(s):
    nq, nkv, hd, group = s["nq"], s["nkv"], s["hd"], s["nq"] // s["nkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    for b, n, r0, r in _of_sequences(s):
        page, at = _slots(s, b, 0, n + r)
        k = s["k"][s["layer"], page, :, at].double()  # [n + r, nkv, hd]
        v = s["v"][s["layer"], page, :, at].double()
        q = s["q"][r0:r0 + r].double().view(r, nkv, group, hd)
        hide = torch.zeros((r, n + r), dtype=torch.bool, device=DEV)
        if s["mask"] is None:
            hide[:, n:] = torch.ones((r, r), dtype=torch.bool, device=DEV).triu(1)
        else:
            for j in range(r):
                hide[:, n + j] = (s["mask"][r0:r0 + r, j // 32] >> (j % 32)) & 1 == 0
        for h in range(nkv):
            score = torch.matmul(q[:, h].reshape(r * group, hd), k[:, h].t().contiguous()) / math.sqrt(hd)
            score = score.view(r, group, n + r).masked_fill(hide[:, None], -math.inf)
            p = torch.softmax(score, -1).view(r * group, n + r)
            out[r0:r0 + r, h * group:(h + 1) * group] = torch.matmul(p, v[:, h].contiguous()).view(r, group, hd)
    return out


def _exact_fork(s):
    page = s["page"]
    k, v = s["k"].double(), s["v"].double()
    table, lens, held, refs = (s[x].tolist() for x in ("table", "lens", "held", "refs"))
    start, src, dst = (s[x].tolist() for x in ("start", "src", "dst"))

    def free_page():
        p = refs.index(0)
        refs[p] = 1
        return p

    for a, b in zip(src, dst):
        full, part = divmod(lens[a], page)
        for i in range(full):
            table[b][i] = table[a][i]
            refs[table[a][i]] += 1
    for a, b in zip(src, dst):
        full, part = divmod(lens[a], page)
        lens[b], held[b] = lens[a], full + (part > 0)
        if part:
            table[b][full] = free_page()
            for c in (k, v):
                c[:, table[b][full], :, :part] = c[:, table[a][full], :, :part]
    for i, b in enumerate(dst):
        while held[b] * page < lens[b] + start[i + 1] - start[i]:
            table[b][held[b]] = free_page()
            held[b] += 1
    whole = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, lens, held, refs)]
    return (k, v, *whole, torch.ones_like(s["made"]))


def _exact_commit(s):
    k, v = s["k"].double(), s["v"].double()
    kept, count = s["kept"].tolist(), s["n_kept"].tolist()
    for b, n, r0, r in _of_sequences(s):
        for j in range(count[b]):
            (pf,), (af,) = _slots(s, b, n + kept[r0 + j], 1)
            (pt,), (at,) = _slots(s, b, n + j, 1)
            for c in (k, v):
                c[:, pt, :, at] = c[:, pf, :, af]
    return k, v, s["lens"] + s["n_kept"]
