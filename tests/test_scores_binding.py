"""CPU checks of the arguments of attention with shaped scores, slot weights,
eviction and draft verification: the binding refuses wrong tensors before the
library is called, the C entry points refuse wrong descriptors, sizes and
overlaps before anything is launched, and the structures match the header."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2609_22335_amd as V
from test_paged_binding import BF, F, ROOT, Dev, cache, on_device_0, refused  # noqa: F401

U8 = torch.uint8
SLOTS = 5 * 16
MASS = (2, 3, 2, SLOTS)


def far(shape, dtype=F, at=1):
    """A tensor that nothing else overlaps."""
    return Dev(shape, dtype, ptr=0x10000 + at * (1 << 32))


def test_make_scores_refuses():
    p = cache()
    refused("slopes must be [nq]", V.make_scores, p, slopes=Dev((4, 1), F))
    refused("slopes must be float32", V.make_scores, p, slopes=Dev((4,), BF))
    refused("depth must be [n_rows]", V.make_scores, p, depth=Dev((7, 1)))
    refused("depth must be int32", V.make_scores, p, depth=Dev((7,), torch.int64))
    refused("span must be [n_rows, 2]", V.make_scores, p, span=Dev((7, 3)))
    refused("span must be [n_rows, 2]", V.make_scores, p, span=Dev((14,)))
    refused("span is on cuda:1", V.make_scores, p, span=Dev((7, 2), dev="cuda:1"))
    refused("window must be an integer", V.make_scores, p, window="8")
    refused("which 32 bits do not hold", V.make_scores, p, window=2 ** 31)
    s = V.make_scores(p)
    assert s.scale == 0.125 and s.cap == 0 and s.window == 0 and not s.slopes and not s.depth and not s.span


def test_score_attention_refuses():
    p, r = cache(), V.make_rows(Dev((3,)), 7)
    q, o, scr, s = far((7, 4, 64), BF), far((7, 4, 64), BF, 2), far((1 << 20,), U8, 3), V.make_scores(p)
    call = V.vla_score_attention
    refused("q must be [7, heads, 64]", call, p, 0, r, s, Dev((6, 4, 64), BF), o, scr)
    refused("out must be [7, 4, 64]", call, p, 0, r, s, q, far((7, 2, 64), BF), scr)
    refused("lse must have shape", call, p, 0, r, s, q, o, scr, lse=far((4, 7)))
    refused("lse must be float32", call, p, 0, r, s, q, o, scr, lse=far((7, 4), BF))
    refused("lse: a tensor is on cuda:1", call, p, 0, r, s, q, o, scr, lse=Dev((7, 4), F, dev="cuda:1"))
    refused("mask must be", call, p, 0, r, s, q, o, scr, mask=Dev((7,)))
    refused("mask holds", call, p, 0, r, s, q, o, scr, mask=Dev((6, 1)))
    refused("scratch must be uint8", call, p, 0, r, s, q, o, Dev((9,), F))
    refused("slopes holds 8", call, p, 0, r, V.make_scores(p, slopes=Dev((8,), F)), q, o, scr)
    refused("depth holds 6", call, p, 0, r, V.make_scores(p, depth=Dev((6,))), q, o, scr)
    refused("span holds 8", call, p, 0, r, V.make_scores(p, span=Dev((8, 2))), q, o, scr)
    refused("layer", call, p, 2, r, s, q, o, scr)
    refused("out must not be q", call, p, 0, r, s, q, q, scr)
    refused("lse overlaps", call, p, 0, r, s, q, o, scr, lse=Dev((7, 4), F, ptr=q.data_ptr() + 64))
    refused("lse overlaps", call, p, 0, r, s, q, o, scr, lse=Dev((7, 4), F, ptr=o.data_ptr()))
    for bad in (dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0), dict(cap=-1.0), dict(cap=float("inf")),
                dict(cap=float("nan")), dict(cap=1e-39), dict(cap=2e38), dict(window=-1)):
        refused(next(iter(bad)), call, p, 0, r, V.make_scores(p, **bad), q, o, scr)


def test_attention_mass_refuses():
    p, r = cache(), V.make_rows(Dev((3,)), 7)
    q, l, m, scr, s = far((7, 4, 64), BF), far((7, 4), F, 2), far(MASS, F, 3), far((1 << 20,), U8, 4), V.make_scores(p)
    call = V.vla_attention_mass
    refused("q must be [7, heads, 64]", call, p, 0, r, s, Dev((6, 4, 64), BF), l, m, scr)
    refused("lse must be a device", call, p, 0, r, s, q, None, m, scr)
    refused("lse must have shape", call, p, 0, r, s, q, far((4, 7), F), m, scr)
    refused("mass must be a device", call, p, 0, r, s, q, l, None, scr)
    refused("mass holds", call, p, 0, r, s, q, l, far((2, 3, 2, SLOTS - 1), F), scr)
    refused("mass must be float32", call, p, 0, r, s, q, l, far(MASS, BF), scr)
    refused("mask holds", call, p, 0, r, s, q, l, m, scr, mask=Dev((6, 1)))
    refused("slopes holds", call, p, 0, r, V.make_scores(p, slopes=Dev((3,), F)), q, l, m, scr)
    refused("cap", call, p, 0, r, V.make_scores(p, cap=-2.0), q, l, m, scr)
    refused("mass overlaps", call, p, 0, r, s, q, l, Dev(MASS, F, ptr=q.data_ptr()), scr)
    refused("mass overlaps", call, p, 0, r, s, q, Dev((7, 4), F, ptr=m.data_ptr() + 400), m, scr)


def test_evict_refuses():
    p, n = cache(), 3
    seqs, keep, kept = far((n,), torch.int32), far((n,), torch.int32, 2), far((n, SLOTS), torch.int32, 3)
    m, o = far(MASS, F, 4), far(MASS, F, 5)
    size = V.vla_pages_evict_scratch(p, n)
    scr = far((size,), U8, 6)
    call = V.vla_pages_evict
    refused("seqs must be [n]", call, p, Dev((3, 1)), keep, m, o, kept, scr)
    refused("seqs must be int32", call, p, Dev((n,), torch.int64), keep, m, o, kept, scr)
    refused("keep holds 2", call, p, seqs, Dev((2,)), m, o, kept, scr)
    refused("keep must be a device", call, p, seqs, None, m, o, kept, scr)
    refused("mass holds", call, p, seqs, keep, far((1, 3, 2, SLOTS), F), o, kept, scr)
    refused("mass_out must be a device", call, p, seqs, keep, m, None, kept, scr)
    refused("kept holds", call, p, seqs, keep, m, o, far((n, SLOTS - 1), torch.int32), scr)
    refused("first must be an integer", call, p, seqs, keep, m, o, kept, scr, first=0.5)
    refused("first and last", call, p, seqs, keep, m, o, kept, scr, first=-1)
    refused("first and last", call, p, seqs, keep, m, o, kept, scr, last=-1)
    refused("scratch: needs", call, p, seqs, keep, m, o, kept, far((size - 1,), U8, 6))
    refused("16-byte", call, p, seqs, keep, m, o, kept, Dev((size,), U8, ptr=0x10008))
    refused("overlaps mass and is not mass", call, p, seqs, keep, m, Dev(MASS, F, ptr=m.data_ptr() + 16), kept, scr)
    refused("overlaps what the call reads", call, p, seqs, keep, m, o, Dev((n, SLOTS), ptr=seqs.data_ptr()), scr)
    refused("overlaps what the call reads", call, p, seqs, keep, m, m, Dev((n, SLOTS), ptr=m.data_ptr()), scr)
    refused("overlaps what the call reads", call, p, seqs, keep, m, o, kept, Dev((size,), U8, ptr=keep.data_ptr()))
    refused("must not overlap", call, p, seqs, keep, m, o, kept, Dev((size,), U8, ptr=o.data_ptr()))
    refused("must not be negative", V.vla_pages_evict_scratch, p, -1)
    assert V._lib.vla_pages_evict_scratch(C.byref(p), (1 << 14) + 1, C.byref(C.c_int64())) == -4
    # nothing to do reads nothing
    assert V._lib.vla_pages_evict(C.byref(p), 0, None, None, 0, 0, None, None, None, None, 0, None) == 0


def test_verify_refuses():
    p, r = cache(), V.make_rows(Dev((3,)), 7)
    t, pr, kept = far((7,), torch.int32), far((7, 100), F, 2), far((7,), torch.int32, 3)
    nk, nx, d, u = (far((2,), torch.int32, 4), far((2,), torch.int32, 5), far((7, 100), F, 6), far((7,), F, 7))
    size = V.vla_verify_drafts_scratch(p, r, 100)
    scr = far((size,), U8, 8)
    call = V.vla_verify_drafts
    refused("tokens holds", call, p, r, Dev((6,)), pr, kept, nk, nx, scr)
    refused("tokens must be a device", call, p, r, None, pr, kept, nk, nx, scr)
    refused("probs must be [7, vocab]", call, p, r, t, far((6, 100), F), kept, nk, nx, scr)
    refused("float32 or bfloat16", call, p, r, t, far((7, 100), torch.float16), kept, nk, nx, scr)
    refused("probs must be a device", call, p, r, t, Dev((7, 100), F, is_cuda=False), kept, nk, nx, scr)
    refused("values must be contiguous", call, p, r, t, Dev((7, 100), F, stride=(200, 2)), kept, nk, nx, scr)
    refused("drafted must be [7, 100]", call, p, r, t, pr, kept, nk, nx, scr, drafted=far((7, 99), F), uniform=u)
    refused("drafted must be torch.float32", call, p, r, t, pr, kept, nk, nx, scr, drafted=far((7, 100), BF), uniform=u)
    refused("drafted needs uniform", call, p, r, t, pr, kept, nk, nx, scr, drafted=d)
    refused("uniform must be float32", call, p, r, t, pr, kept, nk, nx, scr, uniform=far((7,), torch.int32))
    refused("parent holds", call, p, r, t, pr, kept, nk, nx, scr, parent=Dev((5,)))
    refused("kept holds", call, p, r, t, pr, far((6,), torch.int32), nk, nx, scr)
    refused("n_kept must have shape", call, p, r, t, pr, kept, far((3,), torch.int32), nx, scr)
    refused("next must have shape", call, p, r, t, pr, kept, nk, far((7,), torch.int32), scr)
    refused("row stride", call, p, r, t, Dev((7, 100), F, stride=(50, 1)), kept, nk, nx, scr)
    refused("alignment", call, p, r, t, Dev((7, 100), F, ptr=0x10002), kept, nk, nx, scr)
    refused("scratch: needs", call, p, r, t, pr, kept, nk, nx, far((size - 1,), U8, 8))
    refused("overlaps what the call reads", call, p, r, t, pr, t, nk, nx, scr)
    refused("overlaps what the call reads", call, p, r, t, pr, kept, nk, nx, Dev((size,), U8, ptr=pr.data_ptr() + 1600))
    refused("overlaps what the call reads", call, p, r, t, pr, kept, Dev((2,), ptr=u.data_ptr()), nx, scr, uniform=u)
    refused("must not overlap", call, p, r, t, pr, kept, nk, nk, scr)
    refused("vocab", V.vla_verify_drafts_scratch, p, r, 0)
    refused("vocab", V.vla_verify_drafts_scratch, p, r, 2 ** 28 + 1)


def test_verify_without_rows_refuses():
    """Entries of a batch without rows are answered, so what the answers go to is
    looked at, and nothing else."""
    p, r = cache(), V.make_rows(Dev((3,)), 0)
    none, nk, nx, scr = Dev((0,), ptr=None), far((2,), torch.int32, 4), far((2,), torch.int32, 5), far((16,), U8, 8)
    call = V.vla_verify_drafts
    refused("n_kept holds 1", call, p, r, none, Dev((0, 9), F), none, far((1,), torch.int32), nx, scr)
    refused("next must have shape", call, p, r, none, Dev((0, 9), F), none, nk, far((3,), torch.int32), scr)
    refused("must not overlap", call, p, r, none, Dev((0, 9), F), none, nk, Dev((2,), ptr=nk.data_ptr() + 4), scr)
    refused("drafted needs uniform", call, p, r, none, Dev((0, 9), F), none, nk, nx, scr, drafted=Dev((0, 9), F))
    x, d = C.c_void_p(0x10000), V.vla_drafts(0, 9, None, None, None, 0, None, 0, None)
    lib, args = V._lib.vla_verify_drafts, (C.byref(p), C.byref(r), C.byref(d), None)
    for out in ((None, x), (x, None)):
        assert lib(*args, *out, None, 0, None) == -1
        assert "NULL" in V.vla_last_error()


@pytest.mark.parametrize("field,value,msg", [
    ("dtype", 2, "dtype"), ("head_dim", 48, "head_dim"), ("page_len", 24, "page_len"), ("k", None, "NULL"),
])
def test_descriptor_is_checked(field, value, msg):
    p = cache()
    setattr(p, field, value)
    r = V.make_rows(Dev((3,)), 7)
    for call in (lambda: V.vla_score_attention_scratch(p, r, 4), lambda: V.vla_attention_mass_scratch(p, r, 4),
                 lambda: V.vla_pages_evict_scratch(p, 2), lambda: V.vla_verify_drafts_scratch(p, r, 10)):
        refused(msg, call)


def test_null_arguments_are_errors():
    lib, p, r = V._lib, C.byref(cache()), C.byref(V.make_rows(Dev((3,)), 7))
    x, s = C.c_void_p(0x10000), C.byref(V.make_scores(cache()))
    assert lib.vla_score_attention(p, 0, r, None, None, 0, 4, x, 256, x, 256, None, x, 0, None) == -1
    assert "scores" in V.vla_last_error()
    assert lib.vla_score_attention(p, 0, r, s, x, 0, 4, x, 256, x, 256, None, x, 0, None) == -1
    assert "mask_words" in V.vla_last_error()
    assert lib.vla_score_attention_scratch(p, r, 4, None) == -1
    assert lib.vla_attention_mass(p, 0, r, s, None, 0, 4, x, 256, None, x, x, 0, None) == -1
    assert lib.vla_attention_mass(p, 0, r, s, None, 0, 4, x, 256, x, None, x, 0, None) == -1
    assert lib.vla_attention_mass_scratch(p, r, 4, None) == -1
    assert lib.vla_pages_evict(p, 2, None, x, 0, 0, x, x, x, x, 0, None) == -1
    assert lib.vla_pages_evict_scratch(p, 2, None) == -1
    assert lib.vla_verify_drafts(p, r, None, x, x, x, x, 0, None) == -1
    d = V.vla_drafts(0, 100, None, None, 0x10000, 100, None, 0, None)
    assert lib.vla_verify_drafts(p, r, C.byref(d), x, x, x, x, 0, None) == -1
    assert lib.vla_verify_drafts_scratch(p, r, 100, None) == -1
    # nothing to do reads nothing
    none = C.byref(V.make_rows(Dev((1,)), 0))
    assert lib.vla_score_attention(p, 0, none, s, None, 0, 4, None, 0, None, 0, None, None, 0, None) == 0
    assert lib.vla_attention_mass(p, 0, none, s, None, 0, 4, None, 0, None, None, None, 0, None) == 0
    assert lib.vla_verify_drafts(p, none, C.byref(d), None, None, None, None, 0, None) == 0


@pytest.mark.parametrize("struct", ["vla_scores", "vla_drafts"])
def test_structs_match_header(struct):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vla.h")).read(), flags=re.S)
    body = re.search(r"typedef struct " + struct + r"\s*\{(.*?)\}\s*" + struct + ";", src, flags=re.S).group(1)
    fields = []
    for t, names in re.findall(r"^\s*((?:const\s+)?\w+\s*\*?)\s*([\w\s,]+);", body, flags=re.M):
        fields += [(t.replace("const", "").strip(), n.strip()) for n in names.split(",")]
    ctype = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}
    got = getattr(V, struct)._fields_
    assert [n for _, n in fields] == [n for n, _ in got]
    for (t, n), (_, gt) in zip(fields, got):
        assert gt is (C.c_void_p if t.endswith("*") else ctype[t]), n
