"""CPU checks of the paged cache's argument checks: the binding refuses wrong
tensors before the library is called, and the C entry points refuse wrong
descriptors before anything is launched (no GPU here: a call that got past the
checks would fail with another status). The structures match the header."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2609_22335_amd as V

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, F, I = torch.bfloat16, torch.float32, torch.int32


class Dev:
    """Stands in for a device tensor: what the binding's checks read."""

    def __init__(self, shape, dtype=I, is_cuda=True, contiguous=True, stride=None, ptr=0x10000, dev="cuda:0"):
        self.shape, self.dtype, self.is_cuda, self._c, self._p = tuple(shape), dtype, is_cuda, contiguous, ptr
        st, n = [], 1
        for d in reversed(self.shape):
            st.insert(0, n)
            n *= d
        self._n, self._s = n, tuple(stride or st)
        self.device = torch.device(dev)

    def data_ptr(self):
        return self._p

    def numel(self):
        return self._n

    def get_device(self):
        return self.device.index if self.is_cuda else -1

    def stride(self):
        return self._s

    def is_contiguous(self):
        return self._c


@pytest.fixture(autouse=True)
def on_device_0(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


def cache(**bad):
    t = dict(k=Dev((2, 10, 2, 16, 64), BF), v=Dev((2, 10, 2, 16, 64), BF), table=Dev((3, 5)), lens=Dev((3,)),
             held=Dev((3,)), refs=Dev((10,)), status=Dev((1,)))
    t.update(bad)
    return V.make_pages(**t)


def refused(msg, f, *a, **k):
    with pytest.raises(V.VlaError) as e:
        f(*a, **k)
    assert e.value.code == -1 and msg in str(e.value), str(e.value)


@pytest.mark.parametrize("bad,msg", [
    (dict(k=Dev((2, 10, 2, 16, 64), torch.float16)), "bfloat16 or float32"),
    (dict(k=Dev((2, 10, 32, 64), BF)), "k must be [layers"),
    (dict(v=Dev((2, 10, 2, 16, 32), BF)), "v holds"),
    (dict(v=Dev((2, 10, 2, 16, 64), F)), "v must be bfloat16"),
    (dict(k=Dev((2, 10, 2, 16, 64), BF, contiguous=False)), "contiguous"),
    (dict(k=Dev((2, 10, 2, 16, 64), BF, is_cuda=False)), "device"),
    (dict(table=Dev((15,))), "table must be"),
    (dict(table=Dev((3, 5), torch.int64)), "table must be int32"),
    (dict(lens=Dev((4,))), "lens must have shape"),
    (dict(held=Dev((2,))), "held holds"),
    (dict(refs=Dev((9,))), "refs holds"),
    (dict(status=Dev((2,))), "status must have shape"),
    (dict(refs=None), "refs must be"),
    (dict(refs=Dev((10,), dev="cuda:1")), "refs is on cuda:1"),
])
def test_make_pages_refuses(bad, msg):
    refused(msg, cache, **bad)


def test_make_rows_and_rope_refuse():
    refused("start must be", V.make_rows, None, 4)
    refused("start must be [n_entries + 1]", V.make_rows, Dev((0,)), 4)
    refused("seqs must have shape", V.make_rows, Dev((4,)), 4, Dev((4,)))
    refused("seqs is on", V.make_rows, Dev((4,)), 4, Dev((3,), dev="cuda:1"))
    refused("both tables", V.make_rope_norm, Dev((9, 32), F))
    refused("sin holds", V.make_rope_norm, Dev((9, 32), F), Dev((9, 16), F))
    refused("q_gain must be float32", V.make_rope_norm, None, None, Dev((64,), BF))
    assert V.make_rope_norm(Dev((9, 24), F), Dev((9, 24), F)).rot_dim == 48


def test_calls_refuse_wrong_operands():
    p, r = cache(), V.make_rows(Dev((3,)), 7)
    rope = V.make_rope_norm(Dev((9, 32), F), Dev((9, 32), F), Dev((64,), F), Dev((64,), F))
    q, k = Dev((7, 4, 64), BF), Dev((7, 2, 64), BF)
    refused("q must be [7, heads, 64]", V.vla_qk_norm_rope, p, 0, r, rope, Dev((6, 4, 64), BF), k, k, q)
    refused("k must be [7, 2, 64]", V.vla_qk_norm_rope, p, 0, r, rope, q, q, k, q)
    refused("v must be torch.bfloat16", V.vla_qk_norm_rope, p, 0, r, rope, q, k, Dev((7, 2, 64), F), q)
    refused("q_out must be [7, 4, 64]", V.vla_qk_norm_rope, p, 0, r, rope, q, k, k, k)
    refused("contiguous", V.vla_qk_norm_rope, p, 0, r, rope, Dev((7, 4, 64), BF, stride=(64, 448, 1)), k, k, q)
    refused("pos holds", V.vla_qk_norm_rope, p, 0, r, rope, q, k, k, q, pos=Dev((6,)))
    refused("q_gain holds", V.vla_qk_norm_rope, p, 0, r, V.make_rope_norm(q_gain=Dev((32,), F)), q, k, k, q)
    refused("layer", V.vla_qk_norm_rope, p, 2, r, rope, q, k, k, q)
    refused("nq must be", V.vla_qk_norm_rope, p, 0, r, rope, Dev((7, 3, 64), BF), k, k, Dev((7, 3, 64), BF))
    refused("rot_dim", V.vla_qk_norm_rope, p, 0, r, V.make_rope_norm(Dev((9, 4), F), Dev((9, 4), F)), q, k, k, q)
    refused("eps", V.vla_qk_norm_rope, p, 0, r, V.make_rope_norm(q_gain=Dev((64,), F), eps=0), q, k, k, q)
    refused("16-byte", V.vla_qk_norm_rope, p, 0, r, rope, Dev((7, 4, 64), BF, ptr=0x10008), k, k, q)
    refused("16-byte", V.vla_qk_norm_rope, p, 0, r, rope, Dev((7, 4, 64), BF, stride=(260, 64, 1)), k, k, q)
    refused("row stride", V.vla_qk_norm_rope, p, 0, r, rope, Dev((7, 4, 64), BF, stride=(64, 64, 1)), k, k, q)
    refused("q's row stride", V.vla_qk_norm_rope, p, 0, r, rope, Dev((7, 4, 64), BF, stride=(512, 64, 1)), k, k, q)
    refused("the current device is 0", V.vla_qk_norm_rope, cache(**{n: Dev(s, t, dev="cuda:1") for n, s, t in [
        ("k", (2, 10, 2, 16, 64), BF), ("v", (2, 10, 2, 16, 64), BF), ("table", (3, 5), I), ("lens", (3,), I),
        ("held", (3,), I), ("refs", (10,), I), ("status", (1,), I)]}),
        0, V.make_rows(Dev((3,), dev="cuda:1"), 7), V.make_rope_norm(),
        *(Dev(s, BF, dev="cuda:1") for s in ((7, 4, 64), (7, 2, 64), (7, 2, 64), (7, 4, 64))))
    refused("a tensor is on cuda:1", V.vla_qk_norm_rope, p, 0, r, rope, q, k, k, Dev((7, 4, 64), BF, dev="cuda:1"))

    scr = Dev((1 << 20,), torch.uint8)
    refused("mask must be", V.vla_tree_attention, p, 0, r, q, q, scr, mask=Dev((7,)))
    refused("mask holds", V.vla_tree_attention, p, 0, r, q, q, scr, mask=Dev((6, 1)))
    refused("mask must be int32", V.vla_tree_attention, p, 0, r, q, q, scr, mask=Dev((7, 1), torch.int64))
    refused("scratch must be uint8", V.vla_tree_attention, p, 0, r, q, q, Dev((9,), F))
    refused("out must be [7, 4, 64]", V.vla_tree_attention, p, 0, r, q, k, scr)
    refused("out must not be q", V.vla_tree_attention, p, 0, r, q, q, scr)
    refused("scale", V.vla_tree_attention, p, 0, r, q, Dev((7, 4, 64), BF, ptr=0x20000), scr, scale=0.0)
    refused("scale", V.vla_tree_attention, p, 0, r, q, Dev((7, 4, 64), BF, ptr=0x20000), scr, scale=float("inf"))
    refused("src must be", V.vla_pages_fork, p, Dev((2, 2)), Dev((4,)), Dev((4,)))
    refused("dst must have shape", V.vla_pages_fork, p, Dev((2,)), Dev((3,)), Dev((2,)))
    refused("made holds", V.vla_pages_fork, p, Dev((2,)), Dev((2,)), Dev((1,)))
    refused("kept holds", V.vla_pages_commit, p, r, Dev((6,)), Dev((2,)))
    refused("n_kept must have shape", V.vla_pages_commit, p, r, Dev((7,)), Dev((3,)))
    refused("kept needs n_kept", V.vla_pages_commit, p, r, Dev((7,)))
    refused("seqs must be int32", V.vla_pages_release, p, Dev((2,), torch.int64))


@pytest.mark.parametrize("field,value,msg", [
    ("dtype", 2, "dtype"), ("layers", 0, "positive"), ("kv_heads", -1, "positive"), ("n_pages", 0, "positive"),
    ("head_dim", 48, "head_dim"), ("head_dim", 288, "head_dim"), ("page_len", 24, "page_len"),
    ("page_len", 8, "page_len"), ("page_len", 512, "page_len"), ("n_pages", (1 << 28) + 1, "2^28"),
    ("max_pages", 1 << 27, "2^30"), ("k", None, "NULL"), ("status", None, "NULL"), ("v", 0x10008, "aligned"),
])
def test_descriptor_is_checked(field, value, msg):
    p = cache()
    setattr(p, field, value)
    r = V.make_rows(Dev((3,)), 0)
    for call in (lambda: V.vla_pages_init(p), lambda: V.vla_pages_reserve(p, r),
                 lambda: V.vla_tree_attention_scratch(p, r, 4), lambda: V.vla_pages_commit(p, r),
                 lambda: V.vla_pages_release(p, Dev((1,))),
                 lambda: V.vla_pages_fork(p, Dev((1,)), Dev((1,)), Dev((1,)))):
        refused(msg, call)


def test_fp32_head_dim_is_at_most_128():
    refused("head_dim", V.vla_pages_init, cache(k=Dev((1, 10, 2, 16, 160), F), v=Dev((1, 10, 2, 16, 160), F)))


def test_null_arguments_are_errors():
    lib, p, r = V._lib, C.byref(cache()), V.make_rows(Dev((3,)), 7)
    assert lib.vla_pages_init(None, None) == -1
    assert lib.vla_pages_reserve(p, None, None) == -1
    assert lib.vla_qk_norm_rope(p, 0, C.byref(r), None, None, 4, None, 256, None, 128, None, 128, None, 256, None) == -1
    assert lib.vla_tree_attention_scratch(p, C.byref(r), 4, None) == -1
    assert lib.vla_pages_fork(p, 2, None, None, None, None) == -1
    assert lib.vla_pages_fork(p, -1, None, None, None, None) == -1
    assert lib.vla_pages_release(p, 1, None, None) == -1
    assert lib.vla_ctx_to_pages(None, None, p, 0, None, None) == -1
    bad = V.make_rows(Dev((3,)), -1)
    assert lib.vla_pages_reserve(p, C.byref(bad), None) == -1
    # nothing to do reads nothing
    assert lib.vla_pages_fork(p, 0, None, None, None, None) == 0
    assert lib.vla_pages_release(p, 0, None, None) == 0


def test_grids_of_2_to_32_threads_are_refused():
    lib, p, x = V._lib, C.byref(cache()), C.c_void_p(0x10000)
    n = 1 << 24
    r = V.make_rows(Dev((n + 1,)), 1 << 28)
    assert lib.vla_pages_release(p, n, x, None) == -4
    assert lib.vla_pages_fork(p, n, x, x, x, None) == -4
    assert lib.vla_pages_commit(p, C.byref(r), x, x, None) == -4
    rope = V.make_rope_norm()
    assert lib.vla_qk_norm_rope(p, 0, C.byref(r), C.byref(rope), None, 4, x, 256, x, 128, x, 128, x, 256, None) == -4
    assert "grid" in V.vla_last_error()


@pytest.mark.parametrize("struct", ["vla_pages", "vla_rows", "vla_rope_norm"])
def test_structs_match_header(struct):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vla.h")).read(), flags=re.S)
    body = re.search(r"typedef struct " + struct + r"\s*\{(.*?)\}\s*" + struct + ";", src, flags=re.S).group(1)
    fields = []
    for t, names in re.findall(r"^\s*((?:const\s+)?\w+\s*\*?)\s*([\w\s,]+);", body, flags=re.M):
        fields += [(t.replace("const", "").strip(), n.strip()) for n in names.split(",")]
    ctype = {"int32_t": C.c_int32, "float": C.c_float}
    got = getattr(V, struct)._fields_
    assert [n for _, n in fields] == [n for n, _ in got]
    for (t, n), (_, gt) in zip(fields, got):
        assert gt is (C.c_void_p if t.endswith("*") else ctype[t]), n
