"""The C ABI of the paged cache on the CPU: exports, sizes and refusals, all of
which happen before any GPU work."""

import ctypes
import os
import re

import numpy as np
import pytest

from oracle import paged_oracle as PO
from paper_2606_01790_amd import starkv as sk

torch = pytest.importorskip("torch")

from paper_2606_01790_amd import paged as pg  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "starkv_paged.h")

pytestmark = pytest.mark.skipif(not os.path.exists(sk.LIB_PATH),
                                reason="libstarkv.so not built")

FAKE = 0x10000          # an aligned non-null address; never dereferenced here
BIG = 1 << 40


def cache(**kw):
    base = dict(n_layers=28, H=28, G=4, d=128, dtype=sk.BF16, page_tokens=64, n_pages=500, n_slots=8,
                max_pages=100, reserved=0, layer_stride=500 * 64 * 4 * 128,
                page_stride=64 * 4 * 128, group_stride=64 * 128, token_stride=128, k=FAKE, v=FAKE,
                table=FAKE, len=FAKE, refs=FAKE)
    base.update(kw)
    return pg.Paged(**base)


def name(code):
    return sk.STATUS[code]


def ints(x):
    return (ctypes.c_int32 * len(x))(*x) if x is not None else None


def test_header_symbols_are_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(starkv_[a-z_]+)\s*\(", text))
    assert names == set(pg.SIGNATURES)
    for n in names:
        assert hasattr(pg.lib(), n), n


def test_constants_match_the_header():
    text = open(HEADER).read()
    for n, val in (("STARKV_MAX_SEQS", pg.MAX_SEQS), ("STARKV_MAX_DRAFT_WORDS", pg.MAX_DRAFT_WORDS),
                   ("STARKV_SEQ_OK", PO.OK), ("STARKV_SEQ_NO_PAGES", PO.NO_PAGES),
                   ("STARKV_SEQ_RANGE", PO.RANGE)):
        assert int(re.search(r"#define %s (\d+)" % n, text).group(1)) == val
    assert (pg.SEQ_OK, pg.SEQ_NO_PAGES, pg.SEQ_RANGE) == (PO.OK, PO.NO_PAGES, PO.RANGE)


@pytest.mark.parametrize("kw,code", [
    (dict(n_layers=0), "E_SHAPE"), (dict(G=3), "E_SHAPE"), (dict(G=0), "E_SHAPE"),
    (dict(d=96), "E_SHAPE"), (dict(dtype=2), "E_DTYPE"), (dict(page_tokens=48), "E_SHAPE"),
    (dict(page_tokens=8), "E_SHAPE"), (dict(page_tokens=2048), "E_SHAPE"),
    (dict(n_pages=0), "E_SHAPE"), (dict(n_slots=0), "E_SHAPE"), (dict(max_pages=0), "E_SHAPE"),
    (dict(max_pages=1 << 21), "E_SHAPE"), (dict(reserved=1), "E_SHAPE"),
    (dict(token_stride=120), "E_SHAPE"), (dict(token_stride=132), "E_ALIGN"),
    (dict(token_stride=1 << 27), "E_SHAPE"), (dict(page_stride=-8), "E_SHAPE"), (dict(group_stride=4), "E_ALIGN"),
    (dict(k=None), "E_NULL"), (dict(refs=None), "E_NULL"), (dict(v=FAKE + 8), "E_ALIGN"),
    (dict(table=FAKE + 2), "E_ALIGN"),
])
def test_every_call_rejects_a_bad_cache(kw, code):
    c, L, one = cache(**kw), pg.lib(), ints([1])
    r = ctypes.byref(c)
    lay = sk.KVLayout(0, 128, 512)
    assert name(L.starkv_pages_init(r, None)) == code
    assert name(L.starkv_pages_grow(r, one, 1, one, FAKE, FAKE, BIG, None)) == code
    assert name(L.starkv_pages_write(r, one, 1, one, FAKE, FAKE, ctypes.byref(lay), None)) == code
    assert name(L.starkv_pages_fork(r, one, ints([2]), 1, None)) == code
    assert name(L.starkv_pages_free(r, one, 1, 0, 0, None)) == code
    assert name(L.starkv_pages_compact(r, one, 1, None, FAKE, 0, 4, None, 0, FAKE, FAKE, BIG,
                                       None)) == code
    assert name(L.starkv_attend_tree(r, one, 1, one, FAKE, FAKE, 1, 64, FAKE, None, FAKE, BIG,
                                     None)) == code
    assert name(L.starkv_attend_window(r, one, 1, one, FAKE, 0, 0, 64, FAKE, None, FAKE, BIG,
                                       None)) == code
    assert L.starkv_pages_workspace_bytes(r, 1, 10) == 0
    assert L.starkv_attend_workspace_bytes(r, one, 1, 5000) == 0


def test_a_null_cache():
    L = pg.lib()
    assert name(L.starkv_pages_init(None, None)) == "E_NULL"
    assert L.starkv_pages_workspace_bytes(None, 1, 1) == 0


BAD_SLOTS = [([-1], "E_PARAM"), ([8], "E_PARAM"), (None, "E_NULL"), (list(range(8)) * 33, "E_PARAM")]


@pytest.mark.parametrize("slots,code", BAD_SLOTS + [([3, 3], "E_PARAM")])
def test_slot_lists(slots, code):
    L, c = pg.lib(), cache()
    r, n = ctypes.byref(c), len(slots) if slots else 1
    one, sl = ints([1] * n), ints(slots)
    lay = sk.KVLayout(0, 128, 512)
    assert name(L.starkv_pages_grow(r, sl, n, one, FAKE, FAKE, BIG, None)) == code
    assert name(L.starkv_pages_write(r, sl, n, one, FAKE, FAKE, ctypes.byref(lay), None)) == code
    assert name(L.starkv_pages_fork(r, ints([5] * n), sl, n, None)) == code
    assert name(L.starkv_pages_free(r, sl, n, 0, 0, None)) == code
    assert name(L.starkv_pages_compact(r, sl, n, None, FAKE, 0, 4, None, 0, FAKE, FAKE, BIG,
                                       None)) == code
    if slots != [3, 3]:      # the attentions only read: a slot may repeat
        assert name(L.starkv_attend_window(r, sl, n, one, FAKE, 0, 0, 64, FAKE, None, FAKE, BIG,
                                           None)) == code


def test_negative_counts_of_sequences():
    L, r, one = pg.lib(), ctypes.byref(cache()), ints([1])
    assert name(L.starkv_pages_free(r, one, -1, 0, 0, None)) == "E_PARAM"
    assert name(L.starkv_attend_window(r, one, -1, one, FAKE, 0, 0, 64, FAKE, None, FAKE, BIG,
                                       None)) == "E_PARAM"


def test_empty_calls_do_nothing():
    L, r = pg.lib(), ctypes.byref(cache())
    lay = sk.KVLayout(0, 128, 512)
    assert L.starkv_pages_grow(r, None, 0, None, None, None, 0, None) == 0
    assert L.starkv_pages_write(r, None, 0, None, None, None, ctypes.byref(lay), None) == 0
    assert L.starkv_pages_write(r, ints([1]), 1, ints([0]), None, None, ctypes.byref(lay), None) == 0
    assert L.starkv_pages_fork(r, None, None, 0, None) == 0
    assert L.starkv_pages_free(r, None, 0, 0, 0, None) == 0
    assert L.starkv_pages_compact(r, None, 0, None, None, 0, 0, None, 0, None, None, 0, None) == 0
    assert L.starkv_attend_window(r, None, 0, None, None, 0, 0, 1, None, None, None, 0, None) == 0
    assert L.starkv_attend_tree(r, ints([1, 2]), 2, ints([0, 0]), None, None, 1, 1, None, None, None,
                                0, None) == 0


def test_grow_arguments():
    L, r, one = pg.lib(), ctypes.byref(cache()), ints([1])
    grow = lambda add, status=FAKE, ws=FAKE, wb=BIG: name(
        L.starkv_pages_grow(r, one, 1, ints(add), status, ws, wb, None))
    assert grow([-1]) == "E_PARAM"
    assert grow([(1 << 26) + 1]) == "E_PARAM"
    assert grow(None) == "E_NULL"
    assert grow([1], status=None) == "E_NULL"
    assert grow([1], status=FAKE + 1) == "E_ALIGN"
    assert grow([1], ws=None) == "E_WORKSPACE"
    assert grow([1], ws=FAKE + 8) == "E_ALIGN"
    need = L.starkv_pages_workspace_bytes(r, 1, 1)
    # two fresh pages, one record, a table row, each padded to 256 bytes
    assert need == 256 + 256 + 512
    assert grow([1], wb=need - 1) == "E_WORKSPACE"
    assert L.starkv_pages_workspace_bytes(r, 257, 1) == 0
    assert L.starkv_pages_workspace_bytes(r, 1, -1) == 0


def test_write_arguments():
    L, r, one = pg.lib(), ctypes.byref(cache()), ints([1])

    def write(rows=(2,), k=FAKE, v=FAKE, lay=(0, 128, 512)):
        lay = ctypes.byref(sk.KVLayout(*lay)) if lay else None
        return name(L.starkv_pages_write(r, one, 1, ints(rows), k, v, lay, None))

    assert write(rows=[-1]) == "E_PARAM"
    assert write(rows=[64 * 100 + 1]) == "E_PARAM"     # more than a table row holds
    assert write(rows=None) == "E_NULL"
    assert write(k=None) == "E_NULL"
    assert write(lay=None) == "E_NULL"
    assert write(v=FAKE + 4) == "E_ALIGN"
    assert write(lay=(0, 4, 512)) == "E_ALIGN"
    assert write(lay=(0, 128, -512)) == "E_SHAPE"


def test_fork_arguments():
    L, r = pg.lib(), ctypes.byref(cache())
    fork = lambda a, b: name(L.starkv_pages_fork(r, ints(a), ints(b), len(b), None))
    assert fork([1], [1]) == "E_PARAM"
    assert fork([1, 2], [2, 3]) == "E_PARAM"      # a chain within one call
    assert fork([1, 2], [3, 3]) == "E_PARAM"
    assert fork([9], [3]) == "E_PARAM"


def test_free_arguments():
    L, r, one = pg.lib(), ctypes.byref(cache()), ints([1])
    assert name(L.starkv_pages_free(r, one, 1, -1, 0, None)) == "E_PARAM"
    assert name(L.starkv_pages_free(r, one, 1, 0, -1, None)) == "E_PARAM"


def test_compact_arguments():
    L, r, one = pg.lib(), ctypes.byref(cache()), ints([1])

    def compact(span=None, idx=FAKE, ls=0, B=4, counts=None, tail=0, status=FAKE, ws=FAKE, wb=BIG):
        return name(L.starkv_pages_compact(r, one, 1, ints(span), idx, ls, B, counts, tail, status, ws,
                                           wb, None))

    assert compact(span=[-1]) == "E_PARAM"
    assert compact(idx=None) == "E_NULL"
    assert compact(status=None) == "E_NULL"
    assert compact(idx=FAKE + 2) == "E_ALIGN"
    assert compact(counts=FAKE + 2) == "E_ALIGN"
    assert compact(ls=-1) == "E_SHAPE"
    assert compact(B=-1) == "E_BUDGET"
    assert compact(tail=-1) == "E_BUDGET"
    assert compact(B=1 << 26, tail=1) == "E_BUDGET"
    need = L.starkv_pages_workspace_bytes(r, 1, 4 + 32)
    assert compact(tail=32, wb=need - 1) == "E_WORKSPACE"
    assert compact(ws=None) == "E_WORKSPACE"


def test_attention_arguments():
    L, r = pg.lib(), ctypes.byref(cache())

    def tree(rows=(8,), q=FAKE, mask=FAKE, words=1, max_len=5000, out=FAKE, lse=None, ws=FAKE, wb=BIG):
        return name(L.starkv_attend_tree(r, ints([1]), 1, ints(rows), q, mask, words, max_len, out, lse,
                                         ws, wb, None))

    def window(w=0, s=0, rows=(8,), max_len=5000, ws=FAKE, wb=BIG):
        return name(L.starkv_attend_window(r, ints([1]), 1, ints(rows), FAKE, w, s, max_len, FAKE, None,
                                           ws, wb, None))

    assert tree(rows=[-1]) == "E_PARAM"
    assert tree(rows=[65]) == "E_PARAM"               # more rows than mask bits
    assert tree(words=0) == "E_PARAM" and tree(words=5) == "E_PARAM"
    assert tree(rows=[257], words=4) == "E_PARAM"
    assert tree(rows=None) == "E_NULL"
    assert tree(q=None) == "E_NULL" and tree(mask=None) == "E_NULL" and tree(out=None) == "E_NULL"
    assert tree(q=FAKE + 8) == "E_ALIGN" and tree(out=FAKE + 8) == "E_ALIGN"
    assert tree(mask=FAKE + 4) == "E_ALIGN" and tree(lse=FAKE + 2) == "E_ALIGN"
    assert tree(max_len=0) == "E_PARAM" and tree(max_len=(1 << 26) + 1) == "E_PARAM"
    assert window(w=-1) == "E_PARAM" and window(s=-1) == "E_PARAM"
    assert window(w=(1 << 26) + 1) == "E_PARAM" and window(s=(1 << 26) + 1) == "E_PARAM"
    assert window(rows=[6401]) == "E_PARAM"           # more than a table row holds
    need = L.starkv_attend_workspace_bytes(r, ints([8]), 1, 5000)
    assert need > 0
    assert tree(ws=None) == "E_WORKSPACE" and window(wb=need - 1) == "E_WORKSPACE"
    assert window(ws=FAKE + 8) == "E_ALIGN"
    # a bound above what a table row holds is the table row's
    assert L.starkv_attend_workspace_bytes(r, ints([8]), 1, 6400) == \
        L.starkv_attend_workspace_bytes(r, ints([8]), 1, 1 << 26)
    assert L.starkv_attend_workspace_bytes(r, ints([8]), 1, 0) == 0


def test_attention_of_more_rows_than_a_launch_holds():
    L = pg.lib()
    # 28 layers, 4 groups of 7 heads: 2^23 / 112 tiles of 128 rows, of 16 in float32
    for dtype, tile in ((sk.BF16, 128), (sk.F32, 16)):
        c = ctypes.byref(cache(dtype=dtype, max_pages=1 << 20))
        most = (1 << 23) // 112 * tile // 7
        for rows in ([most + tile], [1] * 255 + [most]):
            assert name(L.starkv_attend_window(c, ints([1] * len(rows)), len(rows), ints(rows), FAKE, 0,
                                               0, 1 << 20, FAKE, None, FAKE, BIG, None)) == "E_PARAM"
    # one layer of one group of 64 heads: 2^26 tokens are 2^32 rows
    c = ctypes.byref(cache(n_layers=1, H=64, G=1, max_pages=1 << 20))
    assert name(L.starkv_attend_window(c, ints([1]), 1, ints([1 << 26]), FAKE, 0, 0, 1, FAKE, None, FAKE,
                                       BIG, None)) == "E_PARAM"


@pytest.mark.parametrize("dtype", [sk.BF16, sk.F32])
@pytest.mark.parametrize("n_layers,n,rows", [(1, 32, 1), (28, 32, 1), (28, 256, 1), (1, 256, 4), (4, 8, 40),
                                             (28, 1, 64)])
def test_workspace_of_long_table_rows(dtype, n_layers, n, rows):
    """At most 4,096 partial tiles of 128 rows, whatever the bound on the
    lengths."""
    c = cache(dtype=dtype, n_layers=n_layers, max_pages=1 << 20)
    got = pg.lib().starkv_attend_workspace_bytes(ctypes.byref(c), ints([rows] * n), n, 1 << 26)
    tile = 16 if dtype == sk.F32 or rows == 1 else 32 if rows == 4 else 128
    assert 0 <= got <= 4096 * tile * (128 + 2) * 4 + 1024


def test_the_binding_refuses_host_tensors():
    k = torch.zeros(1, 4, 2, 16, 64, dtype=torch.bfloat16)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        pg.Cache(k, k.clone(), i(2, 3), i(2), i(4), 4)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        pg.Cache(k.half(), k.half(), i(2, 3), i(2), i(4), 4)
    with pytest.raises(ValueError, match="strides"):
        pg.Cache(k, k.transpose(3, 4), i(2, 3), i(2), i(4), 4)


# ------------------------------------------------------------------ the host model

def small(n_pages=6):
    z = np.zeros((1, n_pages, 1, 4, 2), dtype=np.int32)
    return PO.PagedModel(z, z.copy(), 4, 5)


def test_model_shares_copies_and_frees():
    m = small()
    assert list(m.grow([1], [6])) == [PO.OK]
    rows = np.arange(12, dtype=np.int32).reshape(1, 6, 1, 2) + 1
    m.write([1], [6], rows, -rows)
    m.fork([1, 1], [0, 2])
    assert list(m.refs) == [3, 3, 0, 0, 0, 0]
    assert list(m.grow([0, 1], [1, 2])) == [PO.OK, PO.OK]      # both copy page 1
    assert m.table[0, 1] == 2 and m.table[1, 1] == 3 and list(m.refs) == [3, 1, 1, 1, 0, 0]
    assert (m.k[0, 2, 0, :2] == rows[0, 4:, 0]).all() and (m.k[0, 2, 0, 2:] == 0).all()
    m.free([1, 2])
    assert list(m.refs) == [1, 0, 1, 0, 0, 0] and m.len[1] == 0
    assert list(m.grow([3], [17])) == [PO.NO_PAGES] and list(m.grow([3], [21])) == [PO.RANGE]


def test_model_compacts():
    m = small()
    m.grow([0], [11])
    rows = np.arange(22, dtype=np.int32).reshape(1, 11, 1, 2)
    m.write([0], [11], rows, rows + 100)
    idx = np.array([[[1, 3, 9]]], dtype=np.int32)        # 9 lies in the tail: a zero row
    assert list(m.compact([0], idx, tail=2)) == [PO.OK]
    got = [m.k[0, m.at(0, t)[0], 0, m.at(0, t)[1], 0] for t in range(5)]
    assert m.len[0] == 5 and got == [2, 6, 0, 18, 20]
    assert list(m.compact([0], np.array([[[1]]], dtype=np.int32), span=[3])) == [PO.OK]
    got = [m.k[0, m.at(0, t)[0], 0, m.at(0, t)[1], 0] for t in range(3)]
    assert m.len[0] == 3 and got == [2, 6, 18] and m.refs.sum() == 1


def test_reference_attention_on_closed_forms():
    z = np.zeros((1, 2, 1, 4, 2))
    m = PO.PagedModel(z, z.copy(), 1, 2)
    m.table[0], m.len[0] = [1, 0], 5
    for t in range(5):
        m.v[0, m.at(0, t)[0], 0, m.at(0, t)[1]] = [t, -t]
    f = lambda x: np.asarray(x, dtype=np.float64)
    q = np.zeros((2, 1, 2))
    o, lse, _, _ = PO.attend(m, 0, q, PO.see_window(5, 2, 2, 1), f, 0)
    assert np.allclose(o[:, 0, 0], [(0 + 2 + 3) / 3, (0 + 3 + 4) / 3]) and np.allclose(lse, np.log(3))
    o, lse, _, _ = PO.attend(m, 0, q, PO.see_tree(5, 2, np.array([[2], [0]], dtype=np.uint64)), f, 0)
    assert np.allclose(o[:, 0, 0], [(0 + 1 + 2 + 4) / 4, 1])
    m.k[0, 0, 0, 0] = [3, 4]          # token 4: logit 25 / sqrt(2) for q = (3, 4)
    o, lse, mass, size = PO.attend(m, 0, q + [3, 4], PO.see_window(5, 2, 1, 0), f, 0)
    assert np.allclose(o[:, 0], [[3, -3], [4, -4]]) and np.allclose(mass[1, 0], 4)
    assert np.allclose(lse[1], 25 / np.sqrt(2)) and np.allclose(size[1], 25 / np.sqrt(2))
