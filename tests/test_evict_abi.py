"""The C ABI of 4-bit caches, reading, accumulated weights and eviction on the CPU:
sizes and refusals, all of which happen before any GPU work."""

import ctypes
import os
import re

import pytest

from oracle import evict_oracle as EO
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


def fp4(**kw):
    block = pg.fp4_block_bytes(64, 128)
    return cache(**dict(dict(dtype=pg.FP4, layer_stride=500 * 4 * block, page_stride=4 * block,
                             group_stride=block, token_stride=64), **kw))


def name(code):
    return sk.STATUS[code]


def ints(x):
    return (ctypes.c_int32 * len(x))(*x) if x is not None else None


LAY = sk.KVLayout(0, 128, 512)


def calls(c):
    """Every call on a cache, with arguments that are right."""
    L, r, one = pg.lib(), ctypes.byref(c), ints([1])
    return dict(
        init=lambda: L.starkv_pages_init(r, None),
        grow=lambda: L.starkv_pages_grow(r, one, 1, one, FAKE, FAKE, 0, None),
        write=lambda: L.starkv_pages_write(r, ints([8]), 1, one, FAKE, FAKE, ctypes.byref(LAY), None),
        read=lambda: L.starkv_pages_read(r, ints([8]), 1, one, FAKE, FAKE, ctypes.byref(LAY), None),
        mass=lambda: L.starkv_mass_add(r, ints([8]), 1, one, FAKE, FAKE, 0, 0, 64, FAKE, FAKE, FAKE, BIG, None),
        fork=lambda: L.starkv_mass_fork(r, ints([8]), one, 1, FAKE, None),
        evict=lambda: L.starkv_pages_evict(r, ints([8]), 1, FAKE, 4, 4, 4, FAKE, FAKE, FAKE, BIG, None))


def test_constants_match_the_header():
    text = open(HEADER).read()
    for n, val in (("STARKV_FP4", pg.FP4), ("STARKV_SEQ_SHORT", EO.SHORT)):
        assert int(re.search(r"#define %s (\d+)" % n, text).group(1)) == val
    assert pg.SEQ_SHORT == EO.SHORT


@pytest.mark.parametrize("kw,code", [
    (dict(token_stride=128), "E_SHAPE"), (dict(token_stride=32), "E_SHAPE"), (dict(d=64), "E_SHAPE"),
    (dict(d=96, token_stride=48), "E_SHAPE"), (dict(group_stride=8), "E_ALIGN"), (dict(page_stride=-16), "E_SHAPE"),
    (dict(k=FAKE + 8), "E_ALIGN"), (dict(page_tokens=8), "E_SHAPE"), (dict(dtype=3), "E_DTYPE"),
    (dict(dtype=5), "E_DTYPE"), (dict(G=5), "E_SHAPE"), (dict(v=None), "E_NULL")])
def test_bad_caches(kw, code):
    for n, f in calls(fp4(**kw)).items():
        assert name(f()) == code, n
    r = ctypes.byref(fp4(**kw))
    assert pg.lib().starkv_mass_workspace_bytes(r, ints([900]), 1, 5000) == 0
    assert pg.lib().starkv_evict_workspace_bytes(r, 1, 1, 1, 1) == 0


def test_good_caches():
    """d 64 and 128 of 4 bits pass the cache's check: the slot, or the workspace, is
    refused instead."""
    block = pg.fp4_block_bytes(64, 64)
    for c in (fp4(), fp4(d=64, token_stride=32, group_stride=block, page_stride=4 * block, layer_stride=0), cache()):
        got = {n: name(f()) for n, f in calls(c).items() if n != "init"}
        assert got.pop("grow") == "E_WORKSPACE" and set(got.values()) == {"E_PARAM"}, got
    assert pg.fp4_block_bytes(16, 64) == 544 and pg.fp4_block_bytes(64, 128) == 4352


@pytest.mark.parametrize("c", [cache(), fp4()])
def test_read_arguments(c):
    L, r, one = pg.lib(), ctypes.byref(c), ints([1])

    def read(slots=(1,), rows=(2,), k=FAKE, v=FAKE, lay=(0, 128, 512)):
        lay = ctypes.byref(sk.KVLayout(*lay)) if lay else None
        return name(L.starkv_pages_read(r, ints(slots), len(rows or (1,)), ints(rows), k, v, lay, None))

    assert read(rows=[-1]) == "E_PARAM" and read(rows=[64 * 100 + 1]) == "E_PARAM"
    assert read(rows=None) == "E_NULL" and read(k=None) == "E_NULL" and read(lay=None) == "E_NULL"
    assert read(v=FAKE + 4) == "E_ALIGN" and read(lay=(0, 4, 512)) == "E_ALIGN"
    assert read(lay=(0, 128, -512)) == "E_SHAPE" and read(lay=(1 << 62, 128, 512)) == "E_SHAPE"
    assert read(slots=[-1]) == "E_PARAM" and read(slots=None) == "E_NULL"
    assert L.starkv_pages_read(r, one, 1, ints([0]), None, None, ctypes.byref(LAY), None) == 0
    assert L.starkv_pages_read(r, None, 0, None, None, None, None, None) == 0


@pytest.mark.parametrize("c", [cache(), fp4()])
def test_mass_arguments(c):
    L, r = pg.lib(), ctypes.byref(c)

    def add(slots=(1,), rows=(900,), q=FAKE, lse=FAKE, w=0, s=0, max_len=5000, mass=FAKE, out=FAKE, ws=FAKE,
            wb=BIG):
        return name(L.starkv_mass_add(r, ints(slots), len(slots) if slots else 1, ints(rows), q, lse, w, s,
                                      max_len, mass, out, ws, wb, None))

    assert add(rows=[-1]) == "E_PARAM" and add(rows=[6401]) == "E_PARAM" and add(rows=None) == "E_NULL"
    assert add(slots=[8]) == "E_PARAM" and add(slots=None) == "E_NULL"
    assert add(slots=[1, 1], rows=[1, 1]) == "E_PARAM"         # their masses change: no slot twice
    for k in ("q", "lse", "mass", "out"):
        assert add(**{k: None}) == "E_NULL"
        assert add(**{k: FAKE + 2}) == "E_ALIGN"
    assert add(q=FAKE + 8) == "E_ALIGN"
    assert add(w=-1) == "E_PARAM" and add(s=-1) == "E_PARAM" and add(w=(1 << 26) + 1) == "E_PARAM"
    assert add(max_len=0) == "E_PARAM" and add(max_len=(1 << 26) + 1) == "E_PARAM"
    one_layer = ctypes.byref(cache(n_layers=1))
    need = L.starkv_mass_workspace_bytes(one_layer, ints([900]), 1, 5000)
    assert need > 0 and L.starkv_mass_workspace_bytes(one_layer, ints([1]), 1, 5000) == 0
    r = one_layer
    assert add(ws=None) == "E_WORKSPACE" and add(wb=need - 1) == "E_WORKSPACE" and add(ws=FAKE + 8) == "E_ALIGN"
    assert L.starkv_mass_workspace_bytes(r, ints([900]), 1, 0) == 0
    assert L.starkv_mass_workspace_bytes(r, None, 1, 5000) == 0
    assert L.starkv_mass_add(r, ints([1]), 1, ints([0]), None, None, 0, 0, 1, None, None, None, 0, None) == 0
    assert L.starkv_mass_add(r, None, 0, None, None, None, 0, 0, 1, None, None, None, 0, None) == 0
    # rows of a group beyond 2^30
    wide = ctypes.byref(cache(H=4096, G=1, max_pages=1 << 20))
    assert name(L.starkv_mass_add(wide, ints([1]), 1, ints([(1 << 18) + 1]), FAKE, FAKE, 0, 0, 64, FAKE, FAKE,
                                  FAKE, BIG, None)) == "E_PARAM"


def test_mass_fork_arguments():
    L, r = pg.lib(), ctypes.byref(cache())
    fork = lambda a, b, m=FAKE: name(L.starkv_mass_fork(r, ints(a), ints(b), len(b), m, None))
    assert fork([1], [1]) == "E_PARAM" and fork([1, 2], [2, 3]) == "E_PARAM" and fork([1, 2], [3, 3]) == "E_PARAM"
    assert fork([9], [3]) == "E_PARAM" and fork([1], [2], None) == "E_NULL" and fork([1], [2], FAKE + 2) == "E_ALIGN"
    assert L.starkv_mass_fork(r, None, None, 0, None, None) == 0


@pytest.mark.parametrize("c", [cache(), fp4()])
def test_evict_arguments(c):
    L, r = pg.lib(), ctypes.byref(c)

    def evict(slots=(1, 2), mass=FAKE, keep=10, sinks=4, recent=8, idx=FAKE, status=FAKE, ws=FAKE, wb=BIG):
        return name(L.starkv_pages_evict(r, ints(slots), len(slots) if slots else 1, mass, keep, sinks, recent,
                                         idx, status, ws, wb, None))

    assert evict(slots=[3, 3]) == "E_PARAM" and evict(slots=[8]) == "E_PARAM" and evict(slots=None) == "E_NULL"
    for k in ("keep", "sinks", "recent"):
        assert evict(**{k: -1}) == "E_BUDGET" and evict(**{k: 1 << 26}) == "E_BUDGET"
    for k in ("mass", "idx", "status"):
        assert evict(**{k: None}) == "E_NULL" and evict(**{k: FAKE + 2}) == "E_ALIGN"
    need = L.starkv_evict_workspace_bytes(r, 2, 10, 4, 8)
    assert need >= L.starkv_pages_workspace_bytes(r, 2, 22) + 28 * 2 * 22 * 4
    assert evict(ws=None) == "E_WORKSPACE" and evict(wb=need - 1) == "E_WORKSPACE" and evict(ws=FAKE + 8) == "E_ALIGN"
    assert L.starkv_evict_workspace_bytes(r, 257, 1, 1, 1) == 0 and L.starkv_evict_workspace_bytes(r, 1, -1, 1, 1) == 0
    assert L.starkv_evict_workspace_bytes(r, 1, 1 << 26, 1, 1) == 0
    assert L.starkv_pages_evict(r, None, 0, None, 1, 1, 1, None, None, None, 0, None) == 0


def test_the_binding_refuses_host_tensors():
    k = torch.zeros(1, 4, 2, pg.fp4_block_bytes(16, 64), dtype=torch.uint8)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        pg.Cache(k, k.clone(), i(2, 3), i(2), i(4), 4, 64)
    with pytest.raises(ValueError, match="d: None"):
        pg.Cache(k, k.clone(), i(2, 3), i(2), i(4), 4)
    with pytest.raises(ValueError, match="d: 64, rows of 128"):
        b = torch.zeros(1, 4, 2, 16, 128, dtype=torch.bfloat16)
        pg.Cache(b, b.clone(), i(2, 3), i(2), i(4), 4, 64)
