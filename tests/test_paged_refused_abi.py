"""The page calls that follow a grow's status, on the CPU: refusals, and the
host model of a sequence that a grow left unchanged."""

import ctypes
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402
from paper_2606_01790_amd import starkv as sk  # noqa: E402
from test_paged_abi import FAKE, cache, ints, name, small  # noqa: E402

built = pytest.mark.skipif(not os.path.exists(sk.LIB_PATH), reason="libstarkv.so not built")


@built
def test_write_grown_arguments():
    L = pg.lib()

    def write(c=None, slots=(1,), rows=(2,), k=FAKE, v=FAKE, lay=(0, 128, 512), grown=FAKE):
        lay = ctypes.byref(sk.KVLayout(*lay)) if lay else None
        return name(L.starkv_pages_write_grown(ctypes.byref(c or cache()), ints(slots), len(slots),
                                               ints(rows), k, v, lay, grown, None))

    assert write(grown=None) == "E_NULL"
    assert write(grown=FAKE + 2) == "E_ALIGN"
    assert write(c=cache(dtype=2)) == "E_DTYPE"
    assert write(slots=[1, 1], rows=[1, 1]) == "E_PARAM" and write(slots=[8]) == "E_PARAM"
    assert write(rows=[-1]) == "E_PARAM" and write(rows=None) == "E_NULL"
    assert write(k=None) == "E_NULL" and write(lay=None) == "E_NULL"
    assert write(v=FAKE + 4) == "E_ALIGN" and write(lay=(0, 4, 512)) == "E_ALIGN"
    assert write(lay=(0, 128, -512)) == "E_SHAPE"
    # nothing to write
    assert write(rows=[0], k=None, v=None) == "OK"
    assert L.starkv_pages_write_grown(ctypes.byref(cache()), None, 0, None, None, None, None, None,
                                      None) == 0


def test_model_keeps_what_a_failed_grow_left():
    m = small()
    m.grow([1], [18])
    rows = np.arange(36, dtype=np.int32).reshape(1, 18, 1, 2) + 1
    m.write([1], [18], rows, -rows)
    k0 = m.k.copy()
    st = m.grow([1, 0], [3, 2])
    assert list(st) == [PO.RANGE, PO.OK]
    new = np.full((1, 5, 1, 2), 99, dtype=np.int32)
    m.write([1, 0], [3, 2], new, new, st)
    mine = m.table[1, :5]
    assert np.array_equal(m.k[:, mine], k0[:, mine])
    assert (m.k[0, m.table[0, 0], 0, :2] == 99).all()
    # without the status its last three tokens are written over
    m.write([1], [3], new[:, :3], new[:, :3])
    assert (m.k[0, m.at(1, 17)[0], 0, m.at(1, 17)[1]] == 99).all()


@built
def test_compact_grown_arguments():
    L = pg.lib()

    def compact(c=None, slots=(1,), span=(8,), idx=FAKE, ls=0, B=4, counts=None, tail=0, grown=FAKE,
                status=FAKE, ws=FAKE, wb=1 << 40):
        return name(L.starkv_pages_compact_grown(ctypes.byref(c or cache()), ints(slots), len(slots),
                                                 ints(span), idx, ls, B, counts, tail, grown, status,
                                                 ws, wb, None))

    assert compact(grown=None) == "E_NULL"
    assert compact(grown=FAKE + 2) == "E_ALIGN"
    assert compact(c=cache(d=96)) == "E_SHAPE"
    assert compact(slots=[1, 1], span=[1, 1]) == "E_PARAM" and compact(span=[-1]) == "E_PARAM"
    assert compact(idx=None) == "E_NULL" and compact(status=None) == "E_NULL"
    assert compact(B=-1) == "E_BUDGET" and compact(ls=-1) == "E_SHAPE"
    assert compact(ws=None) == "E_WORKSPACE" and compact(ws=FAKE + 8) == "E_ALIGN"
    assert L.starkv_pages_compact_grown(ctypes.byref(cache()), None, 0, None, None, 0, 0, None, 0, None,
                                        None, None, 0, None) == 0


def test_model_compacts_no_older_tokens():
    m = small()
    m.grow([1, 0], [18, 2])
    rows = np.arange(36, dtype=np.int32).reshape(1, 18, 1, 2) + 1
    m.write([1], [18], rows, -rows)
    k0, row = m.k.copy(), m.table[1].copy()
    st = m.grow([1, 0], [3, 1])
    assert list(st) == [PO.RANGE, PO.OK]
    idx = np.array([[[0], [0]]], dtype=np.int32)
    assert list(m.compact([1, 0], idx, span=[3, 1], grown=st)) == [PO.RANGE, PO.NO_PAGES]
    assert m.len[1] == 18 and np.array_equal(m.table[1], row)
    assert np.array_equal(m.k[:, row], k0[:, row])
    m.free([0])
    assert list(m.compact([1], idx[:, :1], span=[3])) == [PO.OK]
    assert m.len[1] == 16          # without the status, two older tokens are gone


def test_model_keeps_no_dropped_tail():
    m = small(12)
    m.grow([0], [18])
    m.free([0], 1, 5)                # page 0 and the last two
    assert list(m.table[0] >= 0) == [True, False, False, True, True]
    idx = np.zeros((1, 1, 0), dtype=np.int32)
    assert list(m.compact([0], idx, tail=7)) == [PO.RANGE] and m.len[0] == 18
    assert list(m.compact([0], idx, tail=6)) == [PO.OK] and m.len[0] == 6
