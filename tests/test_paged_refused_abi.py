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
