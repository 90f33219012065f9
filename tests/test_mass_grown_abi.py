"""starkv_mass_add_grown on the CPU: it refuses what starkv_mass_add refuses, and a
status that is missing or lies askew, before any GPU work."""

import ctypes

import pytest

from paper_2606_01790_amd import starkv as sk

torch = pytest.importorskip("torch")

import os  # noqa: E402

from paper_2606_01790_amd import paged as pg  # noqa: E402
from test_evict_abi import BIG, FAKE, cache, fp4, ints, name  # noqa: E402

pytestmark = pytest.mark.skipif(not os.path.exists(sk.LIB_PATH),
                                reason="libstarkv.so not built")


@pytest.mark.parametrize("c", [cache(n_layers=1), fp4(n_layers=1)])
def test_arguments(c):
    L, r = pg.lib(), ctypes.byref(c)

    def add(slots=(1,), rows=(900,), q=FAKE, lse=FAKE, w=0, s=0, max_len=5000, mass=FAKE, out=FAKE, grown=FAKE,
            ws=FAKE, wb=BIG):
        return name(L.starkv_mass_add_grown(r, ints(slots), len(slots) if slots else 1, ints(rows), q, lse, w, s,
                                            max_len, mass, out, grown, ws, wb, None))

    for k in ("q", "lse", "mass", "out", "grown"):
        assert add(**{k: None}) == "E_NULL"
        assert add(**{k: FAKE + 2}) == "E_ALIGN"
    assert add(rows=[-1]) == "E_PARAM" and add(rows=[6401]) == "E_PARAM" and add(rows=None) == "E_NULL"
    assert add(slots=[8]) == "E_PARAM" and add(slots=None) == "E_NULL"
    assert add(slots=[1, 1], rows=[1, 1]) == "E_PARAM"
    assert add(w=-1) == "E_PARAM" and add(s=-1) == "E_PARAM" and add(max_len=0) == "E_PARAM"
    need = L.starkv_mass_workspace_bytes(r, ints([900]), 1, 5000)
    assert need > 0 and add(ws=None) == "E_WORKSPACE" and add(wb=need - 1) == "E_WORKSPACE"
    assert add(ws=FAKE + 8) == "E_ALIGN"
    # no rows, no sequences: nothing to do
    assert L.starkv_mass_add_grown(r, ints([1]), 1, ints([0]), None, None, 0, 0, 1, None, None, FAKE, None, 0,
                                   None) == 0
    assert L.starkv_mass_add_grown(r, None, 0, None, None, None, 0, 0, 1, None, None, None, None, 0, None) == 0
