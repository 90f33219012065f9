"""Views of a cache's layers, on the CPU: a view of layers that are not there
is refused, where slicing would give fewer, and the calls on it would leave
the rest of a caller's outputs as they were."""

from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

from paper_2606_01790_amd import paged as pg  # noqa: E402


@pytest.mark.parametrize("first,count", [(3, 1), (2, 2), (0, 4), (-1, 1), (-4, 2), (0, 0), (1, -1)])
def test_layers_that_are_not_there(first, count):
    c = SimpleNamespace(k=torch.zeros(3, 2, 1, 16, 64), n_layers=3)
    with pytest.raises(ValueError, match="layers"):
        pg.Cache.layers(c, first, count)
