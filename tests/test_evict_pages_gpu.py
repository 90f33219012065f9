"""How many free pages an eviction takes: as many as the header says, of the whole call
before any page is let go; with those of one sequence, one sequence at a time."""

import pytest

torch = pytest.importorskip("torch")

from oracle import evict_oracle as EO  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from test_evict_gpu import Both  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp4"])
@pytest.mark.parametrize("keep,sinks,recent", [(40, 4, 8), (16, 0, 0), (45, 0, 3), (44, 4, 1), (0, 0, 32)])
def test_the_pages_of_a_call(dtype, keep, sinks, recent):
    lens, P = [200, 180, 20, 160], 16               # 20: longer than one budget, short for the others
    need = -(-(keep + sinks + recent) // P)
    longer = [n > keep + sinks + recent for n in lens]
    want = [PO.OK if x else EO.SHORT for x in longer]
    last = max(i for i, x in enumerate(longer) if x)
    b = Both(3, lens, P=P, spare=need * sum(longer), dtype=dtype).upload()
    assert list(b.evict(b.slots, keep, sinks, recent, "enough")) == want
    b = Both(3, lens, P=P, spare=need * sum(longer) - 1, dtype=dtype).upload()
    assert list(b.evict(b.slots, keep, sinks, recent, "one less")) == want[:last] + [PO.NO_PAGES] + want[last + 1:]
    # those of one sequence: one after the other
    b = Both(3, lens, P=P, spare=need, dtype=dtype).upload()
    got = [b.evict([s], keep, sinks, recent, "one at a time")[0] for s in b.slots]
    assert list(got) == want


def test_a_full_pool_evicts_nothing():
    b = Both(4, [200, 180], spare=0).upload()
    assert list(b.evict(b.slots, 40, 4, 8)) == [PO.NO_PAGES] * 2
    # what needs no page is let go all the same, and makes room
    assert list(b.evict(b.slots[:1], 0, 0, 0)) == [PO.OK]
    assert list(b.evict(b.slots[1:], 40, 4, 8)) == [PO.OK]
