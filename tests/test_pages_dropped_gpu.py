"""Dropped tokens stay dropped when a sequence is compacted: no row of zeros
takes their place where attention would see it."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_pages_gpu import Both  # noqa: E402

pytestmark = pytest.mark.gpu


def none(n=1, B=0):
    return np.zeros((1, n, B), dtype=np.int32)


@pytest.mark.parametrize("dtype,d,P", [("bf16", 64, 16), ("f32", 128, 32)])
def test_a_tail_of_dropped_tokens(dtype, d, P):
    """The window keeps the last tokens; a longer tail, by one page or by
    many, is refused, one that ends at the first kept page is not."""
    b = Both(P=P, d=d, dtype=dtype, n_pages=64, max_pages=12)
    n = 8 * P + 5
    for keep in (5, 6, 2 * P + 5):             # the last page, two, three of the sequence
        b.grow([0, 1], [n, n])
        b.write([0, 1], [n, n])
        b.free([0], first=3, last=keep)        # slot 1 keeps all
        there = 5 + -(-(keep - 5) // P) * P    # tokens behind the last dropped page
        for tail in (there + 1, there + P, 3 * P, 3 * P + 1, 5 * P, n - P - 1):
            if there < tail:
                assert list(b.compact([0], none(), tail=tail)) == [2]
        # among others, and with tokens picked before it
        assert list(b.compact([1, 0], none(2, 2), tail=there + 1)) == [0, 2]
        assert list(b.compact([0], none(1, 2), tail=there)) == [0]
        b.free([0, 1])


@pytest.mark.parametrize("tail", [48, 49, 300, 1030])
def test_tails_of_many_pages_and_sequences(tail):
    """40 sequences, one dropped page in each at another place, before the
    tail or in it."""
    b = Both(nl=1, G=1, H=1, n_pages=4000, n_slots=40, max_pages=90)
    slots = [int(x) for x in np.random.default_rng(9).permutation(40)]
    lens = [70 * 16 + i % 16 for i in range(20)] + [20 * 16 + i for i in range(20)]
    b.grow(slots, lens)
    for i, s in enumerate(slots):              # page 3, or the one i pages before the last
        j = 3 if i % 3 else (lens[i] - 1) // 16 - i
        if j >= 0:
            b.m.refs[b.m.table[s, j]] -= 1
            b.m.table[s, j] = -1
    b.c.table.copy_(torch.from_numpy(b.m.table))
    b.c.refs.copy_(torch.from_numpy(b.m.refs))
    want = b.compact(slots, none(40), tail=tail)
    assert {int(x) for x in want} == {0, 2}


def test_a_tail_longer_than_the_span():
    b = Both(n_pages=40, max_pages=20)
    b.grow([0], [200])
    b.free([0], first=1, last=90)
    assert list(b.compact([0], none(), tail=105, span=[120])) == [2]   # of dropped tokens
    assert list(b.compact([0], none(), tail=50, span=[40])) == [2]     # past the span
    assert list(b.compact([0], none(), tail=60, span=[70])) == [0]
