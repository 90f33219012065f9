"""The reference of 4-bit rows, accumulated weights and eviction against closed
forms (no GPU)."""

import numpy as np
import pytest

from oracle import evict_oracle as EO
from oracle import paged_oracle as PO


def test_quantiser_on_its_grid():
    # every value of the grid comes back, at any power of two
    row = np.zeros(64)
    row[:16] = list(EO.GRID) + [-g for g in EO.GRID]
    for e in (-125, -3, 0, 7, 125):
        q = EO.fp4_quantise(row * 2.0 ** e)
        assert q[32] == e + 127 and np.array_equal(EO.fp4_numbers(q)[:16], row[:16] * 2.0 ** e)
    assert EO.fp4_quantise(row)[0] == 0x10 and EO.fp4_quantise(row)[3] == 0x76 and EO.fp4_quantise(row)[4] == 0x98


@pytest.mark.parametrize("x,want", [(0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2), (3.5, 4), (5, 4),
                                    (5.01, 6), (6.9, 6), (-0.75, -1), (0.2501, 0.5)])
def test_ties_go_to_even_codes(x, want):
    row = np.zeros(64)
    row[0], row[1], row[40] = 7.0, x, 1.0
    got = EO.fp4_numbers(EO.fp4_quantise(row))
    assert got[0] == 6 and got[1] == want and got[40] == 1


def test_scales():
    byte = lambda top: EO.fp4_quantise(np.array([top] + [0.0] * 63))[32]
    assert byte(7.0) == 127 and byte(7.0001) == 128 and byte(3.5) == 126 and byte(3.51) == 127
    assert byte(0.0) == 2 and byte(1e-45) == 2 and byte(3.3e38) == 252
    bad = EO.fp4_quantise(np.array([np.inf] + [1.0] * 63))
    assert bad[32] == 255 and np.isnan(EO.fp4_numbers(bad)[:32]).all() and (EO.fp4_numbers(bad)[32:] == 1).all()
    assert np.isnan(EO.fp4_numbers(EO.fp4_quantise(np.array([1.0] * 63 + [np.nan])))[32:]).all()


def test_the_nearest_value_is_taken():
    r = np.random.default_rng(0)
    x = r.standard_normal((20, 64)) * 2.0 ** r.integers(-20, 20, (20, 1))
    rows = EO.fp4_quantise(x)
    got = EO.fp4_numbers(rows)
    s = 2.0 ** (rows[:, 32:].astype(float) - 127)
    grid = np.concatenate([EO.GRID, [-g for g in EO.GRID]])
    best = np.min(np.abs(x[..., None] - grid * np.repeat(s, 32, 1)[..., None]), -1)
    assert np.array_equal(np.abs(got - x), best)


def model(n, P=4, nl=1):
    z = np.zeros((nl, 12, 1, P, 2))
    m = PO.PagedModel(z, z.copy(), 2, 8)
    m.grow([0], [n])
    for t in range(n):
        p, r = m.at(0, t)
        m.k[:, p, 0, r], m.v[:, p, 0, r] = t, -t
    return m


def test_weights_of_equal_logits():
    """Zero queries: every seen token weighs 1 / seen, each row adds 1 a head."""
    m = model(6)
    q = np.zeros((2, 3, 2))
    see = PO.see_window(6, 2, 3, 1)
    _, lse, _, _ = PO.attend(m, 0, q, see, lambda x: x, 0)
    add, _ = EO.weights(m, 0, q, lse, see, lambda x: x, 0)
    assert np.allclose(add, 3 * np.array([0.25 + 0.25, 0, 0.25, 0.5, 0.5, 0.25])) and np.isclose(add.sum(), 6)
    lse[0] = -np.inf
    assert np.isclose(EO.weights(m, 0, q, lse, see, lambda x: x, 0)[0].sum(), 3)


def test_evicts_the_lightest():
    m = model(12, nl=2)
    mass = np.zeros((2, 2, 32), dtype=np.float32)
    mass[0, 0, :12] = [0, 9, 1, 5, 5, 5, np.nan, 2, 8, 0, 7, 7]
    mass[1, 0, :12] = np.arange(12)
    idx, st = EO.evict(m, [0, 1], mass, 3, 2, 2)
    assert list(st) == [EO.OK, EO.SHORT]
    # sinks 0 1; of 2..9 the NaN, the 8 and the first 5; recent 10 11
    assert list(idx[0, 0]) == [0, 1, 3, 6, 8] and list(idx[1, 0]) == [0, 1, 7, 8, 9] and (idx[:, 1] == -1).all()
    assert m.len[0] == 7 and m.refs.sum() == 2
    rows = lambda l: [m.k[l, m.at(0, t)[0], 0, m.at(0, t)[1], 0] for t in range(7)]
    assert rows(0) == [0, 1, 3, 6, 8, 10, 11] and rows(1) == [0, 1, 7, 8, 9, 10, 11]
    assert np.array_equal(mass[0, 0, :7], [0, 9, 5, np.nan, 8, 7, 7], equal_nan=True)
    assert list(mass[1, 0, :7]) == [0, 1, 7, 8, 9, 10, 11]


def test_eviction_passes_over_dropped_tokens():
    m = model(12)
    mass = np.zeros((1, 2, 32), dtype=np.float32)
    mass[0, 0, :12] = np.arange(12) + 1
    m._let_go(0, [1])                       # tokens 4..7
    idx, st = EO.evict(m, [0], mass, 5, 2, 2)
    assert list(idx[0, 0]) == [0, 1, 2, 3, 8, 9, -1] and st[0] == EO.OK and m.len[0] == 8
    m = model(12)
    m._let_go(0, [2])                       # of the recent ones
    assert list(EO.evict(m, [0], mass, 2, 1, 3)[1]) == [PO.RANGE] and m.len[0] == 12


def test_blocks_of_a_pool():
    pool = np.arange(2 * 3 * 34, dtype=np.uint8).reshape(1, 1, 2, 3, 34)
    blk = EO.fp4_blocks(pool)
    assert blk.shape == (1, 1, 2, 102)
    assert list(blk[0, 0, 0, 32:64]) == list(pool[0, 0, 0, 1, :32]) and list(blk[0, 0, 0, 96:98]) == list(pool[0, 0, 0, 0, 32:])
