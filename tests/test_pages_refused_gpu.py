"""What the page calls cannot do leaves a sequence as it is, and so do the calls
behind it that are given the status: against the host model, bit for bit."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_01790_amd import paged as pg  # noqa: E402
from test_pages_gpu import TYPE, Both, say  # noqa: E402

pytestmark = pytest.mark.gpu


def write_grown(b, slots, rows, status, grown):
    """The device's status and the model's, of the same grow."""
    say(f"write {slots} {rows} behind {list(grown)}")
    k, v = b.rows(sum(rows)), b.rows(sum(rows))
    dev = lambda x: torch.from_numpy(x).cuda().view(TYPE[b.dtype])
    kd = dev(k)
    pg.pages_write(b.c, slots, rows, kd, dev(v), pg.rows_layout(kd), grown=status)
    b.m.write(slots, rows, k, v, grown)
    b.check("write")


@pytest.mark.parametrize("dtype,d,P,order", [("bf16", 64, 16, "plain"), ("bf16", 128, 64, "groups"),
                                             ("f32", 64, 32, "padded"), ("f32", 128, 16, "plain")])
def test_a_write_behind_a_grow_that_failed(dtype, d, P, order):
    """Too few pages, past the table row, and a sequence that grows between
    them: only its rows are written, the others keep every older one."""
    b = Both(P=P, d=d, dtype=dtype, order=order, n_pages=7, max_pages=3)
    b.grow([0, 1, 2], [P + 5, P, 2 * P + 1])
    b.write([0, 1, 2], [P + 5, P, 2 * P + 1])
    before = b.m.k.copy()
    want = b.grow([2, 1, 0], [P, 2, P])
    assert list(want) == [2, 0, 1]
    write_grown(b, [2, 1, 0], [P, 2, P], b.st, want)
    own = b.m.table[1, 1]
    others = [p for p in range(7) if p != own]
    assert np.array_equal(b.m.k[:, others], before[:, others])
    assert not np.array_equal(b.m.k[:, own], before[:, own])
    # all of a list refused, and none
    want = b.grow([0, 2], [P + 1, P])
    assert list(want) == [1, 2]
    write_grown(b, [0, 2], [P + 1, P], b.st, want)
    want = b.grow([0, 1], [1, 1])
    assert list(want) == [0, 0]
    write_grown(b, [0, 1], [1, 1], b.st, want)


def test_a_write_of_many_sequences_behind_a_grow_that_failed():
    """More sequences than the short lists hold, every third past its row."""
    b = Both(nl=1, G=2, n_pages=100, n_slots=40, max_pages=2)
    slots = [int(x) for x in np.random.default_rng(2).permutation(40)]
    b.grow(slots, [20] * 40)
    b.write(slots, [20] * 40)
    add = [30 if i % 3 == 0 else 1 + i % 12 for i in range(40)]
    want = b.grow(slots, add)
    assert [int(x) for x in want] == [2 if i % 3 == 0 else 0 for i in range(40)]
    write_grown(b, slots, add, b.st, want)


def test_replays_that_run_out_of_pages():
    """A captured step of grow and write, replayed past the pool's end with
    eager work between: the sequences stay as they were when it ended, and go
    on when there are pages again."""
    b = Both(n_pages=6, max_pages=8)
    b.grow([0, 3], [16, 30])
    b.write([0, 3], [16, 30])
    k, v = b.rows(14), b.rows(14)
    kd = torch.from_numpy(k).cuda().view(TYPE["bf16"])
    vd = torch.from_numpy(v).cuda().view(TYPE["bf16"])
    st = torch.zeros(2, dtype=torch.int32, device="cuda")

    def step():
        pg.pages_grow(b.c, [0, 3], [7, 7], st, b.ws)
        pg.pages_write(b.c, [0, 3], [7, 7], kd, vd, pg.rows_layout(kd), grown=st)

    def model():
        want = b.m.grow([0, 3], [7, 7])
        b.m.write([0, 3], [7, 7], k, v, want)
        return [int(x) for x in want]

    step()
    seen = [model()]
    b.check("eager")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(9):
        if i == 6:
            b.free([0], 8)            # eager work: pages again
        graph.replay()
        seen.append(model())
        b.check(f"replay {i}")
        assert st.tolist() == seen[-1]
    assert [1, 1] in seen and [0, 1] in seen and seen[-1] != [1, 1]


def test_the_binding_refuses_a_status_of_another_kind():
    b = Both()
    b.grow([0, 1], [3, 3])
    k = torch.zeros(2, 6, 2, 64, dtype=torch.bfloat16, device="cuda")
    write = lambda grown: pg.pages_write(b.c, [0, 1], [3, 3], k, k, pg.rows_layout(k), grown=grown)
    for bad, what in ((torch.zeros(2, dtype=torch.int64, device="cuda"), "grown: torch.int64"),
                      (torch.zeros(1, dtype=torch.int32, device="cuda"), "grown: 2"),
                      (torch.zeros(2, dtype=torch.int32), "device tensor")):
        with pytest.raises(ValueError, match=what):
            write(bad)


def compact_grown(b, slots, idx, grown, tail=0, span=None, counts=None, own=False):
    """`own`: the status goes where the grow's is, as one buffer for both."""
    say(f"compact {slots} behind {list(grown)}")
    cd = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    before = b.st
    out = before if own else b.status(len(slots))
    pg.pages_compact(b.c, slots, torch.from_numpy(idx).cuda(), out, b.ws, tail=tail, span=span,
                     counts=cd, grown=before)
    want = b.m.compact(slots, idx, tail, span, counts, grown)
    b.check("compact")
    b.same_status("compact", want)
    return want


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("dtype,d,P", [("bf16", 128, 16), ("f32", 64, 32)])
def test_a_compaction_behind_a_grow_that_failed(dtype, d, P, own):
    """The end of a speculative step whose draft found no pages: the tokens
    that were there stay, in the pages where they were; the others' paths are
    cut."""
    b = Both(P=P, d=d, dtype=dtype, n_pages=12, max_pages=4)
    lens = [P + 5, P - 2, 3 * P + 1, 9]
    b.grow([0, 1, 2, 3], lens)
    b.write([0, 1, 2, 3], lens)
    row = b.m.table[[2, 0]].copy()
    slots, add = [2, 1, 0, 3], [P, 6, 2 * P, 4]
    b.grow([4], [2 * P])                  # the pool is nearly taken
    want = b.grow(slots, add)
    assert list(want) == [2, 0, 1, 0]
    b.st = b.st[:4].contiguous() if own else b.st
    st = b.st
    write_grown(b, slots, add, st, want)
    b.free([4])                           # pages again, for the fresh ones of the compaction
    idx = np.array([[[0, 2, 5, 6], [0, 1, 3, 5], [1, 2, 4, 9], [3, 2, 1, 0]]], dtype=np.int32)
    got = compact_grown(b, slots, idx, want, span=add, counts=[4, 3, 2, 4], own=own)
    assert list(got) == [2, 0, 1, 0]
    assert np.array_equal(b.m.table[[2, 0]], row)
    assert list(b.m.len[:4]) == [lens[0], P - 2 + 3, lens[2], 9 + 4]


def test_a_compaction_that_follows_a_grow_refuses_for_itself():
    """Behind a grow that went well the call's own refusals are as ever."""
    b = Both(n_pages=8)
    b.grow([0, 1], [20, 40])
    b.write([0, 1], [20, 40])
    want = b.grow([1, 0], [2, 5])
    idx = np.zeros((1, 2, 1), dtype=np.int32)
    assert list(compact_grown(b, [1, 0], idx, want, tail=3, span=[2, 5])) == [2, 0]


def test_the_binding_refuses_a_compaction_with_a_status_of_another_kind():
    b = Both()
    b.grow([0, 1], [3, 3])
    idx = torch.zeros(1, 2, 1, dtype=torch.int32, device="cuda")
    for bad, what in ((torch.zeros(2, dtype=torch.int64, device="cuda"), "grown: torch.int64"),
                      (torch.zeros(1, dtype=torch.int32, device="cuda"), "grown: 2"),
                      (torch.zeros(2, dtype=torch.int32), "device tensor")):
        with pytest.raises(ValueError, match=what):
            pg.pages_compact(b.c, [0, 1], idx, b.st, b.ws, span=[1, 1], grown=bad)
