"""The pages of a cache on the GPU against the host model of
oracle/paged_oracle.py: after every call the table, the lengths, the reference
counts, the status and every bit of the pool are equal.  The pools start full
of NaN, so a row that should not be read shows."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402

pytestmark = pytest.mark.gpu

NAN = {"bf16": 0x7FC1, "f32": 0x7FC00001}
BITS = {"bf16": torch.int16, "f32": torch.int32}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
NP = {"bf16": np.int16, "f32": np.int32}


def say(msg):
    print(f"[pages] {msg}", flush=True)


class Both:
    """A cache on the GPU and its host model, changed in step."""

    def __init__(self, nl=2, G=2, H=4, P=16, d=64, n_pages=24, n_slots=6, max_pages=8, dtype="bf16",
                 order="plain"):
        self.dtype = dtype
        shape = (nl, n_pages, G, P, d)
        pool = np.full(shape, NAN[dtype], dtype=NP[dtype])
        self.m = PO.PagedModel(pool, pool.copy(), n_slots, max_pages)
        if order == "plain":
            mk = lambda: torch.full(shape, NAN[dtype], dtype=BITS[dtype], device="cuda")
        elif order == "padded":      # rows of d + 8 elements
            mk = lambda: torch.full((*shape[:4], d + 8), NAN[dtype], dtype=BITS[dtype],
                                    device="cuda")[..., :d]
        else:                        # the group outermost, the layer inside the page
            mk = lambda: torch.full((G, n_pages, nl, P, d), NAN[dtype], dtype=BITS[dtype],
                                    device="cuda").permute(2, 1, 0, 3, 4)
        self.k, self.v = mk(), mk()
        i32 = dict(dtype=torch.int32, device="cuda")
        # tables with content that init has to clear
        self.c = pg.Cache(self.k.view(TYPE[dtype]), self.v.view(TYPE[dtype]),
                          torch.full((n_slots, max_pages), 7, **i32), torch.full((n_slots,), 9, **i32),
                          torch.full((n_pages,), 5, **i32), H)
        pg.pages_init(self.c)
        self.ws = torch.empty(pg.pages_workspace_bytes(self.c, n_slots, 4 * self.c.cap),
                              dtype=torch.uint8, device="cuda")
        self.rng = np.random.default_rng(nl * 1000 + n_pages)
        self.check("init")

    def check(self, tag):
        torch.cuda.synchronize()
        assert np.array_equal(self.c.table.cpu().numpy(), self.m.table), f"{tag}: table"
        assert np.array_equal(self.c.length.cpu().numpy(), self.m.len), f"{tag}: length"
        assert np.array_equal(self.c.refs.cpu().numpy(), self.m.refs), f"{tag}: refs"
        assert np.array_equal(self.k.cpu().numpy(), self.m.k), f"{tag}: k"
        assert np.array_equal(self.v.cpu().numpy(), self.m.v), f"{tag}: v"
        # every count is the number of entries that name the page
        have = self.m.table[(self.m.table >= 0) & (self.m.table < self.m.n_pages)]
        assert np.array_equal(np.bincount(have, minlength=self.m.n_pages), self.m.refs), tag

    def status(self, n):
        self.st = torch.full((n + 2,), 77, dtype=torch.int32, device="cuda")
        return self.st

    def same_status(self, tag, want):
        got = self.st.cpu().numpy()
        assert np.array_equal(got[:len(want)], want), f"{tag}: status {got} {want}"
        assert (got[len(want):] == 77).all(), f"{tag}: status behind the last sequence"

    def grow(self, slots, add):
        say(f"grow {slots} {add}")
        pg.pages_grow(self.c, slots, add, self.status(len(slots)), self.ws)
        want = self.m.grow(slots, add)
        self.check("grow")
        self.same_status("grow", want)
        return want

    def rows(self, tot):
        c = self.c
        hi = 2 ** 15 if self.dtype == "bf16" else 2 ** 31
        return self.rng.integers(-hi, hi, (c.n_layers, tot, c.G, c.d)).astype(NP[self.dtype])

    def write(self, slots, rows):
        say(f"write {slots} {rows}")
        k, v = self.rows(sum(rows)), self.rows(sum(rows))
        dev = lambda x: torch.from_numpy(x).cuda().view(TYPE[self.dtype])
        kd = dev(k)
        pg.pages_write(self.c, slots, rows, kd, dev(v), pg.rows_layout(kd))
        self.m.write(slots, rows, k, v)
        self.check("write")

    def fork(self, src, dst):
        say(f"fork {src} {dst}")
        pg.pages_fork(self.c, src, dst)
        self.m.fork(src, dst)
        self.check("fork")

    def free(self, slots, first=0, last=0):
        say(f"free {slots} {first} {last}")
        pg.pages_free(self.c, slots, first, last)
        self.m.free(slots, first, last)
        self.check("free")

    def compact(self, slots, idx, tail=0, span=None, counts=None):
        say(f"compact {slots} {idx.shape} tail {tail} span {span} counts {counts}")
        cd = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        pg.pages_compact(self.c, slots, torch.from_numpy(idx).cuda(), self.status(len(slots)),
                         self.ws, tail=tail, span=span, counts=cd)
        want = self.m.compact(slots, idx, tail, span, counts)
        self.check("compact")
        self.same_status("compact", want)
        return want


@pytest.mark.parametrize("dtype,d,P,order", [("bf16", 64, 16, "plain"), ("bf16", 128, 64, "groups"),
                                             ("f32", 64, 32, "padded"), ("f32", 128, 16, "plain")])
def test_a_life_of_three_sequences(dtype, d, P, order):
    """Grown from nothing by one token, to a page's edge, past it; forked;
    both holders written on (each gets its copy of the shared part); trimmed
    to a window, ended, and their pages taken again."""
    b = Both(P=P, d=d, dtype=dtype, order=order)
    b.grow([2], [1])
    b.write([2], [1])
    b.grow([2, 0], [P - 1, P])
    b.write([2, 0], [P - 1, P])
    b.grow([2, 0], [3, 2 * P + 1])
    b.write([2, 0], [3, 2 * P + 1])
    b.fork([2, 0, 2], [5, 1, 3])
    b.write([3], [2])                     # a shared page: nothing is written
    b.grow([2, 5, 1], [1, 2, P])          # 2 and 5 copy P + 3 tokens' last page; 1 its own
    b.write([5, 1, 2], [2, P, 1])
    b.write([3], [P])                     # 3 alone holds its last page now, not the first
    b.free([0], P + 1, 2)                 # nothing lies between
    b.free([1], 1, 1)
    b.free([5], 5)                        # cut to five tokens
    b.grow([5], [4])
    b.write([5], [4])
    b.free([2, 3])
    b.free([3])                           # an empty sequence
    b.grow([3, 2], [P + 5, 0])
    b.fork([2], [5])                      # an empty fork frees what 5 had


def test_grow_serves_in_order_while_pages_last():
    b = Both(n_pages=5, max_pages=4)
    assert list(b.grow([0, 1, 2, 3], [32, 64, 0, 1])) == [0, 1, 0, 1]   # 2, then 4 of 3
    assert list(b.grow([0, 1], [33, 16])) == [2, 0]                     # past the row of 4 pages
    b.fork([0], [4])
    assert list(b.grow([0, 4, 2], [32, 1, 16])) == [0, 1, 1]            # 2 pages, none left
    b.free([0])
    assert list(b.grow([4], [32])) == [0]


def test_bad_entries_are_no_pages():
    b = Both()
    b.grow([0], [40])
    b.write([0], [40])
    # a caller's own table: entries far outside the pool
    for j, bad in ((0, -5), (2, 1 << 30)):
        b.m.refs[b.m.table[0, j]] -= 1
        b.m.table[0, j] = bad
    b.c.table.copy_(torch.from_numpy(b.m.table))
    b.c.refs.copy_(torch.from_numpy(b.m.refs))
    b.write([0], [40])                    # only the middle page's rows
    b.fork([0], [1])
    assert list(b.grow([1], [1])) == [2]  # its last page is none
    b.compact([0], np.arange(40, dtype=np.int32)[None, None, ::5].copy(), tail=0)
    b.free([0, 1])


def test_no_sequence_goes_on_within_a_dropped_page():
    """Back to a length whose last page the window let go: what was dropped
    stays dropped, so the page's further rows cannot be used."""
    b = Both(n_pages=40)
    for n in (40, 48):                              # within a dropped page, and at its end
        b.grow([0, 1], [100, 100])
        b.write([0, 1], [100, 100])
        b.free([0, 1], first=4, last=30)            # pages 1 to 3
        idx = np.zeros((1, 2, 3), dtype=np.int32)
        bad = 2 if n % 16 else 0
        assert list(b.compact([0, 1], idx, span=[100 - n, 20])) == [bad, 0]
        b.free([0], first=n)
        assert list(b.grow([0, 1], [9, 9])) == [bad, 0]
        assert list(b.grow([0], [0])) == [0]
        assert list(b.compact([0], np.zeros((1, 1, 0), dtype=np.int32), span=[0])) == [0]
        b.free([0, 1])


@pytest.mark.parametrize("dtype,d,P", [("bf16", 128, 16), ("f32", 64, 64), ("bf16", 64, 32),
                                       ("f32", 128, 16)])
def test_compact_selection(dtype, d, P):
    """The stage's form: each layer its own tokens, then the tail; also picked
    twice, out of order and out of range, and a sequence of which nothing stays."""
    b = Both(nl=3, P=P, d=d, dtype=dtype, n_pages=40)
    b.grow([0, 4, 2], [5 * P + 3, P, 2 * P + 1])
    b.write([0, 4, 2], [5 * P + 3, P, 2 * P + 1])
    b.fork([0], [1])
    r = np.random.default_rng(5)
    pick = lambda n, B: np.sort(r.permutation(n)[:B])
    idx = np.stack([np.stack([pick(5 * P, 9), pick(P - 3, 9)]) for _ in range(3)]).astype(np.int32)
    b.compact([0, 4], idx, tail=3)
    # picks behind the tail's start, negative ones, one twice, descending
    odd = np.array([[[4, 4, 2, -1, 2 * P, 2 * P + 1, 1 << 30, 0]]], dtype=np.int32)
    b.compact([2], odd, tail=1)
    b.compact([1], np.zeros((1, 1, 0), dtype=np.int32), tail=P + 2)
    b.compact([2, 0], np.zeros((1, 2, 4), dtype=np.int32), counts=[0, -3])
    assert list(b.compact([4, 1], np.zeros((1, 2, 1), dtype=np.int32), tail=13)) == [2, 0]


def test_compact_accepted_paths():
    """A speculative step's end: paths of several lengths, none accepted, all,
    forks that share the draft's page, and a count above the list's."""
    b = Both(P=16, n_pages=40, n_slots=8)
    lens, T = [37, 16, 5, 50, 20], [7, 8, 5, 3, 4]
    b.grow([0, 1, 2, 3, 4], lens)
    b.write([0, 1, 2, 3, 4], lens)
    b.fork([0], [5])
    idx = np.zeros((1, 6, 5), dtype=np.int32)
    idx[0, 0, :3] = [0, 2, 5]
    idx[0, 1, :5] = [0, 1, 4, 5, 7]
    idx[0, 3, :1] = [2]
    idx[0, 4, :4] = [0, 1, 2, 3]
    idx[0, 5, :2] = [1, 6]
    b.compact([0, 1, 2, 3, 4, 5], idx, span=T + [7], counts=[3, 9, 0, 1, 4, 2])
    b.grow([5, 1], [3, 30])
    # a span longer than the sequence is the sequence
    b.compact([4], np.array([[[3, 0]]], dtype=np.int32), span=[1000])


def test_compact_without_free_pages_leaves_the_sequence():
    b = Both(n_pages=7)
    b.grow([0, 1], [40, 48])
    b.write([0, 1], [40, 48])
    idx = np.arange(20, dtype=np.int32)[None, None].repeat(2, 1)
    assert list(b.compact([0, 1], idx)) == [1, 1]
    assert list(b.compact([1, 0], idx[:, :, :3].copy())) == [0, 1]


def test_random_lives():
    """Random calls over a pool that runs out now and then."""
    b = Both(nl=1, G=1, H=1, d=64, P=16, n_pages=30, n_slots=7, max_pages=9)
    r = np.random.default_rng(77)
    for step in range(60):
        slots = r.permutation(7)[:r.integers(1, 5)].tolist()
        op = r.integers(0, 6)
        if op <= 1:
            add = r.integers(0, 40, len(slots)).tolist()
            st = b.grow(slots, add)
            ok = [(s, a) for s, a, x in zip(slots, add, st) if x == 0]
            if ok:
                b.write([s for s, _ in ok], [a for _, a in ok])
        elif op == 2:
            free = [s for s in range(7) if s not in slots]
            dst = r.permutation(free)[:len(slots)].tolist()
            b.fork(slots[:len(dst)], dst)
        elif op == 3:
            b.free(slots, int(r.integers(0, 40)), int(r.integers(0, 40)))
        else:
            B = int(r.integers(0, 30))
            idx = r.integers(-2, 80, (1, len(slots), B)).astype(np.int32)
            span = r.integers(0, 60, len(slots)).tolist() if op == 4 else None
            b.compact(slots, idx, tail=int(r.integers(0, 9)), span=span,
                      counts=r.integers(-1, B + 2, len(slots)).tolist())


def test_many_sequences_and_a_large_pool():
    """256 sequences in one call, a pool of more pages than one scan step
    (8192), most of them taken."""
    n_pages = 20000
    b = Both(nl=1, G=1, H=1, d=64, P=16, n_pages=n_pages, n_slots=256, max_pages=80)
    slots = list(np.random.default_rng(3).permutation(256))
    slots = [int(s) for s in slots]
    b.grow(slots, [1 + (37 * i) % 1200 for i in range(256)])
    b.free(slots[::2])
    b.grow(slots[::2][:100], [900] * 100)
    b.fork(slots[1::2][:20], slots[::2][100:120])
    b.grow(slots[::2][100:120], [3] * 20)


def test_calls_of_more_threads_than_a_launch_holds():
    """A sequence of 2^26 tokens, all but its last page dropped: over 2^32 vectors
    to write in each layer, of one row that stands for all, and a list of 2^22
    tokens to keep, of which three count."""
    G, P, d, most = 64, 1024, 64, 1 << 16
    b = Both(nl=5, G=G, H=G, P=P, d=d, n_pages=4, n_slots=1, max_pages=most)
    b.m.len[0] = most * P
    b.m.table[0, -1], b.m.refs[2] = 2, 1
    b.c.table.copy_(torch.from_numpy(b.m.table))
    b.c.length.copy_(torch.from_numpy(b.m.len))
    b.c.refs.copy_(torch.from_numpy(b.m.refs))
    row = torch.arange(d, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    pg.pages_write(b.c, [0], [(1 << 23) + 1000], row, row, pg.KVLayout(0, 0, 0))
    b.m.k[:, 2] = b.m.v[:, 2] = np.arange(d)
    b.check("write")
    idx = torch.zeros(1, 1, 1 << 22, dtype=torch.int32, device="cuda")
    idx[0, 0, 2] = 9
    ws = torch.empty(pg.pages_workspace_bytes(b.c, 1, 1 << 22), dtype=torch.uint8, device="cuda")
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    pg.pages_compact(b.c, [0], idx, status, ws, span=[P],
                     counts=torch.tensor([3], dtype=torch.int32, device="cuda"))
    assert list(b.m.compact([0], np.array([[[0, 0, 9]]], dtype=np.int32), span=[P])) == [0]
    b.check("compact")
    assert int(status) == 0


def test_a_captured_step_replays():
    """Fork, grow, write and compact in one graph, replayed with eager work
    and synchronizations between: each replay is the eager call's result."""
    b = Both(n_pages=30)
    b.grow([0], [37])
    b.write([0], [37])
    c, P = b.c, 16
    k, v = b.rows(3), b.rows(3)
    kd = torch.from_numpy(k).cuda().view(torch.bfloat16)
    vd = torch.from_numpy(v).cuda().view(torch.bfloat16)
    idx = np.array([[[0, 5, 7, 30]]], dtype=np.int32)
    idxd = torch.from_numpy(idx).cuda()
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step():
        pg.pages_free(c, [1])
        pg.pages_fork(c, [0], [1])
        pg.pages_grow(c, [1], [3], st, b.ws)
        pg.pages_write(c, [1], [3], kd, vd, pg.rows_layout(kd))
        pg.pages_compact(c, [1], idxd, st, b.ws, tail=2)

    def model():
        b.m.free([1])
        b.m.fork([0], [1])
        b.m.grow([1], [3])
        b.m.write([1], [3], k, v)
        b.m.compact([1], idx, tail=2)

    step()
    model()
    b.check("eager")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        graph.replay()
        model()
        b.check(f"replay {i}")
        b.grow([0], [5 + i])          # eager work between the replays
        b.write([0], [5 + i])
