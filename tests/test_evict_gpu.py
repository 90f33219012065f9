"""Eviction by accumulated weight against the host model: the kept tokens, the
statuses, the table, the lengths, the counts, the masses and every row bit for
bit."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import fp4_cache as F  # noqa: E402
from oracle import evict_oracle as EO  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402

pytestmark = pytest.mark.gpu


def say(msg):
    print(f"[evict] {msg}", flush=True)


NP = {"bf16": np.int16, "f32": np.int32, "fp4": np.uint8}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "fp4": torch.uint8}


class Both:
    """A cache of sequences of the given lengths, every row of its own bits, its
    masses, and the host model of both."""

    def __init__(self, seed, lens, nl=2, G=2, d=64, P=16, dtype="bf16", spare=20, masses=None):
        r = self.r = np.random.default_rng(seed)
        self.dtype, self.d = dtype, d
        need = [-(-n // P) for n in lens]
        n_pages, n_slots, width = sum(need) + spare, len(lens) + 1, max(need + [1]) + 1
        row = EO.fp4_row_bytes(d) if dtype == "fp4" else d
        shape = (nl, n_pages, G, P, row)
        mk = lambda: (r.integers(0, 250, shape) if dtype == "fp4" else
                      r.integers(-(1 << 15), 1 << 15, shape)).astype(NP[dtype])
        m = self.m = PO.PagedModel(mk(), mk(), n_slots, width)
        self.slots = r.permutation(n_slots)[:len(lens)].tolist()
        free = r.permutation(n_pages).tolist()
        for b, n in zip(self.slots, lens):
            m.len[b] = n
            for j in range(-(-n // P)):
                m.table[b, j] = free.pop()
                m.refs[m.table[b, j]] = 1
        self.mass = (r.random((nl, n_slots, m.cap)) ** 4 if masses is None else
                     masses(r, (nl, n_slots, m.cap))).astype(np.float32)

    def upload(self):
        m, i32 = self.m, lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        if self.dtype == "fp4":
            self.c = F.cache_of(m, m.k.shape[2], self.d)
        else:
            self.c = pg.Cache(torch.from_numpy(m.k).cuda().view(TYPE[self.dtype]),
                              torch.from_numpy(m.v).cuda().view(TYPE[self.dtype]), i32(m.table), i32(m.len),
                              i32(m.refs), m.k.shape[2])
        self.md = i32(self.mass)
        return self

    def evict(self, slots, keep, sinks, recent, tag=""):
        say(f"{tag} slots {slots} lens {self.m.len[slots].tolist()} keep {keep} sinks {sinks} recent {recent}")
        n, c = len(slots), self.c
        st = torch.full((n + 2,), 77, dtype=torch.int32, device="cuda")
        idx = torch.full((c.n_layers * n * (sinks + keep) + 3,), 77, dtype=torch.int32, device="cuda")
        need = pg.evict_workspace_bytes(c, n, keep, sinks, recent)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        pg.pages_evict(c, slots, self.md, keep, sinks, recent, idx, st, ws)
        want, status = EO.evict(self.m, slots, self.mass, keep, sinks, recent)
        torch.cuda.synchronize()
        assert st.tolist() == list(status) + [77, 77], f"{tag}: {st.tolist()} {status}"
        got = idx.cpu().numpy()
        assert np.array_equal(got[:-3].reshape(want.shape), want), f"{tag}: idx"
        assert (got[-3:] == 77).all(), f"{tag}: behind idx"
        self.check(tag)
        return status

    def check(self, tag):
        c, m = self.c, self.m
        assert np.array_equal(c.table.cpu().numpy(), m.table), f"{tag}: table"
        assert np.array_equal(c.length.cpu().numpy(), m.len), f"{tag}: length"
        assert np.array_equal(c.refs.cpu().numpy(), m.refs), f"{tag}: refs"
        assert np.array_equal(self.md.cpu().numpy(), self.mass, equal_nan=True), f"{tag}: masses"
        for got, want in ((c.k, m.k), (c.v, m.v)):
            if self.dtype == "fp4":
                assert np.array_equal(got.cpu().numpy(), EO.fp4_blocks(want)), f"{tag}: rows"
            else:
                bits = torch.int16 if self.dtype == "bf16" else torch.int32
                assert np.array_equal(got.view(bits).cpu().numpy(), want), f"{tag}: rows"


@pytest.mark.parametrize("dtype,d,P,G", [("bf16", 64, 16, 2), ("f32", 64, 32, 1), ("fp4", 64, 16, 3),
                                         ("fp4", 128, 64, 2), ("bf16", 128, 64, 4)])
@pytest.mark.parametrize("keep,sinks,recent", [(20, 4, 8), (1, 0, 0), (0, 4, 8), (0, 0, 3), (33, 17, 31), (64, 0, 1)])
def test_budgets(dtype, d, P, G, keep, sinks, recent):
    b = Both(keep + d, [200, 90, 33, 12, 0, 131], G=G, d=d, P=P, dtype=dtype).upload()
    b.evict(b.slots, keep, sinks, recent, "budgets")
    b.evict(b.slots, keep // 2, sinks, recent, "again")          # and of what is left


def test_nothing_kept():
    b = Both(1, [50, 0]).upload()
    assert list(b.evict(b.slots, 0, 0, 0)) == [PO.OK, EO.SHORT]
    assert b.m.len[b.slots[0]] == 0 and not b.m.refs.any()


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 1023, 1024, 1025, 4097, 5000])
def test_lengths(n):
    """Around pages, waves and the registers of a block."""
    b = Both(n, [n], nl=1, G=1).upload()
    for keep in sorted({1, n // 2, max(n - 2, 1), n}):
        b = Both(n, [n], nl=1, G=1, spare=n // 16 + 2).upload()
        b.evict(b.slots, keep, 0, 0, f"keep {keep}")
    b = Both(n, [n], nl=1, G=1, spare=n // 16 + 2).upload()
    b.evict(b.slots, n // 3, 1, n // 4)


@pytest.mark.parametrize("n", [16384 + 9, 32768 + 7, 70001])
def test_long_sequences(n):
    """More keys than a wave's registers hold."""
    b = Both(n, [n, 300], nl=2, G=1, P=256, spare=n // 256 + 4).upload()
    b.evict(b.slots, n // 5, 4, 32)


@pytest.mark.parametrize("n", [20000, 33000, 34000, 66000])
def test_long_sequences_of_odd_masses(n):
    """Ties over many waves, numbers of any bits, tokens without a page, little and
    nearly all kept."""
    masses = {"few": lambda r, s: r.integers(0, 3, s), "equal": lambda r, s: np.ones(s),
              "bits": lambda r, s: r.integers(0, 1 << 32, s).astype(np.uint32).view(np.float32),
              "close": lambda r, s: (np.float32(0.7).view(np.int32) + r.integers(0, 40, s)).astype(np.int32).view(np.float32)}
    for name, f in masses.items():
        for keep, sinks in ((7, 0), (n // 2, 70), (n - 400, 3)):
            b = Both(keep, [n], nl=1, G=1, P=256, spare=n // 256 + 4, masses=f)
            b.m._let_go(b.slots[0], [1, 20, 77])
            b.upload().evict(b.slots, keep, sinks, 32, name)


def test_equal_and_odd_masses():
    """Ties go to the lowest token; zeros of both signs are equal; infinities; NaN
    counts as the largest."""
    few = lambda r, s: r.integers(0, 3, s)
    for keep in (1, 7, 60, 150):
        b = Both(keep, [200, 170], masses=few).upload()
        b.evict(b.slots, keep, 3, 5, "ties")
        b = Both(keep, [200, 170], masses=lambda r, s: np.zeros(s)).upload()
        b.evict(b.slots, keep, 3, 5, "all equal")

    def odd(r, s):
        m = r.choice([0.0, -0.0, np.inf, np.nan, 1e-45, 3e38, -1.0, -np.inf, 1.0], s)
        return m

    for keep in (5, 60, 150):
        b = Both(keep, [200, 170], masses=odd).upload()
        b.evict(b.slots, keep, 0, 5, "odd")
    bits = np.array([0x7FC00000, 0xFFC00001, 0x7F800001, 0xFFFFFFFF], dtype=np.uint32).view(np.float32)
    b = Both(9, [200], masses=lambda r, s: np.where(r.random(s) < 0.1, r.choice(bits, s), r.random(s))).upload()
    b.evict(b.slots, 40, 0, 5, "NaN of every kind")


def test_close_masses():
    """Keys that differ in their last bits only, and far apart ones."""
    close = lambda r, s: (np.float32(0.7).view(np.int32) + r.integers(0, 40, s)).astype(np.int32).view(np.float32)
    far = lambda r, s: 2.0 ** r.integers(-149, 127, s)
    for masses in (close, far):
        b = Both(2, [900, 1000], masses=masses).upload()
        b.evict(b.slots, 333, 2, 9)


@pytest.mark.parametrize("dtype", ["bf16", "fp4"])
def test_dropped_tokens(dtype):
    b = Both(3, [200, 200, 200], dtype=dtype)
    s = b.slots
    b.m._let_go(s[0], [2, 3, 5])
    b.m._let_go(s[1], [0, 4])                       # sinks too
    b.m._let_go(s[2], [12])                         # the recent ones: no rows to keep
    b.m.table[s[0], 5] = 1 << 30
    b.upload()
    assert list(b.evict(s, 100, 6, 9)) == [PO.OK, PO.OK, PO.RANGE]
    b = Both(4, [200], dtype=dtype)
    b.m._let_go(b.slots[0], range(1, 11))           # fewer are left than are to be kept
    b.upload()
    b.evict(b.slots, 100, 6, 9, "few left")
    b = Both(5, [100], dtype=dtype)
    b.m._let_go(b.slots[0], range(0, 7))            # none but the recent ones
    b.upload()
    b.evict(b.slots, 10, 6, 0, "none left")


def test_too_few_pages():
    """Sequences are served in order while the pages last; the others keep rows and
    masses."""
    b = Both(6, [200, 180, 160], spare=5).upload()
    st = b.evict(b.slots, 40, 4, 8)                 # 4 pages each, 5 free
    assert list(st) == [PO.OK, PO.NO_PAGES, PO.NO_PAGES]
    assert list(b.evict(b.slots[1:], 40, 4, 8)) == [PO.OK, PO.OK]


def test_forks_and_their_parents():
    """A fork is evicted, its parent keeps the whole; both with their masses."""
    b = Both(7, [150], spare=30).upload()
    s, kid = b.slots[0], [x for x in range(2) if x not in b.slots][0]
    pg.pages_fork(b.c, [s], [kid])
    pg.mass_fork(b.c, [s], [kid], b.md)
    b.m.fork([s], [kid])
    b.mass[:, kid, :150] = b.mass[:, s, :150]
    torch.cuda.synchronize()
    b.check("fork")
    b.evict([kid], 30, 4, 10)
    assert b.m.len[s] == 150 and b.m.len[kid] == 44


def test_as_many_sequences_as_a_call_takes():
    r = np.random.default_rng(8)
    lens = r.integers(0, 60, 256).tolist()
    lens[100] = 2000
    b = Both(8, lens, nl=2, G=1, spare=400).upload()
    b.evict(b.slots, 11, 2, 6)


def test_no_sequences():
    b = Both(9, [50]).upload()
    pg.pages_evict(b.c, [], b.md, 1, 1, 1, torch.zeros(1, dtype=torch.int32, device="cuda"),
                   torch.zeros(1, dtype=torch.int32, device="cuda"), None)
    torch.cuda.synchronize()
    b.check("none")


def test_captured_on_another_stream():
    """A graph of an eviction, replayed with other masses and lengths."""
    b = Both(10, [300, 120], spare=60).upload()
    s, keep, sinks, recent = b.slots, 50, 4, 8
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    idx = torch.zeros(2, 2, sinks + keep, dtype=torch.int32, device="cuda")
    ws = torch.empty(pg.evict_workspace_bytes(b.c, 2, keep, sinks, recent), dtype=torch.uint8, device="cuda")
    b.evict(s, 200, sinks, recent, "eager")
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        pg.pages_evict(b.c, s, b.md, keep, sinks, recent, idx, st, ws)
    pws = torch.empty(pg.pages_workspace_bytes(b.c, 2), dtype=torch.uint8, device="cuda")
    for i, add in enumerate(([3, 0], [40, 70], [1, 33])):
        torch.cuda.synchronize()
        pg.pages_grow(b.c, s, add, st, pws)
        b.m.grow(s, add)
        new = b.r.random(b.mass.shape).astype(np.float32)
        b.mass[:] = new
        b.md.copy_(torch.from_numpy(new))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want, status = EO.evict(b.m, s, b.mass, keep, sinks, recent)
        assert st.tolist() == list(status), i
        assert np.array_equal(idx.cpu().numpy(), want), i
        b.check(f"replay {i}")


def test_the_binding_refuses():
    b = Both(11, [50]).upload()
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    call = lambda mass=b.md, idx=i(2, 1, 14), st=i(1), w=ws, keep=10: pg.pages_evict(
        b.c, b.slots, mass, keep, 4, 8, idx, st, w)
    with pytest.raises(ValueError, match="mass"):
        call(mass=b.md[:1])
    with pytest.raises(ValueError, match="idx"):
        call(idx=i(2, 1, 13))
    with pytest.raises(ValueError, match="status"):
        call(st=i(0))
    with pytest.raises(pg.StarKVError, match="E_WORKSPACE"):
        call(w=ws[:64])
    with pytest.raises(pg.StarKVError, match="E_BUDGET"):
        call(keep=-1)
    call()
    torch.cuda.synchronize()
