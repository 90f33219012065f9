"""The attentions over a cache held in 4 bits against the fp64 reference of
oracle/paged_oracle.py on the numbers that its rows stand for.  Elements become
bf16 numbers exactly, so the bounds are those of bf16 caches.  u = 2^-24, X the
largest sum_j |q_j k_j| / sqrt(d) of a row, n its tokens:
  logits: exact products summed in float32: |dx| <= (d + 4) u X, and the scaling
    and 2^x add 4 u (X + 1);
  weights: both the weight and the sum that it is divided by move by e^|dx| - 1;
    the sums over n tokens by at most (n + 64) u, V's products too;
  so |do| <= E sum_t p_t |v_t| with E = 2 (d + 8) u (X + 1) + 3 (n + 64) u, and
  |dlse| <= E + 2 u |lse|; the weights are rounded to bf16 once, 2^-8 of each, and
  the output once, 2^-8 of it.
Pools are NaN wherever no token was written."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import fp4_cache as F  # noqa: E402
from oracle import evict_oracle as EO  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def say(msg):
    print(f"[fp4 attend] {msg}", flush=True)


class Case:
    """Sequences of the given lengths on pages in random order."""

    def __init__(self, seed, lens, rows, H=4, G=2, d=64, P=16, nl=1, qscale=1.0, order="plain"):
        r = self.r = np.random.default_rng(seed)
        self.lens, self.rows, self.nl, self.H, self.d, self.order = lens, rows, nl, H, d, order
        need = [-(-n // P) for n in lens]
        m = self.m = F.empty_model(nl, sum(need) + 2, G, P, d, len(lens) + 1, max(need + [1]) + 1)
        self.slots = r.permutation(len(lens) + 1)[:len(lens)].tolist()
        free = r.permutation(sum(need) + 2).tolist()
        for b, n in zip(self.slots, lens):
            m.len[b] = n
            for j in range(-(-n // P)):
                p = m.table[b, j] = free.pop()
                m.refs[p] = 1
                fill = min(P, n - j * P)
                x = r.standard_normal((2, nl, G, fill, d)) * 2.0 ** r.integers(-2, 3, (2, 1, 1, 1, d // 32)).repeat(32, -1)
                m.k[:, p, :, :fill], m.v[:, p, :, :fill] = EO.fp4_quantise(x)
        self.q = F.bf16(r.standard_normal((nl, sum(rows), H, d)) * qscale)
        self.upload()

    def upload(self):
        self.c = F.cache_of(self.m, self.H, self.d, self.order)
        tot = sum(self.rows)
        # three rows more than the call has: they stay as they are
        self.out = torch.full((self.nl * tot + 3, self.H, self.d), 7.0, device="cuda").to(torch.bfloat16)
        self.lse = torch.full((self.nl * tot + 3, self.H), 7.0, device="cuda")
        self.qd = F.to_bf16(self.q)

    def call(self, mask=None, window=0, sinks=0, max_len=None, lse=True, stream=None, ws=None):
        max_len = max(self.lens + [1]) if max_len is None else max_len
        if ws is None:
            need = pg.attend_workspace_bytes(self.c, self.rows, max_len)
            ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        lse = self.lse if lse else None
        if mask is not None:
            md = torch.from_numpy(mask.view(np.int64)).cuda()
            pg.attend_tree(self.c, self.slots, self.rows, self.qd, md, self.out, ws, lse=lse,
                           max_len=max_len, stream=stream)
        else:
            pg.attend_window(self.c, self.slots, self.rows, self.qd, window, sinks, self.out, ws,
                             lse=lse, max_len=max_len, stream=stream)

    def check(self, tag, mask=None, window=0, sinks=0, lse=True):
        torch.cuda.synchronize()
        tot, d = sum(self.rows), self.d
        got, got_l = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        assert (got[self.nl * tot:] == 7).all() and (got_l[self.nl * tot:] == 7).all(), \
            f"{tag}: written behind the last row"
        at, worst = 0, 0.0
        for n, T, b in zip(self.lens, self.rows, self.slots):
            if T == 0:
                continue
            see = (PO.see_tree(n, T, mask[at:at + T]) if mask is not None
                   else PO.see_window(n, T, window, sinks))
            for layer in range(self.nl):
                rows = slice(layer * tot + at, layer * tot + at + T)
                o, l, mass, size = PO.attend(self.m, b, self.q[layer, at:at + T], see, EO.fp4_numbers, layer)
                E = (2 * (d + 8) * U * (size + 1) + 3 * (n + 64) * U)[..., None]
                tol = (E * mass + 2.0 ** -8 * (np.abs(o) + mass)) * (1 + 2.0 ** -7) + 1e-30
                fine = np.isfinite(o)
                assert np.array_equal(fine, np.isfinite(got[rows])), f"{tag}: finite rows, L{layer}"
                err = np.abs(got[rows][fine] - o[fine]) / np.broadcast_to(tol, o.shape)[fine]
                worst = max(worst, float(err.max()) if err.size else 0.0)
                assert worst <= 1, f"{tag}: L{layer} slot {b}: {worst:.2f} of the bound"
                if lse:
                    gl, there = got_l[rows], np.isfinite(l)
                    assert np.array_equal(gl[~there], l[~there], equal_nan=True), tag
                    el = np.abs(gl[there] - l[there]) / (E[..., 0] + 2 * U * np.abs(l) + 1e-30)[there]
                    assert el.size == 0 or el.max() <= 1, f"{tag}: lse {el.max():.2f} of the bound"
            at += T
        say(f"{tag}: ok, {worst:.3f} of the bound")


def tree_masks(r, rows, words):
    """Random trees' ancestor bits, with bits behind the last drafted token set, a
    row that sees no drafted token, one that sees all of them."""
    out = []
    for T in rows:
        bits = []
        for j in range(T):
            par = int(r.integers(-1, j)) if j else -1
            bits.append((bits[par] if par >= 0 else 0) | 1 << j)
        if T > 2:
            bits[1], bits[2] = 0, (1 << T) - 1
        junk = (1 << 64 * words) - (1 << T) if 64 * words > T else 0
        out += [[(x | junk) >> 64 * w & (1 << 64) - 1 for w in range(words)] for x in bits]
    return np.array(out, dtype=np.uint64).reshape(-1, words)


def run(tag, case, **kw):
    say(f"{tag}: lens {case.lens} rows {case.rows} H {case.H} d {case.d}")
    case.call(**kw)
    case.check(tag, **{k: v for k, v in kw.items() if k in ("mask", "window", "sinks", "lse")})


SHAPES = [(4, 2, 64, 16), (28, 4, 128, 64), (6, 1, 128, 32), (16, 16, 64, 256), (14, 2, 128, 16), (40, 2, 64, 32)]


@pytest.mark.parametrize("H,G,d,P", SHAPES)
def test_tree(H, G, d, P):
    """Ragged: drafted tokens alone in the cache, one token, a page's edge inside
    the tree, none, more rows than a tile."""
    lens, rows = [5, 1, 70, 33, 16, 200], [5, 1, 20, 2, 0, 9]
    c = Case(H * 7 + d, lens, rows, H, G, d, P, nl=2 if P == 16 else 1)
    run("tree", c, mask=tree_masks(c.r, rows, 1))


@pytest.mark.parametrize("H,G,d,P", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (17, 3), (64, 40)])
def test_window(H, G, d, P, window, sinks):
    lens, rows = [7, 1, 150, 300, 40, 257], [7, 1, 30, 3, 0, 1]
    run("window", Case(H * 5 + d + window, lens, rows, H, G, d, P), window=window, sinks=sinks)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 9, 16, 33, 100])
@pytest.mark.parametrize("H,G,d", [(28, 4, 128), (8, 8, 64), (8, 1, 128)])
def test_row_counts(rows, H, G, d):
    """Around the row tiles, causal and windowed; both kernels."""
    c = Case(rows + H, [rows, rows + 1, 300], [rows] * 3, H, G, d, 16)
    run("causal", c)
    run("window", c, window=50, sinks=5)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 513])
def test_lengths(n):
    """Around pages, steps and splits."""
    for H, G, d, T in ((7, 1, 128, 1), (2, 2, 64, 3), (8, 1, 64, 40), (8, 1, 128, 9)):
        T = min(T, n)
        c = Case(n, [n], [T], H, G, d, 16 if n % 2 else 64)
        run("causal", c)
        run("tree", c, mask=tree_masks(c.r, [T], 1))
        run("window", c, window=max(n // 3, 1), sinks=n // 5)


def test_wide_trees():
    c = Case(3, [256, 300], [256, 130], 4, 2, 64, 32)
    run("wide", c, mask=tree_masks(c.r, c.rows, 4))


@pytest.mark.parametrize("order", ["groups", "padded"])
def test_strided_pools(order):
    for T in (2, 40):
        run(order, Case(8, [90, 41], [T, T], 8, 2, 128, 32, nl=2, order=order), window=33, sinks=2)


@pytest.mark.parametrize("T", [3, 50])
def test_peaked_logits(T):
    run("peaked", Case(4, [400], [T], 8, 2, 64, 16, qscale=12.0))


@pytest.mark.parametrize("T", [3, 40])
def test_rows_that_see_nothing(T):
    c = Case(11, [T, T], [T, T], 4, 2, 64, 16)
    mask = tree_masks(c.r, [T, T], 1)
    mask[1::2] = 0
    run("empty masks", c, mask=mask)
    assert torch.isinf(c.lse[1]).all() and (c.out[1] == 0).all()
    c = Case(12, [2, 0, 50], [T, T, 5], 4, 2, 64, 16)
    run("short", c, window=20, sinks=1)
    run("short tree", c, mask=tree_masks(c.r, [T, T, 5], 1))


@pytest.mark.parametrize("T", [4, 40])
def test_dropped_pages(T):
    c = Case(13, [200, 130], [T, T], 4, 2, 64, 16)
    for b in c.slots:
        c.m.table[b, 2], c.m.table[b, 3], c.m.table[b, 6] = -1, 1 << 30, -(1 << 31)
        c.m.table[b, 4] = c.m.n_pages
    c.upload()
    run("dropped", c)
    run("dropped window", c, window=90, sinks=20)
    run("dropped tree", c, mask=tree_masks(c.r, [T, T], 1))
    c.m.table[:] = -1
    c.upload()
    run("all dropped", c)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [4, 40])
def test_nan_in_masked_places(d, T):
    """Blocks of K and V that are NaN, of tokens that some rows see and others do
    not: the rows that do not see them are as without them."""
    for in_k in (False, True):
        c = Case(14, [60, 150], [T, T], 4, 2, d, 16)
        for b, n in zip(c.slots, c.lens):
            for t, blk in ((n - 1, 0), (n - 2, d // 32 - 1), (n - T + 1, 1), (n - T - 30 if n > T + 30 else 0, 0)):
                p, row = c.m.at(b, t)
                (c.m.k if in_k else c.m.v)[0, p, :, row, d // 2 + blk] = 255
        c.upload()
        run("NaN causal", c, lse=False)
        run("NaN window", c, window=25, sinks=0, lse=False)
        run("NaN tree", c, mask=tree_masks(c.r, [T, T], 1), lse=False)


def test_extreme_scales():
    """Blocks at the ends of the scales: tiny ones lose nothing, huge ones stay
    finite."""
    for T in (2, 40):
        c = Case(15, [90], [T], 4, 2, 64, 16)
        c.m.v[..., 32] = np.where(c.m.v[..., 32] == 255, 255, 2)
        c.m.v[..., 33] = np.where(c.m.v[..., 33] == 255, 255, 240)
        c.m.k[..., 32] = np.where(c.m.k[..., 32] == 255, 255, 3)
        c.upload()
        run("extreme", c)


def test_splits_and_short_bounds():
    for T in (1, 3, 30):
        c = Case(16, [1500, 700, 3], [T, T, min(T, 3)], 4, 2, 128, 32)
        for max_len in (1, 256, 1500, 40000, 1 << 26):
            run(f"max_len {max_len}", c, window=900, sinks=40, max_len=max_len)
            a, l = c.out.clone(), c.lse.clone()
            c.call(window=900, sinks=40, max_len=max_len)
            torch.cuda.synchronize()
            assert torch.equal(a, c.out) and torch.equal(l, c.lse)


@pytest.mark.parametrize("T", [1, 9])
def test_as_many_sequences_as_a_call_takes(T):
    r = np.random.default_rng(40 + T)
    lens = r.integers(0, 40, 256).tolist()
    lens[77] = 2500
    rows = [int(x) for x in r.integers(0, T + 1, 256)]
    rows[77], rows[0], rows[255] = T, 0, 0
    c = Case(41 + T, lens, rows, 4, 2, 64, 16)
    run("causal", c, max_len=3000)
    run("window", c, window=2000, sinks=6, max_len=20000)


def test_a_slot_twice_other_streams_and_no_rows():
    c = Case(17, [70, 70], [4, 4], 4, 2, 64, 16)
    c.m.table[c.slots[1]] = c.m.table[c.slots[0]]
    c.slots[1] = c.slots[0]
    c.upload()
    run("twice", c, window=30, sinks=2, lse=False)
    assert (c.lse == 7).all()
    a, b = Case(18, [900], [5], 8, 2, 128, 32), Case(19, [800], [6], 8, 2, 128, 32)
    ws = [torch.full((pg.attend_workspace_bytes(x.c, x.rows, x.lens[0]),), 255, dtype=torch.uint8,
                     device="cuda") for x in (a, b)]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        a.call(window=700, sinks=4, stream=s1, ws=ws[0])
        b.call(stream=s2, ws=ws[1])
        torch.cuda.synchronize()
        a.check("stream 1", window=700, sinks=4)
        b.check("stream 2")


def test_captured_calls_follow_the_lengths():
    c = Case(21, [400, 90], [2, 2], 8, 2, 128, 16)
    many = Case(22, [300], [40], 8, 2, 128, 16)
    full = list(c.lens)
    ws = [torch.full((max(pg.attend_workspace_bytes(x.c, x.rows, 400), 16),), 255, dtype=torch.uint8,
                     device="cuda") for x in (c, many)]
    calls = lambda: (c.call(window=300, sinks=4, max_len=400, ws=ws[0]), many.call(max_len=400, ws=ws[1]))
    calls()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for lens in ([3, 90], [100, 2], full):
        c.lens = lens
        for b, n in zip(c.slots, lens):
            c.m.len[b] = n
        c.c.length.copy_(torch.from_numpy(c.m.len))
        many.out.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        c.check(f"replay {lens}", window=300, sinks=4)
        many.check("many")


def test_a_long_cache_against_its_bf16_copy():
    """A long cache read back into a bf16 one: the attentions of both agree to the
    rounding of the weights and the output."""
    P, n, H, G, d = 64, 20011, 14, 2, 128
    np_ = n // P + 1
    c = pg.new_cache(1, np_, P, G, d, 1, np_, H, dtype=pg.FP4)
    e = pg.new_cache(1, np_, P, G, d, 1, np_, H)
    ws = torch.empty(pg.pages_workspace_bytes(c, 1), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    kv = torch.randn(2, 1, n, G, d, generator=gen, device="cuda").to(torch.bfloat16)
    back = torch.empty_like(kv)
    lay = pg.rows_layout(kv[0])
    for x in (c, e):
        pg.pages_grow(x, [0], [n], st, ws)
    pg.pages_write(c, [0], [n], kv[0], kv[1], lay)
    pg.pages_read(c, [0], [n], back[0], back[1], lay)
    pg.pages_write(e, [0], [n], back[0], back[1], lay)
    for T in (1, 4, 300):
        q = torch.randn(1, T, H, d, generator=gen, device="cuda").to(torch.bfloat16)
        got = []
        for x in (c, e):
            aws = torch.empty(max(16, pg.attend_workspace_bytes(x, [T], n)), dtype=torch.uint8, device="cuda")
            out, lse = torch.empty_like(q), torch.empty(1, T, H, device="cuda")
            pg.attend_window(x, [0], [T], q, 0, 0, out, aws, lse=lse, max_len=n)
            got.append((out.double(), lse.double()))
        torch.cuda.synchronize()
        (o1, l1), (o2, l2) = got
        # every weight and output of each is off by a rounding of 2^-8 at most, weights by
        # both signs: |o1 - o2| <= 2 * 2^-8 (sum p |v| + |o|), and sum p |v| <= max |v|
        top = back[1].abs().amax().double()
        assert bool(((o1 - o2).abs() <= 2 * 2.0 ** -8 * 1.01 * (top + o2.abs())).all())
        assert (o1 - o2).norm() <= 2.0 ** -7 * o2.norm()
        # logits of 128 products each, sums over n tokens
        assert (l1 - l2).abs().max() <= 2 * (2 * 136 * U * 60 + 3 * (n + 64) * U)


def test_the_binding_refuses():
    P, d = 16, 64
    z = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    k = z(1, 4, 2, pg.fp4_block_bytes(P, d))
    mk = lambda a, b, dd: pg.Cache(a, b, i(2, 3), i(2), i(4), 4, dd)
    with pytest.raises(ValueError, match="d: None"):
        mk(k, k.clone(), None)
    with pytest.raises(ValueError, match="64 or 128"):
        mk(k, k.clone(), 96)
    with pytest.raises(ValueError, match="blocks of"):
        mk(z(1, 4, 2, 545), z(1, 4, 2, 545), d)
    with pytest.raises(ValueError, match="strides"):
        mk(k, z(1, 4, 2, 544 * 2)[..., ::2], d)
    c = mk(k, k.clone(), d)
    assert c.page_tokens == P and c.dtype == torch.bfloat16
    q = torch.zeros(1, 1, 4, d, device="cuda")
    with pytest.raises(ValueError, match="q: torch.float32"):
        pg.attend_window(c, [0], [1], q, 0, 0, q.clone(), None)
    with pytest.raises(ValueError, match="k: torch.uint8"):
        pg.pages_write(c, [0], [1], k, k, pg.rows_layout(torch.zeros(1, 1, 2, d)))
    with pytest.raises(pg.StarKVError, match="E_SHAPE"):
        pg.pages_init(mk(z(1, 4, 2, pg.fp4_block_bytes(8, d)), z(1, 4, 2, pg.fp4_block_bytes(8, d)), d))
