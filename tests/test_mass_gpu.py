"""Accumulated attention weights against the fp64 reference of
oracle/evict_oracle.py.  u = 2^-24, X the largest sum_j |q_j k_j| / sqrt(d) + |lse| of
what a token gets, N = T * H its weights at most:
  a weight's exponent is a sum of d products (exact ones or of one rounding) in
    float32, scaled, less lse log2(e): off by (d + 4) u X + 4 u (X + 1), and 2^x by 2 u;
  N additions of positive numbers: (N + 64) u, and one to the old mass;
  so |dm| <= 1.01 (((d + 8) u (X + 1) + (N + 64) u) add + 2 u m).
Pools are NaN wherever no token was written, and what a call should not write holds
7."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import fp4_cache as F  # noqa: E402
from oracle import evict_oracle as EO  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "fp4": torch.bfloat16}


def say(msg):
    print(f"[mass] {msg}", flush=True)


def rounded(x, dtype):
    return F.bf16(x) if dtype != "f32" else np.asarray(x, dtype=np.float32).astype(np.float64)


class Case:
    """Sequences of the given lengths on pages in random order, queries of their last
    rows, and the masses and log-sums before the call."""

    def __init__(self, seed, lens, rows, H=4, G=2, d=64, P=16, dtype="bf16", nl=1, qscale=1.0, order="plain"):
        r = self.r = np.random.default_rng(seed)
        self.lens, self.rows, self.nl, self.H, self.d, self.dtype, self.order = lens, rows, nl, H, d, dtype, order
        need = [-(-n // P) for n in lens]
        n_pages, slots, width = sum(need) + 2, len(lens) + 1, max(need + [1]) + 1
        if dtype == "fp4":
            m = F.empty_model(nl, n_pages, G, P, d, slots, width)
        else:
            pool = np.full((nl, n_pages, G, P, d), np.nan)
            m = PO.PagedModel(pool, pool.copy(), slots, width)
        self.m = m
        self.slots = r.permutation(slots)[:len(lens)].tolist()
        free = r.permutation(n_pages).tolist()
        for b, n in zip(self.slots, lens):
            m.len[b] = n
            for j in range(-(-n // P)):
                p = m.table[b, j] = free.pop()
                m.refs[p] = 1
                fill = min(P, n - j * P)
                x = rounded(r.standard_normal((nl, G, fill, d)), dtype)
                m.k[:, p, :, :fill] = EO.fp4_quantise(x) if dtype == "fp4" else x
        self.to_f64 = EO.fp4_numbers if dtype == "fp4" else lambda x: x
        self.q = rounded(r.standard_normal((nl, sum(rows), H, d)) * qscale, dtype)
        self.mass = r.random((nl, slots, m.cap)).astype(np.float32)
        self.sees = {}

    def upload(self, window=0, sinks=0):
        """The log-sums are those of the rows that see the window."""
        m, dt = self.m, TYPE[self.dtype]
        if self.dtype == "fp4":
            self.c = F.cache_of(m, self.H, self.d, self.order)
        else:
            k = torch.from_numpy(m.k).cuda().to(dt)
            if self.order == "groups":
                k = k.permute(2, 1, 0, 3, 4).contiguous().permute(2, 1, 0, 3, 4)
            elif self.order == "padded":
                k = torch.cat([k, k[..., :16]], -1)[..., :self.d]
            i32 = lambda x: torch.from_numpy(x).cuda()
            self.c = pg.Cache(k, k, i32(m.table), i32(m.len), i32(m.refs), self.H)
        self.lse = np.zeros((self.nl, sum(self.rows), self.H), dtype=np.float32)
        at = 0
        for b, n, T in zip(self.slots, self.lens, self.rows):
            see = PO.see_window(n, T, window, sinks)
            for l in range(self.nl):
                with np.errstate(all="ignore"):
                    _, lse, _, _ = PO.attend(self.only_k(), b, self.q[l, at:at + T], see, self.to_f64, l)
                self.lse[l, at:at + T] = lse
            at += T
        self.qd = torch.from_numpy(self.q).cuda().to(dt)
        self.md = torch.from_numpy(self.mass).cuda()

    def only_k(self):
        x = PO.PagedModel(self.m.k, self.m.k, *self.m.table.shape)
        x.table, x.len = self.m.table, self.m.len
        return x

    def call(self, window=0, sinks=0, max_len=None, out=None, ws=None, stream=None, lse=None):
        max_len = max(self.lens + [1]) if max_len is None else max_len
        if ws is None:
            need = pg.mass_workspace_bytes(self.c, self.rows, max_len)
            ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        self.out = torch.full_like(self.md, 7.0) if out is None else out
        lse = torch.from_numpy(self.lse).cuda() if lse is None else lse
        pg.mass_add(self.c, self.slots, self.rows, self.qd, lse, window, sinks, self.md, self.out, ws,
                    max_len=max_len, stream=stream)

    def check(self, tag, window=0, sinks=0):
        torch.cuda.synchronize()
        got, at, worst = self.out.double().cpu().numpy(), 0, 0.0
        rest = np.ones(got.shape, dtype=bool)
        for b, n, T in zip(self.slots, self.lens, self.rows):
            if T == 0:
                continue
            see = PO.see_window(n, T, window, sinks)
            rest[:, b, :n] = False
            for l in range(self.nl):
                add, size = EO.weights(self.m, b, self.q[l, at:at + T], self.lse[l, at:at + T].astype(float), see,
                                       self.to_f64, l)
                old = np.where(np.arange(n) < n - T, self.mass[l, b, :n].astype(float), 0)
                want, mine = old + add, got[l, b, :n]
                assert np.array_equal(np.isnan(want), np.isnan(mine)), f"{tag}: NaN, slot {b} layer {l}"
                tol = 1.01 * (((self.d + 8) * U * (size + 1) + (T * self.H + 64) * U) * add + 2 * U * want) + 1e-37
                fine = np.isfinite(want)
                assert np.array_equal(want[~fine], mine[~fine], equal_nan=True), tag
                err = np.abs(mine - want)[fine] / tol[fine]
                worst = max(worst, float(err.max()) if err.size else 0.0)
                assert worst <= 1, f"{tag}: slot {b} layer {l}: {worst:.2f} of the bound"
            at += T
        # tokens behind the last and sequences of no rows are as they were
        assert (got[rest] == 7).all(), f"{tag}: written elsewhere"
        say(f"{tag}: ok, {worst:.3f} of the bound")


def run(tag, c, window=0, sinks=0, **kw):
    say(f"{tag}: lens {c.lens} rows {c.rows} H {c.H} d {c.d} {c.dtype} window {window} {sinks}")
    c.upload(window, sinks)
    c.call(window, sinks, **kw)
    c.check(tag, window, sinks)


SHAPES = [(4, 2, 64, 16, "bf16"), (28, 4, 128, 64, "bf16"), (6, 1, 128, 32, "fp4"), (16, 16, 64, 256, "bf16"),
          (14, 2, 64, 16, "f32"), (3, 1, 128, 16, "f32"), (40, 2, 64, 32, "fp4"), (8, 8, 128, 16, "fp4")]


@pytest.mark.parametrize("H,G,d,P,dtype", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (17, 3), (64, 40)])
def test_shapes_and_windows(H, G, d, P, dtype, window, sinks):
    """Ragged: rows that are the whole sequence, one token, none, and more than a
    tile of rows; and one token of each."""
    lens, rows = [7, 1, 150, 300, 40, 257], [7, 1, 30, 3, 0, 1]
    run("ragged", Case(H * 5 + d + window, lens, rows, H, G, d, P, dtype, nl=2 if P == 16 else 1), window, sinks)
    run("tokens", Case(H + window, lens, [1] * 6, H, G, d, P, dtype), window, sinks)


@pytest.mark.parametrize("rows", [1, 2, 5, 9, 16, 33, 64, 100, 129])
@pytest.mark.parametrize("H,G,d,dtype", [(28, 4, 128, "bf16"), (8, 8, 64, "bf16"), (8, 1, 64, "fp4"),
                                         (7, 1, 128, "f32")])
def test_row_counts(rows, H, G, d, dtype):
    c = Case(rows + H, [rows, rows + 1, 300], [rows] * 3, H, G, d, 16, dtype)
    run("causal", c)
    run("window", c, 50, 5)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 129, 255, 256, 257, 513])
def test_lengths(n):
    """Around pages, tiles and a wave's tokens."""
    for H, G, d, T, dtype in ((7, 1, 128, 1, "bf16"), (2, 2, 64, 3, "fp4"), (8, 1, 64, 40, "bf16"),
                              (16, 2, 128, 9, "fp4"), (2, 1, 64, 5, "f32")):
        T = min(T, n)
        run("causal", Case(n, [n], [T], H, G, d, 16 if n % 2 else 64, dtype))
        run("window", Case(n, [n], [T], H, G, d, 16 if n % 2 else 64, dtype), max(n // 3, 1), n // 5)


@pytest.mark.parametrize("dtype", ["bf16", "fp4", "f32"])
@pytest.mark.parametrize("T", [2, 60])
def test_short_and_long_bounds(dtype, T):
    """max_len smaller and larger than the sequences: the same sums; twice the same
    bits."""
    c = Case(T, [700, 300, 5], [T, T, min(T, 5)], 8, 2, 64, 32, dtype)
    for max_len in (1, 64, 256, 300, 700, 5000, 1 << 26):
        run(f"max_len {max_len}", c, 400, 20, max_len=max_len)
        a = c.out.clone()
        c.call(400, 20, max_len=max_len)
        torch.cuda.synchronize()
        assert torch.equal(a, c.out)


@pytest.mark.parametrize("G", [1, 2, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp4", "f32"])
def test_whole_tiles_of_few_groups(dtype, G):
    """Enough tiles for the card: of 256 tokens below four groups, of four parts from
    there on."""
    c = Case(G, [700, 513, 40], [3, 1, 2], 8, G, 64, 32, dtype, nl=60)
    run("causal", c)
    run("window", c, 300, 20)


@pytest.mark.parametrize("dtype", ["bf16", "fp4", "f32"])
def test_split_products(dtype):
    """One sequence of many rows: its products are shared by several blocks, joined
    in order."""
    c = Case(5, [700], [300], 16, 2, 64, 16, dtype)
    assert pg.lib() and (c.upload() or pg.mass_workspace_bytes(c.c, c.rows, 700)) > 0
    run("split", c)
    run("split window", c, 150, 30)
    run("bound below the length", c, max_len=300)      # tiles behind it are not shared


@pytest.mark.parametrize("T", [3, 40])
def test_in_place_and_again(T):
    """out may be mass; two tokens' weights one after the other."""
    c = Case(6, [200, 90], [T, T], 4, 2, 64, 16)
    c.upload()
    c.call()
    a = c.out.clone()
    c.call(out=c.md)
    torch.cuda.synchronize()
    for b, n in zip(c.slots, c.lens):
        assert torch.equal(c.md[:, b, :n], a[:, b, :n])
    keep = torch.from_numpy(c.mass).cuda()
    for b, n in zip(c.slots, c.lens):
        assert torch.equal(c.md[:, b, n:], keep[:, b, n:])
    other = [b for b in range(3) if b not in c.slots][0]
    assert torch.equal(c.md[:, other], keep[:, other])


@pytest.mark.parametrize("dtype", ["bf16", "fp4", "f32"])
@pytest.mark.parametrize("T", [4, 40])
def test_dropped_pages_and_rows_without_a_token(dtype, T):
    c = Case(13, [200, 130, 2, 0], [T, T, T, T], 4, 2, 64, 16, dtype)
    for b in c.slots[:2]:
        c.m.table[b, 2], c.m.table[b, 3], c.m.table[b, 6] = -1, 1 << 30, -(1 << 31)
        c.m.table[b, 4] = c.m.n_pages
    run("dropped", c)
    run("dropped window", c, 90, 20)
    c.m.table[:] = -1
    run("all dropped", c)


@pytest.mark.parametrize("T", [3, 40])
def test_rows_whose_log_sum_is_minus_infinity(T):
    """They add nothing, whatever their logits are."""
    c = Case(14, [120], [T], 8, 2, 64, 16)
    c.q[0, 1, 3] = 1e38
    c.upload()
    c.lse[0, 1, 3] = c.lse[0, T - 1] = -np.inf
    c.call()
    c.check("dead rows")


@pytest.mark.parametrize("dtype", ["bf16", "fp4", "f32"])
@pytest.mark.parametrize("T", [4, 40])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_rows_of_a_bad_log_sum(dtype, T, bad):
    """They add nothing, to the tokens that they see and to the others."""
    c = Case(16, [130, T + 1], [T, T], 8, 2, 64, 16, dtype)
    for window, sinks in ((0, 0), (20, 3)):
        c.upload(window, sinks)
        c.lse[0, 1, 3] = c.lse[0, T + 2, :] = bad
        c.call(window, sinks)
        c.check(f"bad rows {window}", window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "fp4", "f32"])
@pytest.mark.parametrize("T", [4, 40])
def test_infinities_and_nan(dtype, T):
    """In K: they spoil the masses of their own tokens where rows see them, and no
    others."""
    for bad in ((np.nan, np.inf, -np.inf) if dtype != "fp4" else (np.nan,)):
        c = Case(15, [60, 150], [T, T], 4, 2, 64, 16, dtype)
        c.upload(25, 0)
        lse = c.lse
        for b, n in zip(c.slots, c.lens):
            for t in (n - 1, n - 2, max(n - T - 30, 0)):
                p, row = c.m.at(b, t)
                if dtype == "fp4":
                    c.m.k[0, p, 0, row, 32] = 255
                else:
                    c.m.k[0, p, 0, row, 5] = bad
        c.upload(25, 0)
        c.lse = lse                      # finite ones, as if they had been unseen
        c.call(25, 0)
        c.check(f"{bad}", 25, 0)


@pytest.mark.parametrize("order", ["groups", "padded"])
@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp4"])
def test_strided_pools_and_peaked_logits(order, dtype):
    for T in (2, 40):
        run(order, Case(8, [90, 41], [T, T], 8, 2, 128, 32, dtype, nl=2, order=order, qscale=6.0), 33, 2)


@pytest.mark.parametrize("T", [1, 9])
def test_as_many_sequences_as_a_call_takes(T):
    r = np.random.default_rng(40 + T)
    lens = r.integers(0, 40, 256).tolist()
    lens[77] = 1500
    rows = [int(x) for x in r.integers(0, T + 1, 256)]
    rows[77], rows[0], rows[255] = T, 0, 0
    run("causal", Case(41 + T, lens, rows, 10, 2, 64, 16), max_len=2000)
    run("window", Case(41 + T, lens, rows, 10, 2, 64, 16), 700, 6, max_len=20000)


def test_heads_of_a_group():
    for H, G, T, dtype in ((300, 1, 2, "bf16"), (129, 1, 1, "f32"), (64, 64, 2, "bf16"), (64, 64, 40, "fp4")):
        run(f"H {H} G {G}", Case(31 + H, [70, 5], [T, 1], H, G, 64, 16, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp4"])
def test_many_groups_and_large_tiles(dtype):
    """64 groups, and by the bound so many tokens that tiles have four parts: the most
    LDS."""
    lens, rows = [20 + i % 25 for i in range(118)] + [150, 1700], [1] * 119 + [0]
    run("64 groups", Case(3, lens, rows, 64, 64, 64, 16, dtype))


def test_layer_by_layer_and_streams():
    c = Case(16, [300, 77], [3, 3], 8, 2, 64, 16, nl=3)
    c.upload()
    c.call()
    torch.cuda.synchronize()
    whole = c.out.clone()
    lse, s = torch.from_numpy(c.lse).cuda(), torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.full_like(whole, 7.0)
    torch.cuda.synchronize()
    for l in range(3):
        pg.mass_add(c.c.layers(l), c.slots, c.rows, c.qd[l:l + 1], lse[l:l + 1], 0, 0, c.md[l:l + 1],
                    out[l:l + 1], None, max_len=300, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(out, whole)


def test_captured_calls_follow_the_lengths():
    a, b = Case(17, [400, 90], [2, 2], 8, 2, 128, 16), Case(18, [600], [150], 8, 2, 64, 16)
    full = list(a.lens)
    b.upload()
    a.upload()
    ws = torch.full((max(pg.mass_workspace_bytes(b.c, b.rows, 600), 16),), 255, dtype=torch.uint8, device="cuda")
    la, lb = torch.from_numpy(a.lse).cuda(), torch.from_numpy(b.lse).cuda()
    a.call(lse=la)
    b.call(ws=ws, lse=lb)
    torch.cuda.synchronize()
    b.check("eager")
    outs = a.out, b.out
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.call(lse=la, out=outs[0], max_len=400)
        b.call(ws=ws, lse=lb, out=outs[1])
    for lens in ([3, 90], [100, 2], full):
        a.lens = lens
        for slot, n in zip(a.slots, lens):
            a.m.len[slot] = n
        a.c.length.copy_(torch.from_numpy(a.m.len))
        for o in outs:
            o.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        a.check(f"replay {lens}")
        b.check("many")


@pytest.mark.parametrize("dtype", ["bf16", "fp4"])
def test_the_attention_s_own_log_sums(dtype):
    """Long sequences: each row's weights of a layer add up to the heads, and the sums
    agree with float64 ones by torch."""
    P, H, G, d = 64, 14, 2, 128
    lens, rows = [9000, 3001], [700, 1]
    width = -(-max(lens) // P)
    c = pg.new_cache(1, 2 * width, P, G, d, 2, width, H, dtype=pg.FP4 if dtype == "fp4" else torch.bfloat16)
    ws = torch.empty(pg.pages_workspace_bytes(c, 2), dtype=torch.uint8, device="cuda")
    st = torch.zeros(2, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    kv = torch.randn(2, 1, sum(lens), G, d, generator=gen, device="cuda").to(torch.bfloat16)
    back = torch.empty_like(kv)
    pg.pages_grow(c, [0, 1], lens, st, ws)
    pg.pages_write(c, [0, 1], lens, kv[0], kv[1], pg.rows_layout(kv[0]))
    pg.pages_read(c, [0, 1], lens, back[0], back[1], pg.rows_layout(kv[0]))
    tot = sum(rows)
    q = torch.randn(1, tot, H, d, generator=gen, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(1, tot, H, device="cuda")
    for window, sinks in ((0, 0), (2000, 300)):
        aws = torch.empty(max(16, pg.attend_workspace_bytes(c, rows, 9000),
                              pg.mass_workspace_bytes(c, rows, 9000)), dtype=torch.uint8, device="cuda")
        pg.attend_window(c, [0, 1], rows, q, window, sinks, out, aws, lse=lse, max_len=9000)
        mass = pg.new_mass(c)
        pg.mass_add(c, [0, 1], rows, q, lse, window, sinks, mass, mass, aws, max_len=9000)
        torch.cuda.synchronize()
        at = row = 0
        for b, (n, T) in enumerate(zip(lens, rows)):
            K = back[0, 0, at:at + n].double().transpose(0, 1)               # [G, n, d]
            want = torch.zeros(n, dtype=torch.float64, device="cuda")
            t, p = torch.arange(n, device="cuda"), torch.arange(n - T, n, device="cuda")[:, None]
            see = t <= p
            if window:
                see &= (t > p - window) | (t < sinks)
            for h in range(H):
                x = q[0, row:row + T, h].double() @ K[h * G // H].t().contiguous() / d ** 0.5
                want += torch.softmax(x.masked_fill(~see, -float("inf")), 1).sum(0)
            got = mass[0, b, :n].double()
            # the attention's lse is off by E + 2 u |lse| too (as in the tests of the
            # attentions, X <= 60), the weights by e^that
            E = 2 * (d + 8) * U * 61 + 3 * (n + 64) * U + 2 * U * 20
            tol = (1.01 * (E + (d + 8) * U * 81 + (T * H + 64) * U) + 2 * U) * want + 1e-30
            assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())
            assert abs(float(got.sum()) - T * H) <= 1e-3 * T * H
            at, row = at + n, row + T


def test_forks_take_their_masses():
    c = Case(19, [70, 33, 0], [1, 1, 1], 4, 2, 64, 16, nl=2)
    c.upload()
    free = [b for b in range(4) if b not in c.slots][0]
    want = torch.from_numpy(c.mass.copy())
    want[:, free, :70] = want[:, c.slots[0], :70]
    pg.mass_fork(c.c, [c.slots[0]], [free], c.md)
    torch.cuda.synchronize()
    assert torch.equal(c.md.cpu(), want)
    want[:, [free, c.slots[0]], :33] = want[:, [c.slots[1]], :33]
    pg.mass_fork(c.c, [c.slots[1], c.slots[1]], [free, c.slots[0]], c.md)
    torch.cuda.synchronize()
    assert torch.equal(c.md.cpu(), want)


def test_offsets_past_32_bits():
    """Masses of more than 2^31 elements: a slot far behind the first."""
    nl, slots, P = 1, 40, 1024
    width = (1 << 26) // P
    i32 = dict(dtype=torch.int32, device="cuda")
    k = torch.randn(nl, 2, 1, P, 64, device="cuda").to(torch.bfloat16)
    table = torch.full((slots, width), -1, **i32)
    table[39, 0], table[38, 0] = 1, 0
    c = pg.Cache(k, k, table, torch.zeros(slots, **i32), torch.ones(2, **i32), 2)
    c.length[39], c.length[38] = 700, 5
    mass = torch.empty(nl, slots, c.cap, device="cuda")
    mass[:, 38:, :1024] = 1
    q = torch.randn(1, 50, 2, 64, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(1, 50, 2, device="cuda")
    ws = torch.empty(max(pg.attend_workspace_bytes(c, [50], 700), pg.mass_workspace_bytes(c, [50], 700), 16),
                     dtype=torch.uint8, device="cuda")
    pg.attend_window(c, [39], [50], q, 0, 0, out, ws, lse=lse, max_len=700)
    pg.mass_add(c, [39], [50], q, lse, 0, 0, mass, mass, ws, max_len=700)
    pg.mass_fork(c, [39], [38], mass)
    torch.cuda.synchronize()
    # 650 old ones and 50 rows of two heads
    assert abs(float(mass[0, 39, :700].sum()) - 750) < 0.01 and float(mass[0, 39, 700]) == 1
    assert torch.equal(mass[0, 38, :701], mass[0, 39, :701])


def test_the_binding_refuses():
    c = Case(20, [40], [2], 4, 2, 64, 16)
    c.upload()
    lse = torch.from_numpy(c.lse).cuda()
    call = lambda q=c.qd, l=lse, m=c.md, o=c.md, rows=(2,): pg.mass_add(
        c.c, c.slots, list(rows), q, l, 0, 0, m, o, None, max_len=40)
    with pytest.raises(ValueError, match="q: torch.float32"):
        call(q=c.qd.float())
    with pytest.raises(ValueError, match="lse"):
        call(l=lse.double())
    with pytest.raises(ValueError, match="lse"):
        call(l=lse[:, :1])
    with pytest.raises(ValueError, match="mass"):
        call(m=c.md[:, :1])
    with pytest.raises(ValueError, match="out"):
        call(o=c.md.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError, match="one number per slot"):
        call(rows=(1, 1))
    with pytest.raises(ValueError, match="mass"):
        pg.mass_fork(c.c, [0], [1], c.md.double())
    call()
    torch.cuda.synchronize()
