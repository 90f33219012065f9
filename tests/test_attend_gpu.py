"""The attentions over a paged cache against the fp64 reference of
oracle/paged_oracle.py.  Pools are full of NaN wherever no token was written.

Bounds, from the roundings made.  u = 2^-24, X the largest sum_j |q_j k_j| /
sqrt(d) of a row, n its tokens:
  logits: exact products (bf16) or products of one rounding (float32), summed
    in float32: |dx| <= (d + 4) u X, and the scaling and 2^x add 4 u (X + 1);
  weights: both the weight and the sum that it is divided by move by
    e^|dx| - 1; the sums over n tokens by at most (n + 64) u, V's products too;
  so |do| <= E sum_t p_t |v_t| with E = 2 (d + 8) u (X + 1) + 3 (n + 64) u, and
  |dlse| <= E + 2 u |lse|;
  bf16 caches: the weights are rounded once, 2^-8 of each, and the output
    once, 2^-8 of it (float32: u of it)."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402
from paper_2606_01790_amd import workload as WL  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
BITS = {"bf16": torch.int16, "f32": torch.int32}


def say(msg):
    print(f"[attend] {msg}", flush=True)


def to_f64(dtype):
    if dtype == "f32":
        return lambda x: np.asarray(x, dtype=np.float64)
    return lambda x: (np.asarray(x).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_store(x, dtype):
    return x.astype(np.float32) if dtype == "f32" else WL.f32_to_bf16_bits(x.astype(np.float32))


def dev(x, dtype):
    if dtype == "f32":
        return torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).cuda().view(torch.bfloat16)


class Case:
    """Sequences of the given lengths on pages in random order."""

    def __init__(self, seed, lens, rows, H=4, G=2, d=64, P=16, dtype="bf16", nl=1, qscale=1.0,
                 slack=2, order="plain"):
        r = np.random.default_rng(seed)
        self.r, self.lens, self.rows, self.H, self.dtype, self.nl = r, lens, rows, H, dtype, nl
        need = [-(-n // P) for n in lens]
        n_pages = sum(need) + slack
        shape = (nl, n_pages, G, P, d)
        nan = np.full(shape, np.nan, dtype=np.float32)
        k, v = to_store(nan, dtype), to_store(nan, dtype)
        m = self.m = PO.PagedModel(k, v, len(lens) + 1, max(need + [1]) + 1)
        self.slots = r.permutation(len(lens) + 1)[:len(lens)].tolist()
        free = r.permutation(n_pages).tolist()
        for b, n in zip(self.slots, lens):
            m.len[b] = n
            for t in range(n):
                if t % P == 0:
                    p = m.table[b, t // P] = free.pop()
                    m.refs[p] = 1
                k[:, p, :, t % P] = to_store(r.standard_normal((nl, G, d)), dtype)
                v[:, p, :, t % P] = to_store(r.standard_normal((nl, G, d)), dtype)
        tot = sum(rows)
        self.q = to_store(r.standard_normal((nl, tot, H, d)) * qscale, dtype)
        self.order = order
        self.upload()

    def upload(self):
        m, dt = self.m, self.dtype
        k, v = dev(m.k, dt), dev(m.v, dt)
        if self.order == "groups":      # the group outermost
            k = k.permute(2, 1, 0, 3, 4).contiguous().permute(2, 1, 0, 3, 4)
            v = v.permute(2, 1, 0, 3, 4).contiguous().permute(2, 1, 0, 3, 4)
        elif self.order == "padded":
            pad = lambda x: torch.cat([x, x[..., :16]], -1)[..., :x.shape[-1]]
            k, v = pad(k), pad(v)
        self.c = pg.Cache(k, v, torch.from_numpy(m.table).cuda(), torch.from_numpy(m.len).cuda(),
                          torch.from_numpy(m.refs).cuda(), self.H)
        tot = sum(self.rows)
        # three rows more than the call has: they stay as they are
        self.out = torch.full((self.nl * tot + 3, self.H, self.c.d), 7.0, device="cuda").to(k.dtype)
        self.lse = torch.full((self.nl * tot + 3, self.H), 7.0, device="cuda")
        self.qd = dev(self.q, dt)

    def call(self, mask=None, window=0, sinks=0, max_len=None, lse=True, stream=None, ws=None):
        max_len = max(self.lens + [1]) if max_len is None else max_len
        if ws is None:
            need = pg.attend_workspace_bytes(self.c, self.rows, max_len)
            # a workspace that holds NaN: nothing is read that was not written
            ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        lse = self.lse if lse else None
        if mask is not None:
            md = torch.from_numpy(mask.view(np.int64)).cuda()
            pg.attend_tree(self.c, self.slots, self.rows, self.qd, md, self.out, ws, lse=lse,
                           max_len=max_len, stream=stream)
        else:
            pg.attend_window(self.c, self.slots, self.rows, self.qd, window, sinks, self.out, ws,
                             lse=lse, max_len=max_len, stream=stream)

    def sees(self, mask, window, sinks):
        at = 0
        for n, T in zip(self.lens, self.rows):
            yield (at, T, PO.see_tree(n, T, mask[at:at + T]) if mask is not None
                   else PO.see_window(n, T, window, sinks))
            at += T

    def check(self, tag, mask=None, window=0, sinks=0, lse=True):
        torch.cuda.synchronize()
        tot, d = sum(self.rows), self.c.d
        got = self.out.double().cpu().numpy()
        got_l = self.lse.double().cpu().numpy()
        assert (got[self.nl * tot:] == 7).all() and (got_l[self.nl * tot:] == 7).all(), \
            f"{tag}: written behind the last row"
        f = to_f64(self.dtype)
        worst = 0.0
        for layer in range(self.nl):
            for (at, T, see), b in zip(self.sees(mask, window, sinks), self.slots):
                if T == 0:
                    continue
                rows = slice(layer * tot + at, layer * tot + at + T)
                o, l, mass, size = PO.attend(self.m, b, f(self.q[layer, at:at + T]), see, f, layer)
                n = see.shape[1]
                E = (2 * (d + 8) * U * (size + 1) + 3 * (n + 64) * U)[..., None]
                low = 2.0 ** -8 if self.dtype == "bf16" else U
                tol = E * mass + low * np.abs(o) + (2.0 ** -8 * mass if self.dtype == "bf16" else 0)
                tol = tol * (1 + 2.0 ** -7) + 1e-30
                fine = np.isfinite(o)
                assert np.array_equal(fine, np.isfinite(got[rows])), f"{tag}: finite rows, L{layer}"
                assert np.array_equal(np.isnan(o), np.isnan(got[rows])), f"{tag}: NaN rows"
                err = np.abs(got[rows][fine] - o[fine]) / np.broadcast_to(tol, o.shape)[fine]
                worst = max(worst, float(err.max()) if err.size else 0.0)
                assert worst <= 1, f"{tag}: L{layer} slot {b}: {worst:.2f} of the bound"
                if lse:
                    gl = got_l[rows]
                    there = np.isfinite(l)
                    assert np.array_equal(gl[~there & ~np.isnan(l)], l[~there & ~np.isnan(l)]), tag
                    assert np.array_equal(np.isnan(gl), np.isnan(l)), tag
                    tl = E[..., 0] + 2 * U * np.abs(l) + 1e-30
                    el = np.abs(gl[there] - l[there]) / tl[there]
                    assert el.size == 0 or el.max() <= 1, f"{tag}: lse {el.max():.2f} of the bound"
        say(f"{tag}: ok, {worst:.3f} of the bound")


def tree_masks(r, rows, words):
    """Random trees' ancestor bits, with bits behind the last drafted token
    set (they mean nothing), a row that sees no drafted token, one that sees
    all of them."""
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
    say(f"{tag}: lens {case.lens} rows {case.rows} H {case.H} {case.dtype}")
    case.call(**kw)
    case.check(tag, **{k: v for k, v in kw.items() if k in ("mask", "window", "sinks", "lse")})


SHAPES = [  # H, G, d, P, dtype
    (4, 2, 64, 16, "bf16"), (28, 4, 128, 64, "bf16"), (6, 1, 128, 32, "bf16"), (16, 16, 64, 256, "bf16"),
    (14, 2, 64, 16, "f32"), (3, 1, 128, 16, "f32"), (40, 2, 64, 32, "bf16")]


@pytest.mark.parametrize("H,G,d,P,dtype", SHAPES)
def test_tree(H, G, d, P, dtype):
    """Ragged: drafted tokens alone in the cache, one token, a page's edge
    inside the tree, none, more rows than a tile."""
    lens, rows = [5, 1, 70, 33, 16, 200], [5, 1, 20, 2, 0, 9]
    c = Case(H * 7 + d, lens, rows, H, G, d, P, dtype, nl=2 if P == 16 else 1)
    run("tree", c, mask=tree_masks(c.r, rows, 1))


@pytest.mark.parametrize("H,G,d,P,dtype", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (17, 3), (64, 40)])
def test_window(H, G, d, P, dtype, window, sinks):
    lens, rows = [7, 1, 150, 300, 40, 257], [7, 1, 30, 3, 0, 1]
    c = Case(H * 5 + d + window, lens, rows, H, G, d, P, dtype)
    run("window", c, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_wide_trees(dtype):
    """Four words of mask; a tree that is the whole cache, one that is not."""
    rows = [256, 130]
    c = Case(3, [256, 300], rows, 4, 2, 64, 32, dtype)
    run("wide", c, mask=tree_masks(c.r, rows, 4))


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 9, 16, 33, 64, 100, 129])
@pytest.mark.parametrize("H,G,d", [(28, 4, 128), (8, 8, 64)])
def test_row_counts(rows, H, G, d):
    """Around the row tiles, causal and windowed."""
    lens = [rows, rows + 1, 300]
    c = Case(rows + H, lens, [rows] * 3, H, G, d, 16)
    run("causal", c)
    run("window", c, window=50, sinks=5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,T", [(300, 1, 2), (129, 1, 1), (320, 2, 3), (64, 64, 17)])
def test_heads_of_a_group(H, G, T, dtype):
    """More heads to a group than a block takes rows, and as few as one."""
    c = Case(31 + H, [70, 5], [T, 1], H=H, G=G, d=64, P=16, dtype=dtype)
    run(f"H {H} G {G} T {T} {dtype}", c, mask=tree_masks(c.r, c.rows, 1))
    run(f"H {H} G {G} T {T} {dtype} window", c, window=9, sinks=2)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511,
                               513, 1500])
def test_lengths(n):
    """Around pages, steps and splits."""
    for H, G, d, T in ((7, 1, 128, 1), (2, 2, 64, 3), (8, 1, 64, 40)):
        T = min(T, n)
        c = Case(n, [n], [T], H, G, d, 16 if n % 2 else 64)
        run("causal", c)
        run("tree", c, mask=tree_masks(c.r, [T], 1))
        run("window", c, window=max(n // 3, 1), sinks=n // 5)


@pytest.mark.parametrize("order", ["groups", "padded"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_pools(order, dtype):
    for T in (2, 40):
        c = Case(8, [90, 41], [T, T], 8, 2, 128, 32, dtype, nl=2, order=order)
        run(order, c, window=33, sinks=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_peaked_logits(dtype):
    """Large logits: a few tokens take nearly all the weight, the running
    maximum rises late."""
    for T in (3, 50):
        c = Case(4, [400], [T], 8, 2, 64, 16, dtype, qscale=12.0)
        run("peaked", c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [3, 40])
def test_rows_that_see_nothing(dtype, T):
    """A tree alone in its cache whose rows have empty masks; a sequence
    shorter than its rows (those before its first token see nothing); one of
    no token."""
    c = Case(11, [T, T], [T, T], 4, 2, 64, 16, dtype)
    mask = tree_masks(c.r, [T, T], 1)
    mask[1::2] = 0
    run("empty masks", c, mask=mask)
    assert torch.isinf(c.lse[1]).all() and (c.out[1] == 0).all()
    c = Case(12, [2, 0, 50], [T, T, 5], 4, 2, 64, 16, dtype)
    run("short", c, window=20, sinks=1)
    run("short tree", c, mask=tree_masks(c.r, [T, T, 5], 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [4, 40])
def test_dropped_pages(dtype, T):
    """Pages that a window has left, and entries that name no page, whose
    numbers are far outside the pool."""
    c = Case(13, [200, 130], [T, T], 4, 2, 64, 16, dtype)
    for b in c.slots:
        c.m.table[b, 2], c.m.table[b, 3], c.m.table[b, 6] = -1, 1 << 30, -(1 << 31)
        c.m.table[b, 4] = c.m.n_pages
    c.upload()
    run("dropped", c)
    run("dropped window", c, window=90, sinks=20)
    run("dropped tree", c, mask=tree_masks(c.r, [T, T], 1))
    for b in c.slots:
        c.m.table[b] = -1
    c.upload()
    run("all dropped", c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [4, 40])
def test_infinities_and_nan_in_masked_places(dtype, d, T):
    """K and V of tokens that some rows see and others do not hold infinities
    and NaN: the rows that do not see them are as without them."""
    for bad in (np.inf, -np.inf, np.nan):
        c = Case(14, [60, 150], [T, T], 4, 2, d, 16, dtype)
        val = to_store(np.array([bad]), dtype)[0]
        for b, n in zip(c.slots, c.lens):
            for t, col in ((n - 1, 3), (n - 2, d - 1), (n - T + 1, 17), (n - T - 30 if n > T + 30 else 0, 5)):
                p, row = c.m.at(b, t)
                c.m.v[0, p, :, row, col] = val
                if np.isnan(bad) and t == n - 1:
                    c.m.k[0, p, :, row, 2] = val
        c.upload()
        run(f"{bad} causal", c, lse=False)
        run(f"{bad} window", c, window=25, sinks=0, lse=False)
        run(f"{bad} tree", c, mask=tree_masks(c.r, [T, T], 1), lse=False)


@pytest.mark.parametrize("dtype,T", [("f32", 3), ("f32", 40), ("bf16", 3), ("bf16", 40)])
def test_logits_near_the_largest(dtype, T):
    """Logits near float32's limits stay apart from masked ones, and their
    differences count though no float32 multiple of them by the scale would
    keep them: equal weights over the multiples of 7 that a row sees, none
    elsewhere."""
    c = Case(15, [50], [T], 4, 2, 64, 16, dtype)
    k = np.zeros(64)
    for t in range(50):
        p, row = c.m.at(c.slots[0], t)
        k[0] = -3e37 if t % 7 else -2.9e37
        c.m.k[0, p, :, row] = to_store(k, dtype)
    q = np.zeros(64)
    q[0] = 8.0
    c.q[...] = to_store(q, dtype)
    c.upload()
    c.call()
    torch.cuda.synchronize()
    f = to_f64(dtype)
    v = np.stack([f(c.m.v[0, c.m.at(c.slots[0], t)[0], :, c.m.at(c.slots[0], t)[1]])
                  for t in range(0, 50, 7)])
    for i in range(T):
        n = (50 - T + i) // 7 + 1
        want = v[:n].mean(0).repeat(2, 0)                 # head h is of group h // 2
        got = c.out[i].double().cpu().numpy()
        low = 2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0
        assert np.all(np.abs(got - want) <= low + 64 * U * np.abs(v).max()), i


def test_splits_and_short_bounds():
    """max_len larger and smaller than the sequences: the work is divided
    otherwise, the results stay within the bound; the same call twice gives
    the same bits."""
    for T in (1, 3, 30):
        c = Case(16, [1500, 700, 3], [T, T, min(T, 3)], 4, 2, 128, 32)
        for max_len in (1, 256, 1500, 40000, 1 << 26):
            run(f"max_len {max_len}", c, window=900, sinks=40, max_len=max_len)
            a, l = c.out.clone(), c.lse.clone()
            c.call(window=900, sinks=40, max_len=max_len)
            torch.cuda.synchronize()
            assert torch.equal(a, c.out) and torch.equal(l, c.lse)


@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("bf16", 9), ("bf16", 20), ("f32", 2)])
def test_as_many_sequences_as_a_call_takes(dtype, T):
    """256 sequences, some without rows, some without tokens; one far longer
    than the others, so that all are split for its sake."""
    r = np.random.default_rng(40 + T)
    lens = r.integers(0, 40, 256).tolist()
    lens[77] = 3500
    rows = [int(x) for x in r.integers(0, T + 1, 256)]
    rows[77], rows[0], rows[255] = T, 0, 0
    c = Case(41 + T, lens, rows, 4, 2, 64, 16, dtype)
    run("causal", c, max_len=4000)
    run("window", c, window=3000, sinks=6, max_len=20000)


def test_a_slot_twice_no_lse_and_no_rows():
    c = Case(17, [70, 70], [4, 4], 4, 2, 64, 16)
    c.m.table[c.slots[1]] = c.m.table[c.slots[0]]
    c.slots[1] = c.slots[0]
    c.upload()
    run("twice", c, window=30, sinks=2, lse=False)
    assert (c.lse == 7).all()
    c.rows, c.slots = [0], c.slots[:1]
    c.call()
    pg.attend_window(c.c, [], [], c.qd, 0, 0, c.out, None, max_len=1)
    torch.cuda.synchronize()
    assert (c.lse == 7).all()


def test_other_stream_and_two_workspaces():
    """Two calls at once on two streams, each with its workspace."""
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


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements per K and V: pages at
    its far end, and strides that reach them."""
    P, d, G, H = 64, 128, 1, 4
    n_pages = (1 << 31) // (P * d) + 8              # 2^31 elements and eight pages
    k = torch.empty(1, n_pages, G, P, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    small = Case(20, [200, 100], [3, 40], H, G, d, P)
    m = small.m
    far = lambda p: n_pages - 1 - p
    for p in range(m.n_pages):
        k[:, far(p)] = small.c.k[:, p]
        v[:, far(p)] = small.c.v[:, p]
    table = torch.where(small.c.table >= 0, n_pages - 1 - small.c.table, -1).to(torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    small.c = pg.Cache(k, v, table, small.c.length, refs, H)
    run("far pages", small, window=150, sinks=9)


def test_captured_calls_follow_the_lengths():
    """A graph of two attentions, replayed while the cache grows: each replay
    reads the lengths and tables of its moment."""
    c = Case(21, [400, 90], [2, 2], 8, 2, 128, 16)
    full = list(c.lens)
    need = pg.attend_workspace_bytes(c.c, c.rows, 400)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    mask = tree_masks(c.r, c.rows, 1)
    md = torch.from_numpy(mask.view(np.int64)).cuda()
    out2, lse2 = torch.zeros_like(c.out), torch.zeros_like(c.lse)

    def calls():
        pg.attend_window(c.c, c.slots, c.rows, c.qd, 300, 4, c.out, ws, lse=c.lse, max_len=400)
        pg.attend_tree(c.c, c.slots, c.rows, c.qd, md, out2, ws, lse=lse2, max_len=400)

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
        torch.cuda.synchronize()
        g.replay()
        c.check(f"replay {lens}", window=300, sinks=4)
        keep = c.out, c.lse
        c.out, c.lse = out2, lse2
        c.out[sum(c.rows):] = 7
        c.lse[sum(c.rows):] = 7
        c.check(f"replay tree {lens}", mask=mask)
        c.out, c.lse = keep


def test_the_binding_refuses():
    c = Case(22, [40], [2], 4, 2, 64, 16)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    call = lambda q=c.qd, out=c.out, rows=(2,), lse=None, w=ws: pg.attend_window(
        c.c, c.slots, list(rows), q, 0, 0, out, w, lse=lse, max_len=40)
    with pytest.raises(ValueError, match="q: torch.float32"):
        call(q=c.qd.float())
    with pytest.raises(ValueError, match="contiguous"):
        call(q=c.qd.transpose(1, 2))
    with pytest.raises(ValueError, match="out"):
        call(out=c.out[:1])
    with pytest.raises(ValueError, match="device tensor"):
        call(out=c.out.cpu())
    with pytest.raises(ValueError, match="one number per slot"):
        call(rows=(1, 1))
    with pytest.raises(ValueError, match="lse"):
        call(lse=c.lse.double())
    with pytest.raises(ValueError, match="mask"):
        pg.attend_tree(c.c, c.slots, [2], c.qd, torch.zeros(1, 1, dtype=torch.int64, device="cuda"),
                       c.out, ws)
    with pytest.raises(pg.StarKVError, match="E_PARAM"):
        call(rows=(1 << 20,), q=torch.empty(1, dtype=c.qd.dtype, device="cuda").expand(
            1 << 28).contiguous(), out=torch.empty(1 << 28, dtype=c.qd.dtype, device="cuda"))
    with pytest.raises(ValueError, match="strides"):
        pg.Cache(c.c.k, c.c.v.transpose(0, 1).contiguous(), c.c.table, c.c.length, c.c.refs, 4)
    with pytest.raises(ValueError, match="refs"):
        pg.Cache(c.c.k, c.c.v, c.c.table, c.c.length, c.c.refs[:-1], 4)
    with pytest.raises(ValueError, match="idx"):
        pg.pages_compact(c.c, c.slots, torch.zeros(3, 1, 2, dtype=torch.int32, device="cuda"),
                         torch.zeros(1, dtype=torch.int32, device="cuda"), ws)
    call()                                    # and takes the call that is right
    torch.cuda.synchronize()
    c.check("right", lse=False)
