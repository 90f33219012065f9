"""The paged calls in a run, as a serving program makes them: a prompt is
written into pages and compressed by the stage's own selection, forked for
sampled actions, extended by drafted trees whose accepted paths are kept, and
decoded with a window whose dropped pages go back to the pool; layer by layer
where a model would, and the steady part again as a captured graph."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402
from paper_2606_01790_amd import starkv as sk  # noqa: E402

pytestmark = pytest.mark.gpu

NL, H, G, D, W, P = 3, 14, 2, 64, 8, 32
ROWS, COLS, TEXT = 9, 13, 40
BF = torch.bfloat16


def f64(t):
    return t.double().cpu().numpy()


def model_of(c):
    """The host model with what the cache holds now."""
    m = PO.PagedModel(f64(c.k), f64(c.v), *c.table.shape)
    m.table, m.len = c.table.cpu().numpy(), c.length.cpu().numpy()
    m.refs = c.refs.cpu().numpy()
    return m


def near(out, c, slots, rows, q, sees, tag):
    """Against the fp64 reference: weights and output rounded to bf16 (2^-8
    each, of the weighted |v| and of the value), and float32 sums."""
    m, at = model_of(c), 0
    for b, T in zip(slots, rows):
        for layer in range(c.n_layers):
            o, _, mass, _ = PO.attend(m, b, f64(q[layer, at:at + T]), sees(b, T, at, m), lambda x: x, layer)
            got = f64(out[layer, at:at + T])
            tol = 2.0 ** -8 * (mass + np.abs(o)) * 1.01 + 1e-5 * mass
            assert np.all(np.abs(got - o) <= tol), f"{tag}: slot {b} layer {layer}"
        at += T


def sound(c):
    """The counts are the entries that name each page."""
    t, r = c.table.cpu().numpy(), c.refs.cpu().numpy()
    assert np.array_equal(np.bincount(t[t >= 0], minlength=len(r)), r)


def test_generation_over_a_compressed_prompt():
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev).to(BF)
    L = ROWS * COLS + TEXT
    q, k, v = rand(NL, H, W, D), rand(NL, G, L, D), rand(NL, G, L, D)
    # the stage: score, statistics, selection of 30 tokens
    dims, p, B = sk.make_dims(NL, H, G, D, L, W, sk.BF16), sk.params_default(), 30
    f32 = dict(dtype=torch.float32, device=dev)
    S, sbar, s = torch.empty(NL * G * (L - W), **f32), torch.empty(NL * (L - W), **f32), torch.empty(NL * (L - W), **f32)
    gstar = torch.empty(NL * (L - W), dtype=torch.uint8, device=dev)
    idx = torch.empty(NL, 1, B, dtype=torch.int32, device=dev)
    cap = ROWS * COLS
    state = torch.empty(sk.state_bytes(dims, cap), dtype=torch.uint8, device=dev)
    scal = torch.empty(NL * sk.scalars_count(dims), **f32)
    ws = torch.empty(sk.workspace_bytes(dims), dtype=torch.uint8, device=dev)
    lay = sk.contiguous_layout(k, dims)
    sk.state_init(dims, state, cap)
    sk.score(dims, p, q, k, lay, S, sbar, gstar, ws)
    sk.update_state_select(dims, p, S, sbar, gstar, [(0, ROWS, COLS, 1)], 1, state, cap, scal, B, s, idx)
    ko = torch.empty(NL, G, B + W, D, dtype=BF, device=dev)
    vo = torch.empty_like(ko)
    sk.compact(dims, k, v, lay, idx, B, ko, vo)

    # the same within pages
    c = pg.new_cache(NL, 40, P, G, D, 5, 12, H)
    pws = torch.empty(pg.pages_workspace_bytes(c, 5), dtype=torch.uint8, device=dev)
    st = torch.full((5,), 9, dtype=torch.int32, device=dev)
    pg.pages_grow(c, [2], [L], st, pws)
    for layer in range(NL):            # written as a prefill does, layer by layer
        pg.pages_write(c.layers(layer), [2], [L], k[layer], v[layer],
                       sk.KVLayout(0, k.stride(1), k.stride(2)))
    pg.pages_fork(c, [2], [0])         # the whole prompt stays in slot 0
    pg.pages_compact(c, [2], idx, st, pws, tail=W)
    n = B + W
    torch.cuda.synchronize()
    assert int(st[0]) == 0 and c.length.tolist() == [L, 0, n, 0, 0]
    sound(c)
    t = torch.arange(n, device=dev)
    page, row = c.table[2].long()[t // P], t % P
    assert torch.equal(c.k[:, page, :, row].permute(1, 2, 0, 3), ko)
    assert torch.equal(c.v[:, page, :, row].permute(1, 2, 0, 3), vo)
    # a decoded token over them: starkv_decode's answer, rounded to bf16
    qd = rand(NL, 1, H, D)
    out = torch.empty_like(qd)
    aws = torch.empty(max(16, pg.attend_workspace_bytes(c, [24] * 4, L + 64)), dtype=torch.uint8, device=dev)
    pg.attend_window(c, [2], [1], qd, 0, 0, out, aws, max_len=n)
    ref = torch.empty(NL * H * D, **f32)
    dws = torch.empty(sk.decode_workspace_bytes(dims, n), dtype=torch.uint8, device=dev)
    sk.decode(dims, qd, ko, vo, sk.KVLayout(G * n * D, n * D, D), n, ref, dws)
    mass = torch.empty_like(ref)       # sum p |v|, for the rounded weights
    sk.decode(dims, qd, ko, vo.abs(), sk.KVLayout(G * n * D, n * D, D), n, mass, dws)
    err = (out.float().flatten() - ref).abs()
    assert bool((err <= 2.0 ** -8 * 1.01 * (mass + ref.abs())).all())

    # three actions from the compressed prompt, one from the whole one: trees
    # of different sizes, one forward of all layers
    slots, rows = [1, 3, 4, 0], [5, 24, 11, 7]
    pg.pages_fork(c, [2, 2, 2], slots[:3])
    pg.pages_grow(c, slots, rows, st, pws)
    tot = sum(rows)
    kn, vn, qn = rand(NL, tot, G, D), rand(NL, tot, G, D), rand(NL, tot, H, D)
    pg.pages_write(c, slots, rows, kn, vn, pg.rows_layout(kn))
    r = np.random.default_rng(1)
    bits, paths = [], []
    for T in rows:
        par = [-1] + [int(r.integers(0, j)) for j in range(1, T)]
        own = []
        for j in range(T):
            own.append((own[par[j]] if par[j] >= 0 else 0) | 1 << j)
        bits += own
        path = [T - 1]
        while par[path[-1]] >= 0:
            path.append(par[path[-1]])
        paths.append(path[::-1])
    mask = torch.tensor(np.array(bits, dtype=np.uint64).view(np.int64)[:, None], device=dev)
    outn = torch.empty_like(qn)
    pg.attend_tree(c, slots, rows, qn, mask, outn, aws, max_len=L + 24)
    sound(c)
    b64 = np.array(bits, dtype=np.uint64)[:, None]
    near(outn, c, slots, rows, qn,
         lambda b, T, at, m: PO.see_tree(int(m.len[b]), T, b64[at:at + T]), "tree")
    # the accepted paths stay
    most = max(map(len, paths))
    acc = torch.tensor([[x + [0] * (most - len(x)) for x in paths]], dtype=torch.int32, device=dev)
    cnt = torch.tensor([len(x) for x in paths], dtype=torch.int32, device=dev)
    before = c.length.tolist()
    pg.pages_compact(c, slots, acc, st, pws, span=rows, counts=cnt)
    sound(c)
    want = list(before)
    for b, T, x in zip(slots, rows, paths):
        want[b] += len(x) - T
    assert c.length.tolist() == want and st.tolist()[:4] == [0] * 4
    at = 0
    for b, T, x in zip(slots, rows, paths):
        n1 = want[b]
        tt = torch.arange(n1 - len(x), n1, device=dev)
        page, row = c.table[b].long()[tt // P], tt % P
        assert torch.equal(c.k[:, page, :, row].transpose(0, 1), kn[:, [at + j for j in x]])
        at += T

    # tokens decoded with a window; what it has left is freed
    window, sinks = 40, 3
    k1, v1, q1 = rand(NL, 4, G, D), rand(NL, 4, G, D), rand(NL, 4, H, D)
    out1 = torch.empty_like(q1)
    ones = [1] * 4

    def token():
        pg.pages_grow(c, slots, ones, st, pws)
        pg.pages_write(c, slots, ones, k1, v1, pg.rows_layout(k1))
        for layer in range(NL):
            one = views[layer]
            pg.attend_window(one, slots, ones, q1[layer:layer + 1], window, sinks, out1[layer:layer + 1],
                             aws, max_len=L + 64)
        pg.pages_free(c, slots, sinks, window)

    views = [c.layers(layer) for layer in range(NL)]
    sees = lambda b, T, at, m: PO.see_window(int(m.len[b]), T, window, sinks)
    token()
    torch.cuda.synchronize()
    near(out1, c, slots, ones, q1, sees, "token")
    sound(c)
    # the whole prompt's middle is gone: of its 158 to 165 tokens the last 40
    # begin in page 3, the sinks are in page 0
    assert c.table[0, 1:3].tolist() == [-1, -1] and int(c.table[0, 0]) >= 0 and int(c.table[0, 3]) >= 0
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        token()
    for i in range(4):
        k1.copy_(rand(NL, 4, G, D))
        q1.copy_(rand(NL, 4, H, D))
        torch.cuda.synchronize()
        n0 = c.length.tolist()
        g.replay()
        torch.cuda.synchronize()
        assert st.tolist()[:4] == [0] * 4
        assert c.length.tolist() == [x + (b in slots) for b, x in enumerate(n0)]
        near(out1, c, slots, ones, q1, sees, f"replay {i}")
        sound(c)
    # all ends: every page is free again
    pg.pages_free(c, [0, 1, 2, 3, 4])
    torch.cuda.synchronize()
    assert not c.refs.any() and not c.length.any() and (c.table == -1).all()
