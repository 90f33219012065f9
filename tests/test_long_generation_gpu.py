"""The calls of a long generation in a run, as a serving program makes them: prompts
go into a cache (of 4 bits, or bf16) layer by layer, their attention's weights are
added up, samples fork with them, tokens are decoded and weighed, and sequences that
outgrow a budget are evicted; the steady part again as a captured graph.  Each step
is held against the references on what the cache held at its time."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import fp4_cache as F  # noqa: E402
from oracle import evict_oracle as EO  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402
from paper_2606_01790_amd import starkv as sk  # noqa: E402

pytestmark = pytest.mark.gpu

NL, H, G, D, P = 2, 14, 2, 64, 16
U = 2.0 ** -24
BF = torch.bfloat16


def f64(t):
    return t.double().cpu().numpy()


def say(msg):
    print(f"[long] {msg}", flush=True)


class Held:
    """What the references say of a step's attention and weights."""

    def __init__(self, c, mass):
        self.c, self.m0 = c, mass.cpu().numpy().astype(float)

    def attention(self, out, lse, q, slots, rows, window, sinks, tag):
        """Bounds as in the tests of the attentions."""
        m, num = F.model_of(self.c)
        at = 0
        for b, T in zip(slots, rows):
            n = int(m.len[b])
            see = PO.see_window(n, T, window, sinks)
            for l in range(NL):
                o, s, w, size = PO.attend(m, b, f64(q[l, at:at + T]), see, num, l)
                E = 2 * (D + 8) * U * (size + 1) + 3 * (n + 64) * U
                tol = (E[..., None] * w + 2.0 ** -8 * (np.abs(o) + w)) * (1 + 2.0 ** -7) + 1e-30
                assert np.all(np.abs(f64(out[l, at:at + T]) - o) <= tol), f"{tag}: slot {b} layer {l}"
                assert np.all(np.abs(f64(lse[l, at:at + T]) - s) <= E + 2 * U * np.abs(s)), f"{tag}: lse"
            at += T

    def weights(self, mass, lse, q, slots, rows, window, sinks, tag):
        """Bounds as in the tests of the weights."""
        m, num = F.model_of(self.c)
        got, at = mass.cpu().numpy().astype(float), 0
        want = self.m0.copy()
        tol = np.zeros_like(want)
        for b, T in zip(slots, rows):
            n = int(m.len[b])
            see = PO.see_window(n, T, window, sinks)
            for l in range(NL):
                add, size = EO.weights(m, b, f64(q[l, at:at + T]), f64(lse[l, at:at + T]), see, num, l)
                want[l, b, :n] = np.where(np.arange(n) < n - T, want[l, b, :n], 0) + add
                tol[l, b, :n] = 1.01 * (((D + 8) * U * (size + 1) + (T * H + 64) * U) * add + 2 * U * want[l, b, :n])
            at += T
        assert np.all(np.abs(got - want) <= tol + 1e-37), f"{tag}: {np.max(np.abs(got - want) / (tol + 1e-37))}"


def sound(c):
    t, r = c.table.cpu().numpy(), c.refs.cpu().numpy()
    assert np.array_equal(np.bincount(t[t >= 0], minlength=len(r)), r)


@pytest.mark.parametrize("dtype", [pg.FP4, BF], ids=["fp4", "bf16"])
def test_a_long_generation(dtype):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(9)
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev).to(BF)
    n_slots, width = 4, 16
    c = pg.new_cache(NL, 60, P, G, D, n_slots, width, H, dtype=dtype)
    mass = pg.new_mass(c)
    views = [c.layers(l) for l in range(NL)]
    st = torch.full((n_slots,), 9, dtype=torch.int32, device=dev)
    pws = torch.empty(pg.pages_workspace_bytes(c, n_slots), dtype=torch.uint8, device=dev)
    need = max(max(pg.attend_workspace_bytes(x, r, c.cap), pg.mass_workspace_bytes(x, r, c.cap))
               for x in (c, views[0]) for r in ([120, 75], [1] * 3))
    aws = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)

    # two prompts, as a prefill of layer after layer makes them
    lens = [120, 75]
    q, k, v = rand(NL, 195, H, D), rand(NL, 195, G, D), rand(NL, 195, G, D)
    out, lse = torch.empty_like(q), torch.empty(NL, 195, H, device=dev)
    held = Held(c, mass)
    pg.pages_grow(c, [0, 1], lens, st, pws)
    for l in range(NL):
        pg.pages_write(views[l], [0, 1], lens, k[l], v[l], sk.KVLayout(0, D, G * D), grown=st)
        pg.attend_window(views[l], [0, 1], lens, q[l], 0, 0, out[l], aws, lse=lse[l])
        pg.mass_add(views[l], [0, 1], lens, q[l], lse[l], 0, 0, mass[l:l + 1], mass[l:l + 1], aws)
    torch.cuda.synchronize()
    held.attention(out, lse, q, [0, 1], lens, 0, 0, "prompt")
    held.weights(mass, lse, q, [0, 1], lens, 0, 0, "prompt")
    say("prompts")
    # what was written is what is read
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    pg.pages_read(c, [0, 1], lens, kb, vb, pg.rows_layout(kb))
    torch.cuda.synchronize()
    for got, new in ((kb, k), (vb, v)):
        want = EO.fp4_numbers(EO.fp4_quantise(f64(new))) if c.fp4 else f64(new)
        assert np.array_equal(f64(got), want)

    # a sample forks with its weights; three sequences decode
    pg.pages_fork(c, [0], [2])
    pg.mass_fork(c, [0], [2], mass)
    slots, ones = [0, 1, 2], [1, 1, 1]
    q1, k1, v1 = rand(NL, 3, H, D), rand(NL, 3, G, D), rand(NL, 3, G, D)
    o1, l1 = torch.empty_like(q1), torch.empty(NL, 3, H, device=dev)

    def token():
        pg.pages_grow(c, slots, ones, st, pws)
        pg.pages_write(c, slots, ones, k1, v1, pg.rows_layout(k1), grown=st)
        pg.attend_window(c, slots, ones, q1, 0, 0, o1, aws, lse=l1)
        pg.mass_add(c, slots, ones, q1, l1, 0, 0, mass, mass, aws)

    for i in range(3):
        q1.copy_(rand(NL, 3, H, D))
        k1.copy_(rand(NL, 3, G, D))
        held = Held(c, mass)
        token()
        torch.cuda.synchronize()
        assert st.tolist()[:3] == [0, 0, 0]
        held.attention(o1, l1, q1, slots, ones, 0, 0, f"token {i}")
        held.weights(mass, l1, q1, slots, ones, 0, 0, f"token {i}")
        sound(c)
    say("tokens")
    # as a captured step, replayed over growing sequences
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        token()
    for i in range(3):
        q1.copy_(rand(NL, 3, H, D))
        v1.copy_(rand(NL, 3, G, D))
        torch.cuda.synchronize()
        held = Held(c, mass)
        g.replay()
        torch.cuda.synchronize()
        held.attention(o1, l1, q1, slots, ones, 0, 0, f"replay {i}")
        held.weights(mass, l1, q1, slots, ones, 0, 0, f"replay {i}")
    assert c.length.tolist() == [126, 81, 126, 0]

    # the budget: 60 heavy tokens, 4 sinks, 16 recent ones; the second sequence just fits
    keep, sinks, recent = 61, 4, 16
    idx = torch.empty(NL, 3, sinks + keep, dtype=torch.int32, device=dev)
    ews = torch.empty(pg.evict_workspace_bytes(c, 3, keep, sinks, recent), dtype=torch.uint8, device=dev)
    m, _ = F.model_of(c)
    masses = mass.cpu().numpy()
    pg.pages_evict(c, slots, mass, keep, sinks, recent, idx, st, ews)
    torch.cuda.synchronize()
    want, status = EO.evict(m, slots, masses, keep, sinks, recent)
    assert st.tolist()[:3] == list(status) == [0, EO.SHORT, 0]
    assert np.array_equal(idx.cpu().numpy(), want) and np.array_equal(mass.cpu().numpy(), masses)
    assert c.length.tolist() == [81, 81, 81, 0] and np.array_equal(c.table.cpu().numpy(), m.table)
    now, _ = F.model_of(c)
    assert np.array_equal(now.k, m.k, equal_nan=True) and np.array_equal(now.v, m.v, equal_nan=True)
    sound(c)
    say("evicted")
    # and on with the captured step
    for i in range(2):
        k1.copy_(rand(NL, 3, G, D))
        torch.cuda.synchronize()
        held = Held(c, mass)
        g.replay()
        torch.cuda.synchronize()
        held.attention(o1, l1, q1, slots, ones, 0, 0, f"after {i}")
        held.weights(mass, l1, q1, slots, ones, 0, 0, f"after {i}")
    # a draft's accepted path joins, then is weighed as any rows are
    held = Held(c, mass)
    T = 6
    pg.pages_grow(c, [1], [T], st, pws)
    kt, vt, qt = rand(NL, T, G, D), rand(NL, T, G, D), rand(NL, T, H, D)
    pg.pages_write(c, [1], [T], kt, vt, pg.rows_layout(kt), grown=st)
    path = torch.tensor([[[0, 2, 5]]], dtype=torch.int32, device=dev)
    pg.pages_compact(c, [1], path, st, pws, span=[T], grown=st)
    qa = qt[:, [0, 2, 5]].contiguous()
    oa, la = torch.empty_like(qa), torch.empty(NL, 3, H, device=dev)
    pg.attend_window(c, [1], [3], qa, 0, 0, oa, aws, lse=la)
    pg.mass_add(c, [1], [3], qa, la, 0, 0, mass, mass, aws)
    torch.cuda.synchronize()
    assert c.length.tolist()[1] == 86
    held.attention(oa, la, qa, [1], [3], 0, 0, "accepted")
    held.weights(mass, la, qa, [1], [3], 0, 0, "accepted")
    pg.pages_free(c, [0, 1, 2, 3])
    torch.cuda.synchronize()
    assert not c.refs.any() and not c.length.any()
