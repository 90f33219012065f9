"""Added weights behind a grow that found no pages: a sequence that it left unchanged
keeps every mass bit for bit, and the others get what they get without it, in both
kernels, eagerly and in a replayed graph."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_01790_amd import paged as pg  # noqa: E402
from test_long_generation_gpu import BF, Held, sound  # noqa: E402
from test_long_generation_gpu import D, G, H, NL, P  # noqa: E402
from test_mass_gpu import Case, say  # noqa: E402

pytestmark = pytest.mark.gpu

# masses of odd bits, which only a copy keeps
ODD = np.array([0x80000000, 0x7F800001, 0xFFC12345, 0x00000001, 0x7F800000], dtype=np.uint32).view(np.float32)


def bits(t):
    return t.view(torch.int32)


@pytest.mark.parametrize("dtype", ["bf16", "fp4", "f32"])
@pytest.mark.parametrize("lens,rows,nl", [([200, 130, 70, 40], [3, 3, 2, 0], 2), ([200, 130, 70, 300], [40, 40, 40, 0], 2),
                                          ([700, 600, 5, 9], [300, 300, 5, 0], 1), ([130] * 3, [1] * 3, 1)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (30, 5)])
def test_kept_masses(dtype, lens, rows, nl, window, sinks):
    """Few rows, many, and so many that their products are shared and joined."""
    c = Case(sum(rows), lens, rows, 8, 2, 64, 16, dtype, nl=nl)
    c.mass.reshape(-1)[::7] = np.resize(ODD, c.mass.reshape(-1)[::7].shape)
    c.upload(window, sinks)
    ws = torch.full((max(pg.mass_workspace_bytes(c.c, rows, 700), 16),), 255, dtype=torch.uint8, device="cuda")
    lse = torch.from_numpy(c.lse).cuda()
    run = lambda out, mass, **kw: pg.mass_add(c.c, c.slots, c.rows, c.qd, lse, window, sinks, mass, out, ws,
                                              max_len=700, **kw)
    plain = torch.full_like(c.md, 7.0)
    run(plain, c.md)
    for status in ([0] * 4, [1, 0, 0, 0], [0, 1, 2, 0], [0, 3, 0, 1], [2, 1, -5, 9]):
        status = status[:len(lens)]
        say(f"grown {status}")
        grown = torch.tensor(status, dtype=torch.int32, device="cuda")
        out, same = torch.full_like(c.md, 7.0), c.md.clone()
        run(out, c.md, grown=grown)
        run(same, same, grown=grown)
        torch.cuda.synchronize()
        want, want_same = torch.full_like(c.md, 7.0), c.md.clone()
        for b, n, T, s in zip(c.slots, lens, rows, status):
            if T:
                want[:, b, :n] = c.md[:, b, :n] if s else plain[:, b, :n]
                want_same[:, b, :n] = want[:, b, :n]
        assert torch.equal(bits(out), bits(want)), f"{status}: out"
        assert torch.equal(bits(same), bits(want_same)), f"{status}: in place"


@pytest.mark.parametrize("dtype", [pg.FP4, BF], ids=["fp4", "bf16"])
def test_a_step_in_a_full_pool(dtype):
    """A captured step of grow, write, attention and weights over two sequences, of
    which the second finds no page, until the first makes room."""
    dev, gen = torch.device("cuda"), torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev).to(BF)
    lens, slots, ones = [4 * P - 2, 3 * P], [0, 1], [1, 1]
    c = pg.new_cache(NL, 7, P, G, D, 2, 6, H, dtype=dtype)           # every page is taken
    mass = pg.new_mass(c)
    st = torch.full((2,), 9, dtype=torch.int32, device=dev)
    pws = torch.empty(pg.pages_workspace_bytes(c, 2), dtype=torch.uint8, device=dev)
    aws = torch.empty(max(16, *(f(c, r, c.cap) for f in (pg.attend_workspace_bytes, pg.mass_workspace_bytes)
                                for r in (lens, ones))), dtype=torch.uint8, device=dev)
    tot = sum(lens)
    q, k, v = rand(NL, tot, H, D), rand(NL, tot, G, D), rand(NL, tot, G, D)
    out, lse = torch.empty_like(q), torch.empty(NL, tot, H, device=dev)
    pg.pages_grow(c, slots, lens, st, pws)
    pg.pages_write(c, slots, lens, k, v, pg.rows_layout(k), grown=st)
    pg.attend_window(c, slots, lens, q, 0, 0, out, aws, lse=lse)
    pg.mass_add(c, slots, lens, q, lse, 0, 0, mass, mass, aws, grown=st)
    torch.cuda.synchronize()
    assert st.tolist() == [0, 0] and c.length.tolist() == lens and bool((c.refs == 1).all())
    q1, k1, v1 = rand(NL, 2, H, D), rand(NL, 2, G, D), rand(NL, 2, G, D)
    o1, l1 = torch.empty_like(q1), torch.empty(NL, 2, H, device=dev)

    def token():
        pg.pages_grow(c, slots, ones, st, pws)
        pg.pages_write(c, slots, ones, k1, v1, pg.rows_layout(k1), grown=st)
        pg.attend_window(c, slots, ones, q1, 0, 0, o1, aws, lse=l1)
        pg.mass_add(c, slots, ones, q1, l1, 0, 0, mass, mass, aws, grown=st)

    def step(run, want, tag):
        """`want`: the statuses.  Sequences that grew have the reference's weights."""
        say(f"{tag}: lengths {c.length.tolist()}, statuses {want} expected")
        q1.copy_(rand(NL, 2, H, D))
        k1.copy_(rand(NL, 2, G, D))
        held, old = Held(c, mass), mass.clone()
        run()
        torch.cuda.synchronize()
        assert st.tolist() == want, tag
        for b in slots:
            if want[b]:
                assert torch.equal(bits(mass[:, b]), bits(old[:, b])), f"{tag}: masses of {b}"
        grew = [b for b in slots if not want[b]]
        held.weights(mass, l1[:, grew].contiguous(), q1[:, grew].contiguous(), grew, [1] * len(grew), 0, 0, tag)
        sound(c)

    step(token, [0, 1], "eager")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        token()
    step(g.replay, [0, 1], "replay")
    step(g.replay, [1, 1], "both full")
    pg.pages_free(c, [0], keep_first=2 * P)          # two pages back
    step(g.replay, [0, 0], "room")
    step(g.replay, [0, 0], "room again")
    assert c.length.tolist() == [2 * P + 2, 3 * P + 2]
    # what was kept decides what is evicted
    idx = torch.empty(NL, 1, 10, dtype=torch.int32, device=dev)
    pg.pages_free(c, [0])
    ews = torch.empty(pg.evict_workspace_bytes(c, 1, 10, 0, 4), dtype=torch.uint8, device=dev)
    old, n = mass[:, 1].clone(), 3 * P + 2
    pg.pages_evict(c, [1], mass, 10, 0, 4, idx, st, ews)
    torch.cuda.synchronize()
    top = torch.topk(old[:, :n - 4], 10).indices.sort().values
    assert st.tolist()[0] == 0 and torch.equal(idx[:, 0].long(), top)


def test_the_binding_refuses():
    c = Case(20, [40], [2], 4, 2, 64, 16)
    c.upload()
    lse = torch.from_numpy(c.lse).cuda()
    call = lambda g: pg.mass_add(c.c, c.slots, c.rows, c.qd, lse, 0, 0, c.md, c.md, None, max_len=40, grown=g)
    i32 = dict(dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="grown"):
        call(torch.zeros(0, **i32))
    with pytest.raises(ValueError, match="grown"):
        call(torch.zeros(1, device="cuda"))
    call(torch.zeros(1, **i32))
    torch.cuda.synchronize()
