"""Attention at the ends of its ranges: a sequence of 2^26 tokens of which a
window has dropped nearly all pages, and as many row tiles as a call takes."""

import math

import pytest

torch = pytest.importorskip("torch")

from paper_2606_01790_amd import paged as pg  # noqa: E402
from test_attend_gpu import TYPE, U  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,T", [("bf16", 3), ("bf16", 40), ("f32", 3)])
def test_a_sequence_of_as_many_tokens_as_a_table_holds(dtype, T):
    """The first page and the last two are there, of 65,536: causal, under a
    window with sinks, and as a tree, against the tokens that are left.
    Bounds as derived in test_attend_gpu.py."""
    P, D, H, n = 1024, 64, 4, 1 << 26
    g = torch.Generator(device="cuda").manual_seed(T)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda").to(TYPE[dtype])
    k, v, q = new(1, 3, 1, P, D), new(1, 3, 1, P, D), new(1, T, H, D)
    table = torch.full((1, n // P), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, -2], table[0, -1] = 2, 0, 1
    c = pg.Cache(k, v, table, torch.tensor([n], dtype=torch.int32, device="cuda"),
                 torch.ones(3, dtype=torch.int32, device="cuda"), H)
    ws = torch.full((max(16, pg.attend_workspace_bytes(c, [T], n)),), 255, dtype=torch.uint8, device="cuda")
    t = torch.cat([torch.arange(P), torch.arange(n - 2 * P, n)]).cuda()
    K = torch.cat([k[0, 2, 0], k[0, 0, 0], k[0, 1, 0]]).double()
    V = torch.cat([v[0, 2, 0], v[0, 0, 0], v[0, 1, 0]]).double()
    p = torch.arange(n - T, n, device="cuda")[:, None]
    mask = torch.tensor([[(1 << i + 1) - 1 & 0x5555555555] for i in range(T)], dtype=torch.int64, device="cuda")
    j = t - (n - T)
    tree = (j < 0) | ((mask >> j.clamp(0, 63)) & 1 == 1)
    for tag, see in (("causal", t <= p), ("window", (t <= p) & ((t > p - 1500) | (t < 5))), ("tree", tree)):
        print(f"[attend] {dtype} {T} rows {tag}", flush=True)
        out, lse = torch.full_like(q, math.nan), torch.full((1, T, H), math.nan, device="cuda")
        if tag == "tree":
            pg.attend_tree(c, [0], [T], q, mask, out, ws, lse=lse, max_len=n)
        else:
            w, s = (1500, 5) if tag == "window" else (0, 0)
            pg.attend_window(c, [0], [T], q, w, s, out, ws, lse=lse, max_len=n)
        torch.cuda.synchronize()
        kt = K.t().contiguous()
        for h in range(H):
            x = q[0, :, h].double() @ kt / math.sqrt(D)
            X = (q[0, :, h].double().abs() @ kt.abs() / math.sqrt(D)).masked_fill(~see, 0).amax(1)
            x = x.masked_fill(~see, -math.inf)
            w = torch.softmax(x, 1)
            o, mass, ref = w @ V, w @ V.abs(), torch.logsumexp(x, 1)
            E = 2 * (D + 8) * U * (X + 1) + 3 * (len(t) + 64) * U
            low = 2.0 ** -8 if dtype == "bf16" else U
            tol = (E[:, None] * mass + low * o.abs() + (2.0 ** -8 * mass if dtype == "bf16" else 0)) * 1.01
            assert bool(((out[0, :, h].double() - o).abs() <= tol).all()), f"{tag} head {h}"
            assert bool(((lse[0, :, h].double() - ref).abs() <= E + 2 * U * ref.abs()).all()), f"{tag} head {h}"


def test_as_many_row_tiles_as_a_call_takes():
    """4,096 layers (of one memory), 16 groups, 128 sequences of one token: 2^23
    row tiles, each a block.  Every layer gives what the first does, and that
    is what a call of one layer gives; one sequence more is refused."""
    NL, G, P, D, n = 4096, 16, 16, 64, 128
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn(1, n, G, P, D, generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn(1, n, G, P, D, generator=g, device="cuda").to(torch.bfloat16)
    i32 = dict(dtype=torch.int32, device="cuda")
    args = (torch.arange(n, **i32)[:, None].contiguous(), torch.arange(n, **i32) % 17, torch.ones(n, **i32), G)
    one = pg.Cache(k, v, *args)
    all_ = pg.Cache(k.expand(NL, -1, -1, -1, -1), v.expand(NL, -1, -1, -1, -1), *args)
    assert all_.c.layer_stride == 0
    q1 = torch.randn(1, n, G, D, generator=g, device="cuda").to(torch.bfloat16)
    o1, l1 = torch.full_like(q1, math.nan), torch.full((1, n, G), math.nan, device="cuda")
    slots, rows = list(range(n)), [1] * n
    pg.attend_window(one, slots, rows, q1, 0, 0, o1, None, lse=l1, max_len=16)
    q = q1.expand(NL, -1, -1, -1).contiguous()
    out, lse = torch.full_like(q, math.nan), torch.full((NL, n, G), math.nan, device="cuda")
    assert pg.attend_workspace_bytes(all_, rows, 16) == 0
    pg.attend_window(all_, slots, rows, q, 0, 0, out, None, lse=lse, max_len=16)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(o1).all()) and bool((o1[0, args[1] == 0] == 0).all())
    assert bool((out == o1).all()) and bool((lse == l1).all())
    with pytest.raises(pg.StarKVError, match="E_PARAM"):
        pg.attend_window(all_, slots + [0], rows + [1], torch.empty(NL, n + 1, G, D, dtype=q.dtype, device="cuda"),
                         0, 0, torch.empty(NL, n + 1, G, D, dtype=q.dtype, device="cuda"), None, max_len=16)
