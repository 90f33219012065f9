"""Accepted drafts weighed with the log-sums that the tree's attention gave their rows:
an accepted row saw the prefix, its ancestors and itself, which are the tokens before
it once the path is compacted.  Against 64 bits, with the exact log-sums there.

Bound: a log-sum of the attention is off by E + 2 u |lse|, E = 2 (d + 8) u (X + 1) +
3 (n + 64) u as in the tests of the attentions, and a weight by e^that - 1; the added
weights are off as in test_mass_gpu.py from there on."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import fp4_cache as F  # noqa: E402
from oracle import evict_oracle as EO  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp4"])
@pytest.mark.parametrize("T,H,G,d", [(6, 4, 2, 64), (24, 14, 2, 128), (60, 4, 4, 64)])
def test_the_tree_s_log_sums(dtype, T, H, G, d):
    NL, P, lens = 2, 16, [70, 33, 150]
    dt = {"bf16": torch.bfloat16, "f32": torch.float32, "fp4": pg.FP4}[dtype]
    dev, gen, r = torch.device("cuda"), torch.Generator(device="cuda").manual_seed(T), np.random.default_rng(T)
    c = pg.new_cache(NL, 60, P, G, d, 3, 16, H, dtype=dt)
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev).to(c.dtype)
    slots, st = [0, 1, 2], torch.zeros(3, dtype=torch.int32, device=dev)
    pws = torch.empty(pg.pages_workspace_bytes(c, 3), dtype=torch.uint8, device=dev)
    for new in (lens, [T] * 3):
        pg.pages_grow(c, slots, new, st, pws)
        k, v = rand(NL, sum(new), G, d), rand(NL, sum(new), G, d)
        pg.pages_write(c, slots, new, k, v, pg.rows_layout(k), grown=st)
    # trees, their ancestors' bits, and of each a path from a root down
    parents = [[int(r.integers(max(-1, j - 4), j)) for j in range(T)] for _ in slots]
    bits, paths = [], []
    for par in parents:
        own = []
        for j in range(T):
            own.append((own[par[j]] if par[j] >= 0 else 0) | 1 << j)
        bits += own
        tip = int(r.integers(T // 2, T))
        paths.append([j for j in range(T) if own[tip] >> j & 1])
    mask = torch.from_numpy(np.array(bits, dtype=np.uint64).reshape(-1, 1).view(np.int64)).to(dev)
    q = rand(NL, 3 * T, H, d)
    out, lse = torch.empty_like(q), torch.empty(NL, 3 * T, H, device=dev)
    rows = [len(p) for p in paths]
    need = max(pg.attend_workspace_bytes(c, [T] * 3, c.cap), pg.mass_workspace_bytes(c, rows, c.cap), 16)
    ws = torch.empty(need, dtype=torch.uint8, device=dev)
    pg.attend_tree(c, slots, [T] * 3, q, mask, out, ws, lse=lse)
    B = max(rows)
    idx = torch.tensor([p + [0] * (B - len(p)) for p in paths], dtype=torch.int32, device=dev)
    pg.pages_compact(c, slots, idx.repeat(NL, 1, 1), st, pws, span=[T] * 3, grown=st,
                     counts=torch.tensor(rows, dtype=torch.int32, device=dev))
    at = torch.tensor([b * T + j for b, p in enumerate(paths) for j in p], device=dev)
    mass = torch.rand(NL, 3, c.cap, generator=gen, device=dev)
    old = mass.double().cpu().numpy()
    pg.mass_add(c, slots, rows, q[:, at].contiguous(), lse[:, at].contiguous(), 0, 0, mass, mass, ws, grown=st)
    torch.cuda.synchronize()
    assert st.tolist() == [0, 0, 0] and c.length.tolist() == [n + k for n, k in zip(lens, rows)]
    m, num = F.model_of(c)
    got, qa, first, worst = mass.double().cpu().numpy(), q[:, at].double().cpu().numpy(), 0, 0.0
    for b, k in zip(slots, rows):
        n = int(m.len[b])
        see = PO.see_window(n, k, 0, 0)
        for l in range(NL):
            mine = qa[l, first:first + k]
            _, exact, _, X = PO.attend(m, b, mine, see, num, l)
            add, size = EO.weights(m, b, mine, exact, see, num, l)
            want = np.where(np.arange(n) < n - k, old[l, b, :n], 0) + add
            E = np.max(2 * (d + 8) * U * (X + 1) + 3 * (n + 64) * U + 2 * U * np.abs(exact))
            tol = 1.01 * ((E + (d + 8) * U * (size + 1) + (k * H + 64) * U) * add + 2 * U * want) + 1e-37
            worst = max(worst, float(np.max(np.abs(got[l, b, :n] - want) / tol)))
            assert worst <= 1, f"slot {b} layer {l}: {worst:.2f} of the bound"
        first += k
    print(f"[tree] {dtype} T {T} paths {rows}: {worst:.3f} of the bound", flush=True)
