"""Attention of many rows over several long sequences of very different
lengths, whose steps the device divides by the lengths that it finds: against
the definition in 64 bits, head by head on the GPU.  Bounds as derived in
test_attend_gpu.py: exact bf16 products summed in float32, X the largest sum_j
|q_j k_j| / sqrt(d) of a row, u = 2^-24, n its tokens,
  E = 2 (d + 8) u (X + 1) + 3 (n + 64) u, |dlse| <= E + 2 u |lse|,
  |do| <= (E + 2^-8) sum_t p_t |v_t| + 2^-8 |o|."""

import math

import pytest

torch = pytest.importorskip("torch")

from paper_2606_01790_amd import paged as pg  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
H, G, D, P = 8, 2, 128, 64
STEP, TILE, SLOTS = 64, 128, 512      # tokens of a step, rows of a tile, blocks at a time


class Batch:
    def __init__(self, seed, lens, rows, nl, words=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        h = torch.Generator().manual_seed(seed)
        self.lens, self.rows, self.nl = lens, rows, nl
        need = [-(-n // P) for n in lens]
        perm = torch.randperm(sum(need) + 3, generator=h).to(torch.int32)
        table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32)
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = perm[at:at + m]
            at += m
        new = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
        k, v = new(nl, sum(need) + 3, G, P, D), new(nl, sum(need) + 3, G, P, D)
        refs = torch.zeros(sum(need) + 3, dtype=torch.int32, device="cuda")
        self.c = pg.Cache(k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), refs, H)
        self.tot = sum(rows)
        self.q = new(nl, self.tot, H, D)
        if words:
            bits = torch.randint(-2 ** 63, 2 ** 63 - 1, (self.tot, words), generator=h)
            own = torch.cat([torch.arange(T) for T in rows])          # its own bit, and random others
            for w in range(words):
                bits[:, w] |= torch.where(own // 64 == w, torch.ones((), dtype=torch.int64) << own % 64, 0)
            self.mask = bits.cuda()
        self.out = torch.full((nl, self.tot, H, D), math.nan, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((nl, self.tot, H), math.nan, device="cuda")

    def workspace(self):
        self.need = pg.attend_workspace_bytes(self.c, self.rows, max(self.lens))
        return torch.full((max(self.need, 16),), 255, dtype=torch.uint8, device="cuda")

    def chosen(self, ws):
        """The steps of a split: what the device chose, at the workspace's end,
        and what the rule says: the least with which the blocks of all splits
        fit the slots, or as many times them as leave 96 steps to a block."""
        tiles = [-(-T * H // G // TILE) for T in self.rows]
        steps = [-(-n // STEP) for n in self.lens]
        lgs = self.nl * G
        work = sum(t * s for t, s in zip(tiles, steps))
        rounds = max(1, round(work * lgs / (SLOTS * 96)))
        target = max(1, int(SLOTS * rounds / lgs))
        per = quotient = max(4, -(-work // target))
        while sum(t * -(-s // per) for t, s in zip(tiles, steps)) > target:
            per += max(1, per >> 4)
        splits = self.need // (sum(tiles) * lgs * TILE * (D + 2) * 4)
        return int(ws[self.need - 256:self.need - 252].view(torch.int32)), per, quotient, rounds, splits

    def check(self, tag, see_of):
        at, worst = 0, 0.0
        for b, (n, T) in enumerate(zip(self.lens, self.rows)):
            t = torch.arange(n, device="cuda")
            page, row = self.c.table[b].long()[t // P], t % P
            see = see_of(b, at, n, T, t)
            for layer in range(self.nl):
                for h in range(H):
                    g = h * G // H
                    K = self.c.k[layer, page, g, row].double()
                    V = self.c.v[layer, page, g, row].double()
                    q = self.q[layer, at:at + T, h].double()
                    kt = K.t().contiguous()
                    x = q @ kt / math.sqrt(D)
                    X = (q.abs() @ kt.abs() / math.sqrt(D)).masked_fill(~see, 0).amax(1)
                    x.masked_fill_(~see, -math.inf)
                    lse = torch.logsumexp(x, 1)
                    p = torch.softmax(x, 1)
                    o, mass = p @ V, p @ V.abs()
                    E = 2 * (D + 8) * U * (X + 1) + 3 * (n + 64) * U
                    tol = ((E[:, None] + 2.0 ** -8) * mass + 2.0 ** -8 * o.abs()) * (1 + 2.0 ** -7)
                    worst = max(worst, float(((self.out[layer, at:at + T, h].double() - o).abs() / tol).max()))
                    el = (self.lse[layer, at:at + T, h].double() - lse).abs() / (E + 2 * U * lse.abs())
                    assert worst <= 1 and float(el.max()) <= 1, f"{tag}: slot {b} layer {layer} head {h}"
            at += T
        print(f"[attend] {tag}: {worst:.3f} of the bound", flush=True)


def causal(window, sinks):
    def see(b, at, n, T, t):
        p = torch.arange(n - T, n, device="cuda")[:, None]
        return (t <= p) & ((t > p - window) | (t < sinks)) if window else t <= p
    return see


# lengths, rows, layers; whether the work is more than one round of blocks, and
# whether it decides the steps, or the longest sequence by the number of splits
BATCHES = [([2000, 12000, 6007], [700, 1000, 9], 2, False, True),
           ([12000, 11500, 12040], [1100, 1050, 1000], 2, True, True),
           ([24000, 901, 13000, 64], [1200, 901, 650, 64], 2, True, False)]


@pytest.mark.parametrize("lens,rows,nl,more,decides", BATCHES)
def test_chunks_behind_sequences_of_unequal_length(lens, rows, nl, more, decides):
    c = Batch(len(lens) + nl, lens, rows, nl)
    ws = c.workspace()
    slots = list(range(len(lens)))
    for window, sinks in ((0, 0), (3000, 70)):
        c.out.fill_(math.nan)
        print(f"[attend] lens {lens} rows {rows} window {window}", flush=True)
        pg.attend_window(c.c, slots, rows, c.q, window, sinks, c.out, ws, lse=c.lse, max_len=max(lens))
        torch.cuda.synchronize()
        if not window:
            got, per, quotient, rounds, splits = c.chosen(ws)
            assert got == per and quotient > 4 and (rounds > 1) == more and splits > 1
            assert (per > -(-max(lens) // STEP // splits)) == decides
        c.check(f"{lens} window {window}", causal(window, sinks))
        again = c.out.clone()
        pg.attend_window(c.c, slots, rows, c.q, window, sinks, c.out, ws, lse=c.lse, max_len=max(lens))
        torch.cuda.synchronize()
        assert torch.equal(again, c.out)


def test_wide_trees_over_sequences_of_unequal_length():
    lens, rows = [9000, 700, 25000, 256], [200, 77, 130, 256]
    c = Batch(7, lens, rows, 2, words=4)
    ws = c.workspace()
    pg.attend_tree(c.c, [0, 1, 2, 3], rows, c.q, c.mask, c.out, ws, lse=c.lse, max_len=max(lens))
    torch.cuda.synchronize()
    got, per, quotient, _, splits = c.chosen(ws)
    assert got == per and quotient > 4 and splits > 1

    def see(b, at, n, T, t):
        j = t - (n - T)
        bit = c.mask[at:at + T][:, j.clamp(0) // 64] >> (j.clamp(0) % 64) & 1
        return (j < 0) | (bit == 1)

    c.check("trees", see)


def test_one_long_sequence_of_many_rows():
    """Splits that the host chose, in more than one round of blocks."""
    for n, T in ((20011, 900), (9000, 65)):
        c = Batch(n, [n], [T], 1)
        ws = c.workspace()
        pg.attend_window(c.c, [0], [T], c.q, 0, 0, c.out, ws, lse=c.lse, max_len=n)
        torch.cuda.synchronize()
        assert c.need > 0
        c.check(f"one of {n}", causal(0, 0))
