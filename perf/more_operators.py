"""The timed calls of long generations: caches held in 4 bits, and eviction.

A GUI agent's trajectory outgrows the cache that its generation reads.  Two
ways make room.  The cache is held in 4 bits (elements e2m1 with a power of two
for every 32 of a row), written, read back and attended to in its pages.  And
of a running generation the tokens that the attention has weighted least are
evicted: every attention's weights are added up per cached token, and now and
then the heaviest tokens, the sinks and the recent ones are kept.  Shapes are
those of the repository's workloads (28 layers, 28 query heads on 4 KV groups
of size 128; screenshots of 69x39 visual tokens; a 20% budget) and generic ones
around them.  Kinds of a case:
  window  attention of the last `rows` tokens per sequence over a 4-bit cache
  tree    attention of `rows` drafted tokens per sequence over a 4-bit cache
  write   K and V of the last `rows` tokens per sequence into a 4-bit cache, and
          the rows that it now stands for read back
  mass    the attention weights of the last `rows` tokens per sequence added to
          the accumulated ones of every cached token
  evict   sequences forked with their accumulated weights, and each fork cut down
          to a budget by them
Every pass ends in the state that it ended in before, so it can be run again.
"""

import math

import torch

own = False      # True: the framework's calls; False: the plain forms

DEV = "cuda"
SHORT = 3        # the status of a sequence that is no longer than what eviction keeps


# ------------------------------------------------------------------ cases

def _case(name, kind, layers=1, seqs=1, lo=1, hi=1, rows=1, ragged=False, H=28, G=4, d=128, P=64,
          cache="fp4", window=0, sinks=0, pct=20, recent=32):
    """Lengths are spread from lo to hi over the sequences; `ragged` spreads
    the rows from 1 to `rows` likewise."""
    c = dict(kind=kind, layers=layers, seqs=seqs, lo=lo, hi=hi, rows=rows, ragged=ragged, H=H, G=G,
             d=d, P=P, cache=cache, window=window, sinks=sinks, pct=pct, recent=recent)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a short conversation, one layer: latency
        _case("fp4-window-1l-short", "window", lo=600, hi=600),
        # one token over fifteen screenshots, uncompressed, all layers
        _case("fp4-window-28l-full-15f", "window", layers=28, lo=40941, hi=40941),
        # one token each for a batch of conversations of every length, one layer
        _case("fp4-window-1l-32seq-decode", "window", seqs=32, lo=37, hi=40941),
        # one screenshot and its text appended to five, one layer of a prefill
        _case("fp4-window-1l-append-frame", "window", lo=13711, hi=13711, rows=2755, window=8192,
              sinks=256),
        # a drafted tree over five screenshots, all layers
        _case("fp4-tree-28l-5f", "tree", layers=28, lo=13711, hi=13711, rows=24),
        # small trees of a batch, head size 64, small pages
        _case("fp4-tree-1l-d64-16seq", "tree", seqs=16, lo=500, hi=13711, rows=7, ragged=True, H=16,
              G=4, d=64, P=32),
        # the prompt of five screenshots
        _case("fp4-write-28l-5f", "write", layers=28, lo=13711, hi=13711, rows=13711),
        # the next token of a batch, one layer: latency
        _case("fp4-write-1l-16seq", "write", seqs=16, lo=500, hi=13711, rows=1),
        # the weights of a decoded token of each of a batch, all layers
        _case("mass-28l-16seq-decode", "mass", layers=28, seqs=16, lo=500, hi=2747, cache="bf16"),
        # the weights of a screenshot's rows over five others, one layer of a prefill
        _case("mass-1l-append-frame", "mass", lo=13711, hi=13711, rows=2755, cache="bf16"),
        # two conversations of five and four screenshots cut down to the stage's budget
        _case("evict-28l-2seq", "evict", layers=28, seqs=2, lo=10956, hi=13711, cache="bf16", sinks=4),
        # a batch of short ones, some of which fit as they are, one layer: latency
        _case("evict-1l-16seq", "evict", seqs=16, lo=100, hi=1500, cache="bf16", sinks=4, pct=40),
    ]


# a drawn case costs no more than the largest listed one
_MOST_SCORES = 28 * 2755 * 13711
_MOST_TOKENS = 28 * 40941


def draw(rng):
    logint = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    kind = rng.choice(["window", "window", "tree", "write", "mass", "mass", "evict"])
    H, G = rng.choice([(28, 4), (28, 4), (32, 8), (16, 2), (12, 2), (16, 16), (14, 2), (6, 1)])
    d = 64 if (H, G) == (14, 2) else rng.choice([128, 128, 128, 64])
    P = rng.choice([16, 32, 64, 64, 128, 256])
    layers, seqs = logint(1, 28), logint(1, 32)
    hi = logint(16, 41000)
    lo = rng.choice([hi, logint(8, hi) if hi > 8 else hi])
    cache = "fp4"
    if kind == "mass":
        cache = rng.choice(["bf16", "bf16", "fp4", "f32"])
    if kind == "evict":
        cache = rng.choice(["bf16", "bf16", "f32"])
    c = _case(None, kind, layers, seqs, lo, hi, 1, rng.random() < 0.5, H, G, d, P, cache)
    if kind == "tree":
        c["rows"] = min(lo, logint(1, 64))
    elif kind in ("window", "mass"):
        # a decoded token, a few, or a chunk of a prefill
        c["rows"] = min(lo, rng.choice([1, logint(1, 16), logint(1, 4000)]))
        c["window"] = rng.choice([0, 0, logint(1, 8192)])
        c["sinks"] = rng.choice([0, 4, logint(1, 512)])
        if c["rows"] > 64:
            c["layers"], c["seqs"] = min(layers, 4), min(seqs, 4)
    elif kind == "write":
        c["rows"] = rng.choice([1, logint(1, lo), lo])
        c["layers"], c["seqs"] = min(layers, 14), min(seqs, 16)
    else:
        c["seqs"], c["pct"] = min(seqs, 4), rng.choice([10, 20, 40])
        c["sinks"], c["recent"] = rng.choice([0, 4, 64]), rng.randint(0, 128)
        c["hi"], c["lo"] = max(hi, 300), max(lo, 100)
    # the plain form pads to the longest sequence and the largest row count
    while c["layers"] * c["seqs"] * c["hi"] > _MOST_TOKENS // (3 if cache != "fp4" or kind == "write" else 1):
        if c["layers"] > 1:
            c["layers"] = (c["layers"] + 1) // 2
        else:
            c["seqs"] = (c["seqs"] + 1) // 2
    if kind in ("tree", "window", "mass"):
        while c["layers"] * c["seqs"] * H * c["rows"] * c["hi"] > _MOST_SCORES:
            if c["layers"] * c["seqs"] > 1:
                c["layers"], c["seqs"] = (c["layers"] + 1) // 2, (c["seqs"] + 1) // 2
            else:
                c["rows"] = (c["rows"] + 1) // 2
    return c


# ------------------------------------------------------------------ sizes

def _spread(a, b, n):
    return [a + (b - a) * i // max(n - 1, 1) for i in range(n)]


def _lens(c):
    # the longest first: no order of a batch is promised
    return _spread(c["hi"], c["lo"], c["seqs"])


def _rows(c):
    return _spread(1, c["rows"], c["seqs"]) if c["ragged"] else [c["rows"]] * c["seqs"]


def _words(c):
    return (max(_rows(c)) + 63) // 64


def _keep(c):
    """Heavy tokens that eviction keeps: a share of the longest sequence."""
    return c["pct"] * c["hi"] // 100


def _row_bytes(c):
    """Of a K (or V) row of one group."""
    return {"bf16": 2 * c["d"], "f32": 4 * c["d"], "fp4": c["d"] // 2 + c["d"] // 32}[c["cache"]]


def _visible(c, n, T):
    """Cached tokens that some row sees, and the (row, token) pairs seen."""
    if c["kind"] == "tree":
        return n, T * (n - T) + T * (T + 1) // 2
    w, s = c["window"] or n, c["sinks"] if c["window"] else 0
    lo = max(n - T - w + 1, 0)
    p = torch.arange(n - T, n, dtype=torch.int64)
    pairs = int((torch.clamp(p + 1, max=w) + torch.clamp(p + 1 - w, 0, s)).sum())
    return n - lo + min(s, lo), pairs


def work(case):
    c = case
    nl, H, G, d, P, kind = c["layers"], c["H"], c["G"], c["d"], c["P"], c["kind"]
    row, e = _row_bytes(c), 4 if c["cache"] == "f32" else 2
    by = fl = 0
    for n, T in zip(_lens(c), _rows(c)):
        if kind in ("tree", "window"):
            seen, pairs = _visible(c, n, T)
            by += nl * (seen * 2 * G * row + 2 * T * H * d * e + 4 * T * H) + 4 * (seen + P - 1) // P
            by += 8 * T * _words(c) if kind == "tree" else 0
            fl += nl * 4 * H * d * pairs
        elif kind == "mass":
            seen, pairs = _visible(c, n, T)
            by += nl * (seen * G * row + T * H * (d * e + 4) + 8 * n - 4 * T) + 4 * (seen + P - 1) // P
            fl += nl * 2 * H * d * pairs
        elif kind == "write":
            # the rows given, their 4 bits written and read, the rows given back
            by += nl * 2 * G * T * (2 * 2 * d + 2 * row) + 8 * (T + P - 1) // P
        else:
            if n > _keep(c) + c["sinks"] + c["recent"]:
                kept = _keep(c) + c["sinks"] + c["recent"]
                by += nl * (kept * (2 * 2 * G * row + 8) + 4 * _keep(c))
            # its weights copied with the fork, then looked through
            by += nl * 12 * n + 8 * (n + P - 1) // P
    return {"bytes": by, "flops": fl}


# ------------------------------------------------------------------ rows in 4 bits

def _to_fp4(x):
    """x [.., d] float32 as (codes [.., d] uint8, scale exponents + 127 [.., d/32]).
    The power of two is that at which the block's largest magnitude lies in
    [3.5, 7] or rounds to there; elements go to the nearest of 0, 0.5, 1, 1.5, 2,
    3, 4, 6, ties to the even code, beyond 6 to 6.  A block that holds an infinity or
    NaN has the byte 255."""
    y = x.unflatten(-1, (-1, 32))
    top = y.abs().amax(-1)
    bits = top.contiguous().view(torch.int32)
    byte = ((bits + 0x1FFFFF) >> 23).sub_(2).clamp_(2, 252)
    y = y.abs() * ((254 - byte) << 23).view(torch.float32).unsqueeze(-1)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5)
            + (y >= 3.5) + (y > 5))
    code |= torch.signbit(x).unflatten(-1, (-1, 32)).to(torch.uint8) << 3
    fine = torch.isfinite(top)
    code = torch.where(fine.unsqueeze(-1), code, torch.zeros_like(code))
    return code.flatten(-2), torch.where(fine, byte, torch.full_like(byte, 255)).to(torch.uint8)


_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _from_fp4(data, scale, dtype=torch.float32):
    """Packed rows [.., d/2] and their scales [.., d/32] as numbers [.., d]."""
    grid = torch.tensor(_GRID + [-g for g in _GRID], dtype=dtype, device=data.device)
    code = torch.stack([data & 15, data >> 4], -1).flatten(-2)
    s = (scale.to(torch.int32) << 23).view(torch.float32).to(dtype)
    s = torch.where(scale == 255, torch.full_like(s, math.nan), s)
    return (grid[code.int()].unflatten(-1, (-1, 32)) * s.unsqueeze(-1)).flatten(-2)


def _pack(code):
    return code[..., 0::2] | code[..., 1::2] << 4


def _planes(pool, c):
    """A pool [layers, pages, G, bytes]: its packed rows [.., P, d/2] and their
    scales [.., P, d/32], as views."""
    n = c["P"] * c["d"] // 2
    return pool[..., :n].unflatten(-1, (c["P"], -1)), pool[..., n:].unflatten(-1, (c["P"], -1))


# ------------------------------------------------------------------ inputs

def _fill(c, shape, g):
    """A pool of keys or values, layer by layer."""
    nl, n_pages, G, P, d = shape
    dt = {"bf16": torch.bfloat16, "f32": torch.float32, "fp4": torch.uint8}[c["cache"]]
    if c["cache"] != "fp4":
        pool = torch.empty(shape, dtype=dt, device=DEV)
        for l in range(nl):
            pool[l].normal_(generator=g)
        return pool
    pool = torch.empty(nl, n_pages, G, P * (d // 2 + d // 32), dtype=dt, device=DEV)
    data, scale = _planes(pool, c)
    for l in range(nl):
        x = torch.empty(shape[1:], dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        code, byte = _to_fp4(x.float())
        data[l], scale[l] = _pack(code), byte
    return pool


def prepare(case, seed):
    """A pool whose pages lie in no order, as after some time of serving."""
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    nl, n, H, G, d, P, kind = c["layers"], c["seqs"], c["H"], c["G"], c["d"], c["P"], c["kind"]
    lens, rows = _lens(c), _rows(c)
    pages = [(x + P - 1) // P for x in lens]
    made = 1 if kind == "evict" else 0                       # forks per sequence
    width = max(pages) + 1
    kept = _keep(c) + c["sinks"] + c["recent"]
    room = sum((kept + P - 1) // P for x in lens if x > kept) if made else 0
    n_pages = sum(pages) + room + 3
    shape = (nl, n_pages, G, P, d)
    k, v = _fill(c, shape, g), _fill(c, shape, g)
    n_slots = n * (1 + made)
    slots = torch.randperm(n_slots, generator=host)[:n].tolist()
    kids = [i for i in range(n_slots) if i not in set(slots)]
    table = torch.full((n_slots, width), -1, dtype=torch.int32)
    perm = torch.randperm(n_pages, generator=host, dtype=torch.int64).to(torch.int32)
    refs, length = torch.zeros(n_pages, dtype=torch.int32), torch.zeros(n_slots, dtype=torch.int32)
    at = 0
    for b in range(n):
        table[slots[b], :pages[b]] = perm[at:at + pages[b]]
        length[slots[b]] = lens[b]
        at += pages[b]
        if kind in ("window", "mass") and c["window"]:
            # the pages that no row will see again are freed
            j = torch.arange(pages[b])
            gone = (j * P >= c["sinks"]) & ((j + 1) * P <= lens[b] - rows[b] - c["window"] + 1)
            table[slots[b], :pages[b]][gone] = -1
    refs[table[table >= 0].long()] = 1
    s = dict(c=c, k=k, v=v, table=table.to(DEV), refs=refs.to(DEV), length=length.to(DEV), slots=slots,
             lens=lens, rows=rows, longest=max(lens))
    tot = sum(rows)
    if kind in ("tree", "window", "mass"):
        # logits of the spread that trained heads have
        dt = torch.float32 if c["cache"] == "f32" else torch.bfloat16
        s["q"] = (1.5 * torch.randn(nl, tot, H, d, generator=g, device=DEV)).to(dt)
    if kind == "tree":
        s["mask"] = _tree(rows, _words(c), host).to(DEV)
    if kind == "write":
        s["kn"] = torch.empty(nl, tot, G, d, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        # values are spread over some powers of two, as from one channel to the next
        s["vn"] = torch.empty_like(s["kn"]).normal_(generator=g)
        s["vn"].mul_(torch.exp2(torch.randint(-6, 7, (d,), generator=g, device=DEV).float())
                     .to(torch.bfloat16))
        s["k1"], s["v1"] = torch.zeros_like(s["kn"]), torch.zeros_like(s["kn"])
    if kind in ("mass", "evict"):
        # weights that earlier tokens have left: a few tokens have most of them
        s["mass"] = torch.rand(nl, n_slots, width * P, generator=g, device=DEV).pow_(6).mul_(9)
    if kind == "mass":
        s["out"] = torch.zeros_like(s["mass"])
        s["lse"] = _log_sums(s)
    if kind == "evict":
        s["kids"], s["src"] = kids, slots
        s["mass"][:, kids] = 0
    return s


def _log_sums(s):
    """What the attention of these rows gave beside its output."""
    c, out = s["c"], torch.empty(s["q"].shape[:3], device=DEV)
    G, at = c["G"], 0
    for slot, n, T in zip(s["slots"], s["lens"], s["rows"]):
        t = torch.arange(n, device=DEV)
        page = s["table"][slot].long()[t // c["P"]]
        see = _sees(c, n, T) & (page >= 0)
        for l in range(c["layers"]):
            K = _rows_of(s, s["k"], l, page.clamp_min(0), t % c["P"]).transpose(0, 1).contiguous()
            for g in range(G):
                q = s["q"][l, at:at + T, g * c["H"] // G:(g + 1) * c["H"] // G].float()
                x = (q @ K[g].t().contiguous()).mul_(1 / math.sqrt(c["d"]))      # [T, hpg, n]
                x.masked_fill_(~see[:, None], -math.inf)
                out[l, at:at + T, g * c["H"] // G:(g + 1) * c["H"] // G] = torch.logsumexp(x, -1)
        at += T
    return out


def _sees(c, n, T):
    t, p = torch.arange(n, device=DEV), torch.arange(n - T, n, device=DEV)[:, None]
    see = t <= p
    if c["window"]:
        see = see & ((t > p - c["window"]) | (t < c["sinks"]))
    return see


def _rows_of(s, pool, l, page, off, dtype=torch.float32):
    """Rows [m, G, d] of a layer as numbers."""
    if s["c"]["cache"] != "fp4":
        return pool[l, page, :, off].to(dtype)
    data, scale = _planes(pool[l], s["c"])
    return _from_fp4(data[page, :, off], scale[page, :, off], dtype)


def _parents(T, host):
    """A tree of T drafted tokens: token j hangs on an earlier one, most often
    on the one just before it."""
    r = torch.rand(T, generator=host).tolist()
    u = torch.rand(T, generator=host).tolist()
    return [-1 if j == 0 else (j - 1 if r[j] < 0.5 else int(u[j] * j)) for j in range(T)]


def _tree(rows, words, host):
    """Bits of each row's ancestors and itself, in 64-bit words."""
    out = []
    for T in rows:
        bits = []
        for j, p in enumerate(_parents(T, host)):
            bits.append((bits[p] if p >= 0 else 0) | 1 << j)
            out.append([(lambda x: x - (1 << 64) if x >> 63 else x)(bits[j] >> 64 * w & (1 << 64) - 1)
                        for w in range(words)])
    return torch.tensor(out, dtype=torch.int64)


# ------------------------------------------------------------------ the framework's calls

def _handle(s):
    """What a serving program makes once: the cache's handle, the workspace
    and the output buffers."""
    from paper_2606_01790_amd import paged as pg
    c, kind = s["c"], s["c"]["kind"]
    h = dict(pg=pg, cache=pg.Cache(s["k"], s["v"], s["table"], s["length"], s["refs"], c["H"], d=c["d"]))
    need = 16
    if kind in ("tree", "window"):
        h["out"] = torch.empty_like(s["q"])
        h["lse"] = torch.empty(s["q"].shape[:3], dtype=torch.float32, device=DEV)
        need = pg.attend_workspace_bytes(h["cache"], s["rows"], s["longest"])
    elif kind == "mass":
        need = pg.mass_workspace_bytes(h["cache"], s["rows"], s["longest"])
    elif kind == "evict":
        n = len(s["kids"])
        h["status"] = torch.zeros(n, dtype=torch.int32, device=DEV)
        h["idx"] = torch.empty(c["layers"], n, c["sinks"] + _keep(c), dtype=torch.int32, device=DEV)
        need = pg.evict_workspace_bytes(h["cache"], n, _keep(c), c["sinks"], c["recent"])
    else:
        h["lay"] = pg.rows_layout(s["kn"])
    h["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return h


def _run_own(s):
    if "handle" not in s:
        s["handle"] = _handle(s)
    h, c = s["handle"], s["c"]
    pg, cache, kind = h["pg"], h["cache"], c["kind"]
    if kind == "tree":
        pg.attend_tree(cache, s["slots"], s["rows"], s["q"], s["mask"], h["out"], h["ws"],
                       lse=h["lse"], max_len=s["longest"])
        return dict(o=h["out"], lse=h["lse"])
    if kind == "window":
        pg.attend_window(cache, s["slots"], s["rows"], s["q"], c["window"], c["sinks"], h["out"],
                         h["ws"], lse=h["lse"], max_len=s["longest"])
        return dict(o=h["out"], lse=h["lse"])
    if kind == "write":
        pg.pages_write(cache, s["slots"], s["rows"], s["kn"], s["vn"], h["lay"])
        pg.pages_read(cache, s["slots"], s["rows"], s["k1"], s["v1"], h["lay"])
        return dict(k=s["k1"], v=s["v1"])
    if kind == "mass":
        pg.mass_add(cache, s["slots"], s["rows"], s["q"], s["lse"], c["window"], c["sinks"], s["mass"],
                    s["out"], h["ws"], max_len=s["longest"])
        return s["out"]
    pg.pages_free(cache, s["kids"])
    pg.pages_fork(cache, s["src"], s["kids"])
    pg.mass_fork(cache, s["src"], s["kids"], s["mass"])
    pg.pages_evict(cache, s["kids"], s["mass"], _keep(c), c["sinks"], c["recent"], h["idx"], h["status"],
                   h["ws"])
    return dict(k=s["k"], v=s["v"], table=s["table"], length=s["length"], refs=s["refs"],
                status=h["status"], idx=h["idx"], mass=s["mass"])


# ------------------------------------------------------------------ the plain forms

def _long(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


def _plain_rows(s, pool, pages):
    """[nl, n, G, Lm, d] float32 of the pages [n, n_pg]"""
    c = s["c"]
    nl, (n, n_pg) = c["layers"], pages.shape
    if c["cache"] == "fp4":
        data, scale = _planes(pool, c)
        x = _from_fp4(data[:, pages], scale[:, pages])
    else:
        x = pool[:, pages].float()
    return x.permute(0, 1, 3, 2, 4, 5).reshape(nl, n, c["G"], n_pg * c["P"], c["d"])


def _plain_logits(s):
    """Logits [nl, n, G, Tm*hpg, Lm] with -infinity where a row does not see,
    and what lays rows out so."""
    c, q = s["c"], s["q"]
    nl, H, G, d, P = c["layers"], c["H"], c["G"], c["d"], c["P"]
    sel, T = _long(s["slots"]), _long(s["rows"])
    n = len(s["slots"])
    n_pg = (s["longest"] + P - 1) // P
    Lm, Tm, hpg = n_pg * P, max(s["rows"]), H // G
    pages = s["table"][sel, :n_pg].long()
    live = (pages >= 0).repeat_interleave(P, dim=1)                      # [n, Lm]
    pages = pages.clamp_min(0)
    K = _plain_rows(s, s["k"], pages)
    first = T.cumsum(0) - T
    i = torch.arange(Tm, device=DEV)
    flat = (first[:, None] + i.clamp_max(Tm)).clamp_max(q.shape[1] - 1)     # [n, Tm]
    lay = lambda x: (x[:, flat].float().view(nl, n, Tm, G, hpg, -1).permute(0, 1, 3, 2, 4, 5)
                     .reshape(nl, n, G, Tm * hpg, -1))
    t = torch.arange(Lm, device=DEV)
    pos = s["length"][sel].long()[:, None] - T[:, None] + i                # [n, Tm]
    if c["kind"] == "tree":
        j = (t[None, None, :] - (s["length"][sel].long() - T)[:, None, None]).expand(n, 1, Lm)
        words = s["mask"][flat]                                            # [n, Tm, words]
        w = words.gather(2, (j // 64).clamp(0, words.shape[2] - 1).expand(n, Tm, Lm))
        see = (j < 0) | ((j < T[:, None, None]) & ((w >> (j % 64)) & 1 > 0))
    else:
        see = t <= pos[:, :, None]
        if c["window"]:
            see &= (t > pos[:, :, None] - c["window"]) | (t < c["sinks"])
    see = see & live[:, None, :] & (i < T[:, None])[:, :, None]
    see = see[:, None, :, None, :].expand(n, G, Tm, hpg, Lm).reshape(1, n, G, Tm * hpg, Lm)
    x = lay(q) @ K.transpose(3, 4).contiguous()
    x.mul_(1 / math.sqrt(d)).masked_fill_(~see, -math.inf)
    back = lambda y: (y.view(nl, n, G, Tm, hpg, -1).permute(0, 1, 3, 2, 4, 5)
                      .reshape(nl, n, Tm, H, -1)[:, i < T[:, None]])
    return x, live, pages, lay, back


def _plain_attend(s):
    x, live, pages, _, back = _plain_logits(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    V = _plain_rows(s, s["v"], pages).masked_fill_(~live[None, :, None, :, None], 0)
    o = torch.where(total > 0, (x @ V) / total, torch.zeros_like(total))
    return dict(o=back(o).to(s["q"].dtype), lse=back(top + total.log()).squeeze(-1).contiguous())


def _plain_mass(s):
    x, _, _, lay, _ = _plain_logits(s)
    lse = lay(s["lse"].unsqueeze(-1))                                      # [nl, n, G, rows, 1]
    x.sub_(torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_()
    add = x.sum((2, 3))                                                    # [nl, n, Lm]
    sel, T = _long(s["slots"]), _long(s["rows"])
    length = s["length"][sel].long()
    t = torch.arange(add.shape[2], device=DEV)
    old = s["mass"][:, sel, :add.shape[2]]
    new = torch.where(t < (length - T)[:, None], old, torch.zeros_like(old)) + add
    s["out"][:, sel, :add.shape[2]] = torch.where(t < length[:, None], new, s["out"][:, sel, :add.shape[2]])
    return s["out"]


def _plain_write(s):
    c, P = s["c"], s["c"]["P"]
    sel, T = _long(s["slots"]), _long(s["rows"])
    who = torch.repeat_interleave(torch.arange(len(sel), device=DEV), T)
    pos = (s["length"][sel].long() - T)[who] + torch.arange(len(who), device=DEV) - (T.cumsum(0) - T)[who]
    page, off = s["table"][sel[who], pos // P].long(), pos % P
    for pool, rows, out in ((s["k"], s["kn"], s["k1"]), (s["v"], s["vn"], s["v1"])):
        data, scale = _planes(pool, c)
        code, byte = _to_fp4(rows.float())                                 # [nl, tot, G, ..]
        data[:, page, :, off] = _pack(code).transpose(0, 1)
        scale[:, page, :, off] = byte.transpose(0, 1)
        out.copy_(_from_fp4(data[:, page, :, off], scale[:, page, :, off]).transpose(0, 1))
    return dict(k=s["k1"], v=s["v1"])


def _plain_evict(s):
    c, P, nl = s["c"], s["c"]["P"], s["c"]["layers"]
    kids, src = _long(s["kids"]), _long(s["src"])
    keep, sinks, recent = _keep(c), c["sinks"], c["recent"]
    # the forks as they were are freed, and made again with their weights
    had = s["table"][kids]
    s["refs"].index_add_(0, had[had >= 0].long(), -torch.ones_like(had[had >= 0]))
    had = s["table"][src]
    s["refs"].index_add_(0, had[had >= 0].long(), torch.ones_like(had[had >= 0]))
    s["table"][kids] = had
    s["length"][kids] = s["length"][src]
    n = s["length"][kids].long()
    t = torch.arange(s["mass"].shape[2], device=DEV)
    s["mass"][:, kids] = torch.where(t < n[:, None], s["mass"][:, src], s["mass"][:, kids])
    # what is kept of each: sinks above all, then by weight, then by place
    m = s["mass"][:, kids]
    m = torch.where(t < sinks, torch.full_like(m, math.inf), m)
    m = torch.where(t < (n - recent)[:, None], m, torch.full_like(m, -math.inf))
    order = torch.sort(m, dim=2, descending=True, stable=True).indices[:, :, :sinks + keep]
    long_ = n > keep + sinks + recent
    status = torch.where(long_, 0, SHORT).to(torch.int32)
    idx = torch.full((nl, len(kids), sinks + keep), -1, dtype=torch.int64, device=DEV)
    idx[:, long_] = order[:, long_].sort(dim=2).values
    big = long_.nonzero().flatten()
    if len(big):
        new = sinks + keep + recent
        need = (new + P - 1) // P
        free = (s["refs"] == 0).nonzero().flatten()[:need * len(big)].view(len(big), need)
        tail = n[big][:, None] - recent + torch.arange(recent, device=DEV)     # [nb, recent]
        frm = torch.cat([idx[:, big], tail.expand(nl, *tail.shape)], 2)        # [nl, nb, new]
        old = s["table"][kids[big]].long()
        r = torch.arange(new, device=DEV)
        to = free[:, r // P]                                                   # [nb, new]
        page = old.expand(nl, *old.shape).gather(2, frm // P)
        l = torch.arange(nl, device=DEV)[:, None, None]
        for pool in (s["k"], s["v"]):
            pool[l, to, :, r % P] = pool[l, page, :, frm % P]
        s["refs"][free] = 1
        s["refs"].index_add_(0, old[old >= 0], -torch.ones_like(old[old >= 0], dtype=torch.int32))
        row = torch.full_like(old, -1)
        row[:, :need] = free
        s["table"][kids[big]] = row.to(torch.int32)
        s["length"][kids[big]] = new
        s["mass"][:, kids[big], :new] = s["mass"][:, kids[big]].gather(2, frm)
    return dict(k=s["k"], v=s["v"], table=s["table"], length=s["length"], refs=s["refs"], status=status,
                idx=idx.to(torch.int32), mass=s["mass"])


def run(s):
    if own:
        return _run_own(s)
    return {"tree": _plain_attend, "window": _plain_attend, "mass": _plain_mass, "write": _plain_write,
            "evict": _plain_evict}[s["c"]["kind"]](s)


# ------------------------------------------------------------------ 64-bit reference

def _exact_rows(x):
    """What x [.., d] in 4 bits stands for, by steps of the grid."""
    y = x.double().unflatten(-1, (-1, 32))
    m, e = torch.frexp(y.abs().amax(-1, keepdim=True))       # m in [0.5, 1)
    e = (e.long() - 3 + (m > 0.875)).clamp(-125, 125)
    power = lambda i: (i + 1023 << 52).view(torch.float64)   # 2^i, exactly
    y = y * power(-e)
    a = y.abs()
    a = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2)))
    return (a.clamp_max(6) * torch.sign(y) * power(e)).flatten(-2)


def exact(case, seed):
    """Sequence by sequence and head by head, from the definition; eviction
    moves and copies what it is given and has no such value."""
    c = case
    if c["kind"] == "evict":
        return None
    s = prepare(c, seed)
    nl, H, G, d, P = c["layers"], c["H"], c["G"], c["d"], c["P"]
    if c["kind"] == "write":
        k, v = torch.empty(s["kn"].shape, dtype=torch.float64, device=DEV), None
        v = torch.empty_like(k)
        for l in range(nl):
            k[l], v[l] = _exact_rows(s["kn"][l]), _exact_rows(s["vn"][l])
        return dict(k=k, v=v)
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device=DEV)
    mass = s["out"].double() if c["kind"] == "mass" else None
    at = 0
    for slot, n, T in zip(s["slots"], s["lens"], s["rows"]):
        t = torch.arange(n, device=DEV)
        page = s["table"][slot].long()[t // P]
        if c["kind"] == "tree":
            see = (t < n - T).expand(T, n).clone()
            bit = s["mask"][at:at + T]
            for j in range(T):
                see[:, n - T + j] = (bit[:, j // 64] >> (j % 64)) & 1 == 1
        else:
            see = _sees(c, n, T)
        see = see & (page >= 0)
        # the tokens that no row sees take no part
        some = see.any(0).nonzero().flatten()
        see, page, off = see[:, some], page[some], some % P
        if mass is not None:
            mass[:, slot, :n - T] = s["mass"][:, slot, :n - T].double()
        for l in range(nl):
            K = _rows_of(s, s["k"], l, page, off, torch.float64)               # [m, G, d]
            V = None if mass is not None else _rows_of(s, s["v"], l, page, off, torch.float64)
            for h in range(H):
                g = h * G // H
                x = s["q"][l, at:at + T, h].double() @ K[:, g].t().contiguous() / math.sqrt(d)
                x = torch.where(see, x, torch.full_like(x, -math.inf))
                if mass is not None:
                    mass[l, slot, some] += torch.exp(x - s["lse"][l, at:at + T, h, None].double()).sum(0)
                    continue
                lse[l, at:at + T, h] = torch.logsumexp(x, 1)
                o[l, at:at + T, h] = torch.nan_to_num(torch.softmax(x, 1)) @ V[:, g].contiguous()
        at += T
    return mass if mass is not None else dict(o=o, lse=lse)
