"""The timed calls of generation over a paged cache.

After the compression stage a GUI agent generates its action.  Its cache lives
in pages: several sequences (actions sampled from one prompt, other users')
share a pool, a sequence grows by the tokens it writes, forks without a copy,
is compressed by the stage's selection, and is read by two attentions: one for
a tree of drafted tokens, one with a sliding window and sink tokens.  Shapes
are those of the repository's workloads (28 layers, 28 query heads on 4 KV
groups of size 128; screenshots of 69x39 visual tokens; a 20% budget; windows
of 32 queries) and generic ones around them.  Kinds of a case:
  tree     attention of `rows` drafted tokens per sequence over its cache
  window   attention of the last `rows` tokens per sequence with a window
  append   children of one or more prompts freed, forked again, grown by a few
           tokens, and these tokens' K and V written
  compact  a prompt forked, and the fork compressed to the stage's selection
  accept   drafting sequences forked, and each fork's drafted tokens cut down
           to its accepted path
Every pass of the last three ends in the state that it ended in before, so it
can be run again: what it makes, the next pass frees first.
"""

import math

import torch

own = False      # True: the framework's calls; False: the plain forms

DEV = "cuda"


# ------------------------------------------------------------------ cases

def _case(name, kind, layers=1, seqs=1, lo=1, hi=1, rows=1, ragged=False, H=28, G=4, d=128, P=64,
          dtype="bf16", window=0, sinks=0, children=1, pct=20, tail=32):
    """Lengths are spread from lo to hi over the sequences; `ragged` spreads
    the rows from 1 to `rows` likewise."""
    c = dict(kind=kind, layers=layers, seqs=seqs, lo=lo, hi=hi, rows=rows, ragged=ragged, H=H, G=G,
             d=d, P=P, dtype=dtype, window=window, sinks=sinks, children=children, pct=pct,
             tail=tail)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one layer of a short conversation, eight drafted tokens: latency
        _case("tree-1l-short", "tree", lo=600, hi=600, rows=8),
        # all layers over the compressed cache of a fifth screenshot
        _case("tree-28l-20pct", "tree", layers=28, lo=2747, hi=2747, rows=24),
        # a batch of users of one layer, lengths and trees of every size, small pages
        _case("tree-1l-16seq-ragged", "tree", seqs=16, lo=500, hi=13711, rows=61, ragged=True, P=16),
        # all layers over the uncompressed cache of fifteen screenshots, the widest tree
        _case("tree-28l-full-15f", "tree", layers=28, lo=40941, hi=40941, rows=64),
        # float32 caches, head size 64
        _case("tree-f32-d64-4seq", "tree", layers=4, seqs=4, lo=700, hi=4001, rows=13, ragged=True,
              H=16, G=4, d=64, P=32, dtype="f32"),
        # one token each for a batch of long conversations, the old pages freed
        _case("window-1l-32seq-decode", "window", seqs=32, lo=37, hi=40941, window=4096, sinks=4),
        # one screenshot and its text appended to five, in one layer of a prefill
        _case("window-1l-append-frame", "window", lo=13711, hi=13711, rows=2755, window=8192,
              sinks=256),
        # the prefill of a long prompt from nothing
        _case("window-1l-prefill", "window", lo=8192, hi=8192, rows=8192, window=4096, sinks=4),
        # eight actions sampled from each of two compressed prompts: the first token
        _case("append-28l-16seq", "append", layers=28, seqs=2, children=8, lo=2723, hi=3100, rows=1),
        # one sequence's next tokens, one layer: latency
        _case("append-1l-1seq", "append", lo=1000, hi=1000, rows=3),
        # the stage's selection applied to the cache of five screenshots
        _case("compact-28l-5f", "compact", layers=28, lo=13711, hi=13711),
        # the accepted paths of a batch that drafts
        _case("accept-28l-16seq", "accept", layers=28, seqs=16, lo=600, hi=6001, rows=32),
    ]


# a drawn case costs no more than the largest listed one
_MOST_FLOPS = 4 * 28 * 28 * 128 * 64 * 40941
_MOST_SCORES = 28 * 8192 * 8192
_MOST_TOKENS = 28 * 40941


def draw(rng):
    logint = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))
    kind = rng.choice(["tree", "tree", "tree", "window", "window", "window", "append", "compact",
                       "accept"])
    H, G = rng.choice([(28, 4), (28, 4), (32, 8), (16, 2), (12, 2), (16, 16), (14, 2), (6, 1)])
    d = 64 if (H, G) == (14, 2) else rng.choice([128, 128, 128, 64])
    P = rng.choice([16, 32, 64, 64, 128, 256])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    layers, seqs = logint(1, 28), logint(1, 32)
    hi = logint(16, 41000)
    lo = rng.choice([hi, logint(8, hi) if hi > 8 else hi])
    c = _case(None, kind, layers, seqs, lo, hi, 1, rng.random() < 0.5, H, G, d, P, dtype)
    if kind == "tree":
        c["rows"] = min(lo, logint(1, 64))
    elif kind == "window":
        # a decoded token, a few, or a chunk of a prefill
        c["rows"] = min(lo, rng.choice([1, logint(1, 16), logint(1, 8192)]))
        c["window"] = rng.choice([0, logint(1, 8192), logint(64, 8192)])
        c["sinks"] = rng.choice([0, 4, logint(1, 512)])
        if c["rows"] > 64:
            c["layers"], c["seqs"] = min(layers, 4), min(seqs, 4)
    elif kind == "append":
        c["seqs"], c["children"] = min(seqs, 8), logint(1, 16)
        c["rows"] = logint(1, 300)
    elif kind == "compact":
        c["seqs"], c["pct"], c["tail"] = min(seqs, 4), rng.choice([10, 20, 40]), rng.randint(0, 64)
        c["hi"] = max(hi, 200)
        c["lo"] = max(lo, 200)
    else:
        c["rows"] = min(lo, logint(1, 64))
    # the plain form pads to the longest sequence and the largest row count
    while c["layers"] * c["seqs"] * c["hi"] > _MOST_TOKENS // (2 if dtype == "f32" else 1):
        if c["layers"] > 1:
            c["layers"] = (c["layers"] + 1) // 2
        else:
            c["seqs"] = (c["seqs"] + 1) // 2
    if kind in ("tree", "window"):
        while c["layers"] * c["seqs"] * H * c["rows"] * c["hi"] > _MOST_SCORES // 2:
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


def _budget(c):
    return c["pct"] * (min(_lens(c)) - c["tail"]) // 100


def _visible(c, n, T):
    """Cached tokens that some row sees, and the (row, token) pairs seen."""
    if c["kind"] == "tree":
        return n, T * (n - T) + T * (T + 1) // 2
    w, s = c["window"] or n, c["sinks"]
    lo = max(n - T - w + 1, 0)
    seen = n - lo + min(s, lo)
    pairs = 0
    for p in (range(n - T, n) if T < 64 else ()):
        pairs += min(p + 1, w) + min(s, max(p + 1 - w, 0))
    if T >= 64:
        p = torch.arange(n - T, n, dtype=torch.int64)
        pairs = int((torch.clamp(p + 1, max=w) + torch.clamp(p + 1 - w, 0, s)).sum())
    return seen, pairs


def work(case):
    c = case
    nl, H, G, d, P = c["layers"], c["H"], c["G"], c["d"], c["P"]
    e = 4 if c["dtype"] == "f32" else 2
    row = 2 * G * d * e                       # K and V of a token in one layer
    by = fl = 0
    for n, T in zip(_lens(c), _rows(c)):
        if c["kind"] in ("tree", "window"):
            seen, pairs = _visible(c, n, T)
            by += nl * (seen * row + 2 * T * H * d * e + 4 * T * H) + 4 * (seen + P - 1) // P
            by += 8 * T * _words(c) if c["kind"] == "tree" else 0
            fl += nl * 4 * H * d * pairs
        elif c["kind"] == "append":
            copied = 2 * (n % P)              # read and written
            fresh = (n + T + P - 1) // P - (n + P - 1) // P
            by += c["children"] * (nl * row * (copied + 2 * T) + 8 * ((n + P - 1) // P + fresh))
        else:
            if c["kind"] == "compact":
                a, kept, idx = 0, _budget(c) + c["tail"], 4 * nl * _budget(c)
            else:
                a, kept, idx = n - T, (T + 1) // 2, 4 * T
            by += nl * row * 2 * (a % P + kept) + idx + 8 * ((n + P - 1) // P)
    return {"bytes": by, "flops": fl}


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    """A pool whose pages lie in no order, as after some time of serving."""
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    nl, n, H, G, d, P, kind = c["layers"], c["seqs"], c["H"], c["G"], c["d"], c["P"], c["kind"]
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    lens, rows = _lens(c), _rows(c)
    pages = [(x + P - 1) // P for x in lens]
    made = {"append": c["children"], "compact": 1, "accept": 1}.get(kind, 0)   # forks per sequence
    grown = [(x + r + P - 1) // P for x, r in zip(lens, rows)] if kind == "append" else pages
    width = max(grown) + 1
    # room for what a pass makes, and some pages that nobody has
    room = {"append": sum(made * (a - b + 1) for a, b in zip(grown, pages)),
            "compact": sum((_budget(c) + c["tail"] + P - 1) // P for _ in lens),
            "accept": sum((r + P - 1) // P + 1 for r in rows)}.get(kind, 0)
    n_pages = sum(pages) + room + 3
    k = torch.empty(nl, n_pages, G, P, d, dtype=dt, device=DEV)
    v = torch.empty_like(k)
    for l in range(nl):
        k[l].normal_(generator=g)
        v[l].normal_(generator=g)
    slots = torch.randperm(n * (1 + made), generator=host)[:n].tolist()
    kids = [i for i in range(n * (1 + made)) if i not in set(slots)]
    table = torch.full((n * (1 + made), width), -1, dtype=torch.int32)
    perm = torch.randperm(n_pages, generator=host, dtype=torch.int64).to(torch.int32)
    refs, length = torch.zeros(n_pages, dtype=torch.int32), torch.zeros(n * (1 + made), dtype=torch.int32)
    at = 0
    for b in range(n):
        table[slots[b], :pages[b]] = perm[at:at + pages[b]]
        length[slots[b]] = lens[b]
        at += pages[b]
        if kind == "window" and c["window"]:
            # the pages that no row will see again are freed
            j = torch.arange(pages[b])
            gone = (j * P >= c["sinks"]) & ((j + 1) * P <= lens[b] - rows[b] - c["window"] + 1)
            table[slots[b], :pages[b]][gone] = -1
    refs[table[table >= 0].long()] = 1
    s = dict(c=c, k=k, v=v, table=table.to(DEV), refs=refs.to(DEV), length=length.to(DEV), slots=slots,
             lens=lens, rows=rows, longest=max(lens))
    tot = sum(rows)
    if kind in ("tree", "window"):
        # logits of the spread that trained heads have
        s["q"] = (1.5 * torch.randn(nl, tot, H, d, generator=g, device=DEV)).to(dt)
    if kind == "tree":
        s["mask"] = _tree(rows, _words(c), host).to(DEV)
    if kind in ("append", "compact", "accept"):
        s["kids"] = kids
        s["src"] = [x for x in slots for _ in range(made)]
    if kind == "append":
        s["new_rows"] = [r for r in rows for _ in range(made)]
        s["kn"] = torch.empty(nl, made * tot, G, d, dtype=dt, device=DEV).normal_(generator=g)
        s["vn"] = torch.empty_like(s["kn"]).normal_(generator=g)
    if kind == "compact":
        B, past = _budget(c), [x - c["tail"] for x in lens]
        s["idx"] = torch.stack([torch.stack([
            torch.rand(m, generator=g, device=DEV).topk(B).indices.sort().values for m in past])
            for _ in range(nl)]).to(torch.int32)
    if kind == "accept":
        s["idx"], s["counts"] = _paths(rows, host)
        s["idx"], s["counts"] = s["idx"].to(DEV), s["counts"].to(DEV)
    return s


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


def _paths(rows, host):
    """A path of at most half of each tree, from its root down: its tokens'
    places in ascending order, and how many they are."""
    idx = torch.zeros(1, len(rows), (max(rows) + 1) // 2, dtype=torch.int32)
    counts = torch.zeros(len(rows), dtype=torch.int32)
    for b, T in enumerate(rows):
        par = _parents(T, host)
        path = [T - 1]
        while par[path[-1]] >= 0:
            path.append(par[path[-1]])
        path = path[::-1][:(T + 1) // 2]
        idx[0, b, :len(path)] = torch.tensor(path, dtype=torch.int32)
        counts[b] = len(path)
    return idx, counts


# ------------------------------------------------------------------ the framework's calls

def _handle(s):
    """What a serving program makes once: the cache's handle, the workspace
    and the output buffers."""
    from paper_2606_01790_amd import paged as pg
    c = s["c"]
    h = dict(pg=pg, cache=pg.Cache(s["k"], s["v"], s["table"], s["length"], s["refs"], c["H"]))
    if c["kind"] in ("tree", "window"):
        h["out"] = torch.empty_like(s["q"])
        h["lse"] = torch.empty(s["q"].shape[:3], dtype=torch.float32, device=DEV)
        need = pg.attend_workspace_bytes(h["cache"], s["rows"], s["longest"])
    else:
        h["status"] = torch.zeros(len(s["kids"]), dtype=torch.int32, device=DEV)
        need = pg.pages_workspace_bytes(h["cache"], len(s["kids"]))
    h["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    if c["kind"] == "append":
        h["lay"] = pg.rows_layout(s["kn"])
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
    pg.pages_free(cache, s["kids"])
    pg.pages_fork(cache, s["src"], s["kids"])
    if kind == "append":
        pg.pages_grow(cache, s["kids"], s["new_rows"], h["status"], h["ws"])
        pg.pages_write(cache, s["kids"], s["new_rows"], s["kn"], s["vn"], h["lay"])
    elif kind == "compact":
        pg.pages_compact(cache, s["kids"], s["idx"], h["status"], h["ws"], tail=c["tail"])
    else:
        pg.pages_compact(cache, s["kids"], s["idx"], h["status"], h["ws"], span=s["rows"],
                         counts=s["counts"])
    return dict(k=s["k"], v=s["v"], table=s["table"], length=s["length"], refs=s["refs"],
                status=h["status"])


# ------------------------------------------------------------------ the plain forms

def _long(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


def _plain_attend(s):
    c, k, v, q = s["c"], s["k"], s["v"], s["q"]
    nl, H, G, d, P = c["layers"], c["H"], c["G"], c["d"], c["P"]
    sel, T = _long(s["slots"]), _long(s["rows"])
    n = len(s["slots"])
    n_pg = (s["longest"] + P - 1) // P
    Lm, Tm, hpg = n_pg * P, max(s["rows"]), H // G
    pages = s["table"][sel, :n_pg].long()
    live = (pages >= 0).repeat_interleave(P, dim=1)                      # [n, Lm]
    lay = lambda x: (x[:, pages.clamp_min(0)].float().permute(0, 1, 3, 2, 4, 5)
                     .reshape(nl, n, G, Lm, d))
    K, V = lay(k), lay(v)
    first = T.cumsum(0) - T
    i = torch.arange(Tm, device=DEV)
    flat = (first[:, None] + i.clamp_max(Tm)).clamp_max(q.shape[1] - 1)     # [n, Tm]
    Q = (q[:, flat].float().view(nl, n, Tm, G, hpg, d).permute(0, 1, 3, 2, 4, 5)
         .reshape(nl, n, G, Tm * hpg, d))
    t = torch.arange(Lm, device=DEV)
    pos = s["length"][sel].long()[:, None] - T[:, None] + i                # [n, Tm]
    ctx = (s["length"][sel].long() - T)[:, None, None]
    if c["kind"] == "tree":
        j = (t[None, None, :] - ctx).expand(n, 1, Lm)
        words = s["mask"][flat]                                            # [n, Tm, words]
        w = words.gather(2, (j // 64).clamp(0, words.shape[2] - 1).expand(n, Tm, Lm))
        see = (j < 0) | ((j < T[:, None, None]) & ((w >> (j % 64)) & 1 > 0))
    else:
        see = t <= pos[:, :, None]
        if c["window"]:
            see &= (t > pos[:, :, None] - c["window"]) | (t < c["sinks"])
    see = (see & live[:, None, :])[:, None, :, None, :].expand(n, G, Tm, hpg, Lm).reshape(
        1, n, G, Tm * hpg, Lm)
    x = Q @ K.transpose(3, 4).contiguous()
    x.mul_(1 / math.sqrt(d)).masked_fill_(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    V = V.masked_fill(~live[None, :, None, :, None], 0)
    o = torch.where(total > 0, (x @ V) / total, torch.zeros_like(total))
    back = lambda y: (y.view(nl, n, G, Tm, hpg, -1).permute(0, 1, 3, 2, 4, 5)
                      .reshape(nl, n, Tm, H, -1)[:, i < T[:, None]])
    return dict(o=back(o).to(q.dtype), lse=back(top + total.log()).squeeze(-1).contiguous())


def _plain_free(s, sel):
    had = s["table"][sel]
    s["refs"].index_add_(0, had[had >= 0].long(), -torch.ones_like(had[had >= 0]))
    s["table"][sel] = -1
    s["length"][sel] = 0


def _plain_fork(s, src, dst):
    had = s["table"][src]
    s["refs"].index_add_(0, had[had >= 0].long(), torch.ones_like(had[had >= 0]))
    s["table"][dst] = had
    s["length"][dst] = s["length"][src]


def _plain_take(s, sel, col0, need):
    """The lowest free pages, in the order of the sequences, into the columns
    col0.. of each one's row; their owners' places in `sel` and the pages."""
    free = (s["refs"] == 0).nonzero().flatten()[:int(need.sum())]
    who = torch.repeat_interleave(torch.arange(len(sel), device=DEV), need)
    off = torch.arange(len(who), device=DEV) - (need.cumsum(0) - need)[who]
    s["table"][sel[who], col0[who] + off] = free.to(torch.int32)
    s["refs"][free] = 1
    return who, off, free


def _plain_append(s):
    c, P = s["c"], s["c"]["P"]
    kids, add = _long(s["kids"]), _long(s["new_rows"])
    _plain_free(s, kids)
    _plain_fork(s, _long(s["src"]), kids)
    n = s["length"][kids].long()
    have, part = (n + P - 1) // P, n % P
    last = s["table"][kids, (have - 1).clamp_min(0)].long()
    cow = (part > 0) & (s["refs"][last] > 1)
    _plain_take(s, kids, have - cow.long(), (n + add + P - 1) // P - have + cow.long())
    s["refs"].index_add_(0, last[cow], -torch.ones_like(last[cow], dtype=torch.int32))
    new = s["table"][kids, (have - 1).clamp_min(0)].long()
    keep = (torch.arange(P, device=DEV) < part[cow][:, None])[None, :, None, :, None]
    s["length"][kids] = (n + add).to(torch.int32)
    who = torch.repeat_interleave(torch.arange(len(kids), device=DEV), add)
    pos = n[who] + torch.arange(len(who), device=DEV) - (add.cumsum(0) - add)[who]
    page = s["table"][kids[who], pos // P].long()
    for pool, rows in ((s["k"], s["kn"]), (s["v"], s["vn"])):
        pool[:, new[cow]] = torch.where(keep, pool[:, last[cow]], pool[:, new[cow]])
        pool[:, page, :, pos % P] = rows.transpose(0, 1)


def _plain_compact(s):
    c, P, nl = s["c"], s["c"]["P"], s["c"]["layers"]
    kids = _long(s["kids"])
    _plain_free(s, kids)
    _plain_fork(s, _long(s["src"]), kids)
    n = s["length"][kids].long()
    B = s["idx"].shape[2]
    accept = c["kind"] == "accept"
    a = n - _long(s["rows"]) if accept else torch.zeros_like(n)
    cnt = s["counts"].long() if accept else torch.full_like(n, B)
    tail = 0 if accept else c["tail"]
    new = a + cnt + tail
    col0 = a // P
    old = s["table"][kids].long()
    need = (new + P - 1) // P - col0
    _plain_take(s, kids, col0, need)
    # every row of the fresh pages up to the new length: where it comes from
    most = B + tail + P
    r = col0[:, None] * P + torch.arange(most, device=DEV)               # [n, most]
    j = r - a[:, None]
    pick = s["idx"].long().expand(nl, len(kids), B)
    pick = pick.gather(2, j.clamp(0, B - 1).expand(nl, *j.shape))
    src = torch.where(j < 0, r, torch.where(j < cnt[:, None], a[:, None] + pick,
                                            n[:, None] - tail + j - cnt[:, None]))
    used = (r < new[:, None])                                            # [n, most]
    b = torch.arange(len(kids), device=DEV)[:, None].expand(r.shape)[used]
    src, r = src[:, used], r[used]                                       # [nl, m], [m]
    to = s["table"][kids[b], r // P].long()
    frm = old[b, src // P]
    l = torch.arange(nl, device=DEV)[:, None]
    for pool in (s["k"], s["v"]):
        got = pool[l, frm, :, src % P]                                   # [nl, m, G, d]
        pool[:, to, :, r % P] = got.transpose(0, 1)
    # the pages from a's on are let go, but for the fresh ones
    cols = torch.arange(old.shape[1], device=DEV)
    let = old[(cols >= col0[:, None]) & (old >= 0)]
    s["refs"].index_add_(0, let, -torch.ones_like(let, dtype=torch.int32))
    tab = s["table"][kids]
    tab[cols >= ((new + P - 1) // P)[:, None]] = -1
    s["table"][kids] = tab
    s["length"][kids] = new.to(torch.int32)


def run(s):
    if own:
        return _run_own(s)
    kind = s["c"]["kind"]
    if kind in ("tree", "window"):
        return _plain_attend(s)
    if kind == "append":
        _plain_append(s)
    else:
        _plain_compact(s)
    return dict(k=s["k"], v=s["v"], table=s["table"], length=s["length"], refs=s["refs"],
                status=torch.zeros(len(s["kids"]), dtype=torch.int32, device=DEV))


# ------------------------------------------------------------------ 64-bit reference

def exact(case, seed):
    """Sequence by sequence and head by head, from the definition; the moves
    of pages copy bits and have no such value."""
    c = case
    if c["kind"] not in ("tree", "window"):
        return None
    s = prepare(c, seed)
    nl, H, G, d, P = c["layers"], c["H"], c["G"], c["d"], c["P"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device=DEV)
    at = 0
    for slot, n, T in zip(s["slots"], s["lens"], s["rows"]):
        t = torch.arange(n, device=DEV)
        page = s["table"][slot].long()[t // P]
        p = torch.arange(n - T, n, device=DEV)[:, None]
        if c["kind"] == "tree":
            see = (t < n - T).expand(T, n).clone()
            bit = s["mask"][at:at + T]
            for j in range(T):
                see[:, n - T + j] = (bit[:, j // 64] >> (j % 64)) & 1 == 1
        else:
            see = t <= p
            if c["window"]:
                see = see & ((t > p - c["window"]) | (t < c["sinks"]))
        see = see & (page >= 0)
        # the tokens that no row sees take no part
        some = see.any(0).nonzero().flatten()
        see, page, off = see[:, some], page[some], some % P
        for l in range(nl):
            K, V = s["k"][l, page, :, off].double(), s["v"][l, page, :, off].double()   # [m, G, d]
            for h in range(H):
                g = h * G // H
                x = s["q"][l, at:at + T, h].double() @ K[:, g].t().contiguous() / math.sqrt(d)
                x = torch.where(see, x, torch.full_like(x, -math.inf))
                lse[l, at:at + T, h] = torch.logsumexp(x, 1)
                o[l, at:at + T, h] = torch.nan_to_num(torch.softmax(x, 1)) @ V[:, g].contiguous()
        at += T
    return dict(o=o, lse=lse)
