"""CPU reference of the paged cache and the attentions over it: the host model
of the bookkeeping, sequence by sequence in plain loops, and the attentions in
fp64 from their definition.  Shares no code with the GPU path."""

from __future__ import annotations

import numpy as np

OK, NO_PAGES, RANGE = 0, 1, 2


class PagedModel:
    """k, v: [n_layers, n_pages, G, P, d] storage arrays of any type."""

    def __init__(self, k, v, n_slots, max_pages):
        self.k, self.v = k, v
        self.P = k.shape[3]
        self.n_pages = k.shape[1]
        self.table = np.full((n_slots, max_pages), -1, dtype=np.int32)
        self.len = np.zeros(n_slots, dtype=np.int32)
        self.refs = np.zeros(self.n_pages, dtype=np.int32)

    @property
    def cap(self):
        return self.table.shape[1] * self.P

    def pages(self, tokens):
        return -(-tokens // self.P)

    def is_page(self, p):
        return 0 <= p < self.n_pages

    def at(self, slot, t):
        """(page, row) of a token, or None where it has no page."""
        p = int(self.table[slot, t // self.P])
        return (p, t % self.P) if self.is_page(p) else None

    def _free_pages(self):
        return [p for p in range(self.n_pages) if self.refs[p] == 0]

    def _take(self, free, need):
        """The first `need` free pages, or None if they do not suffice."""
        if need > len(free):
            return None
        got, free[:need] = free[:need], []
        return got

    def grow(self, slots, add):
        free, status, first = self._free_pages(), [], self.refs.copy()
        short = False
        for b, a in zip(slots, add):
            n = int(self.len[b])
            have, part = self.pages(n), n % self.P
            if n + a > self.cap:
                status.append(RANGE)
                continue
            if a == 0:
                status.append(OK)
                continue
            old = int(self.table[b, have - 1]) if part else -1
            if part and not self.is_page(old):
                status.append(RANGE)
                continue
            replace = part > 0 and first[old] > 1
            need = self.pages(n + a) - have + (1 if replace else 0)
            got = None if short and need else self._take(free, need)
            if got is None:
                short = True           # the sequences after it find too few as well
                status.append(NO_PAGES)
                continue
            col = have - 1 if replace else have
            self.table[b, col:col + need] = got
            self.refs[got] = 1
            if replace:
                for x in (self.k, self.v):
                    x[:, got[0], :, :part] = x[:, old, :, :part]
                self.refs[old] -= 1
            self.len[b] = n + a
            status.append(OK)
        return np.array(status, dtype=np.int32)

    def write(self, slots, rows, k, v, grown=None):
        """k, v: [n_layers, sum(rows), G, d]; grown: the status of the grow
        that made the rows"""
        r = 0
        for i, (b, T) in enumerate(zip(slots, rows)):
            if grown is not None and grown[i] != OK:
                r += T
                continue
            for j in range(T):
                t = int(self.len[b]) - T + j
                w = self.at(b, t) if t >= 0 else None
                if w is not None and self.refs[w[0]] <= 1:
                    self.k[:, w[0], :, w[1]] = k[:, r]
                    self.v[:, w[0], :, w[1]] = v[:, r]
                r += 1

    def _let_go(self, slot, cols):
        for j in cols:
            p = int(self.table[slot, j])
            if self.is_page(p):
                self.refs[p] -= 1
            self.table[slot, j] = -1

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self._let_go(b, range(self.pages(int(self.len[b]))))
            for j in range(self.pages(int(self.len[a]))):
                self.table[b, j] = self.table[a, j]
                if self.is_page(int(self.table[a, j])):
                    self.refs[self.table[a, j]] += 1
            self.len[b] = self.len[a]

    def free(self, slots, keep_first=0, keep_last=0):
        for b in slots:
            n = int(self.len[b])
            keep = set(range(min(keep_first, n))) | set(range(max(n - keep_last, 0), n))
            for j in range(self.pages(n)):
                if not keep & set(range(j * self.P, min((j + 1) * self.P, n))):
                    self._let_go(b, [j])
            if keep_last == 0:
                self.len[b] = min(n, keep_first)

    def compact(self, slots, idx, tail=0, span=None, counts=None, grown=None):
        """idx: [n_layers or 1, n, B]; grown: the status of the grow that made
        the span"""
        free, status, short = self._free_pages(), [], False
        moves = []
        k0, v0 = self.k.copy(), self.v.copy()
        for i, b in enumerate(slots):
            n = int(self.len[b])
            if grown is not None and grown[i] != OK:
                status.append(grown[i])
                continue
            s = n if span is None else min(int(span[i]), n)
            a, B = n - s, idx.shape[2]
            cnt = B if counts is None else min(max(int(counts[i]), 0), B)
            new = a + cnt + tail
            gone = cnt + tail > 0 and a % self.P and not self.is_page(self.table[b, a // self.P])
            lost = tail <= s and any(self.at(b, t) is None for t in range(n - tail, n))
            if tail > s or new > self.cap or gone or lost:
                status.append(RANGE)
                continue
            col = a // self.P if cnt + tail else self.pages(a)
            need = self.pages(new) - col
            got = None if short and need else self._take(free, need)
            if got is None:
                short = True
                status.append(NO_PAGES)
                continue
            row = self.table[b].copy()
            moves.append((i, b, row, col, got, n, s, a, cnt, new))
            status.append(OK)
        for i, b, row, col, got, n, s, a, cnt, new in moves:
            self._let_go(b, range(col, self.pages(n)))
            self.table[b, col:col + len(got)] = got
            self.refs[got] = 1
            self.len[b] = new
            for layer in range(self.k.shape[0]):
                pick = idx[layer if idx.shape[0] > 1 else 0, i]
                for r in range(col * self.P, new):
                    if r < a:
                        t = r
                    elif r < a + cnt:
                        t = int(pick[r - a])
                        t = a + t if 0 <= t < s - tail else -1
                    else:
                        t = n - tail + r - a - cnt
                    p = int(row[t // self.P]) if t >= 0 else -1
                    to = int(self.table[b, r // self.P])
                    for x, x0 in ((self.k, k0), (self.v, v0)):
                        x[layer, to, :, r % self.P] = \
                            x0[layer, p, :, t % self.P] if self.is_page(p) else 0
        return np.array(status, dtype=np.int32)


def attend(model, slot, q, see, to_f64, layer):
    """q [T, H, d] (fp64) of one sequence and layer, see [T, n] which cached
    tokens each row sees.  Returns out [T, H, d], lse [T, H], sum_t p_t |v_t|
    [T, H, d] and the largest sum_j |q_j k_j| / sqrt(d) among seen tokens
    [T, H].  Tokens that a row does not see take no part in it."""
    T, H, d = q.shape
    n = int(model.len[slot])
    G = model.k.shape[2]
    K, V = np.zeros((n, G, d)), np.zeros((n, G, d))
    see = see.copy()
    for t in range(n):
        w = model.at(slot, t)
        if w is None:
            see[:, t] = False
        else:
            K[t] = to_f64(model.k[layer, w[0], :, w[1]])
            V[t] = to_f64(model.v[layer, w[0], :, w[1]])
    out, mass = np.zeros((T, H, d)), np.zeros((T, H, d))
    lse, size = np.full((T, H), -np.inf), np.zeros((T, H))
    with np.errstate(all="ignore"):
        for i in range(T):
            some = np.nonzero(see[i])[0]
            if some.size == 0:
                continue
            for h in range(H):
                g = h * G // H
                k, v = K[some, g], V[some, g]
                x = k @ q[i, h] / np.sqrt(d)
                size[i, h] = np.max(np.abs(k) @ np.abs(q[i, h])) / np.sqrt(d)
                top = x.max()
                e = np.exp(x - top)
                lse[i, h] = top + np.log(e.sum())
                p = e / e.sum()
                out[i, h] = p @ v
                mass[i, h] = p @ np.abs(v)
    return out, lse, mass, size


def see_tree(n, T, mask):
    """mask [T, words] uint64"""
    see = np.zeros((T, n), dtype=bool)
    for i in range(T):
        for t in range(n):
            j = t - (n - T)
            see[i, t] = j < 0 or (j < T and bool(int(mask[i, j // 64]) >> (j % 64) & 1))
    return see


def see_window(n, T, window, sinks):
    see = np.zeros((T, n), dtype=bool)
    for i in range(T):
        p = n - T + i
        for t in range(n):
            see[i, t] = t <= p and (window == 0 or t > p - window or t < sinks)
    return see
