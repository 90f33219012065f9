"""CPU reference of caches held in 4 bits, of accumulated attention weights and of
eviction by them, in plain loops and fp64 from their definitions.  Shares no code
with the GPU path."""

from __future__ import annotations

import numpy as np

from .paged_oracle import OK, PagedModel  # noqa: F401

SHORT = 3
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def fp4_row_bytes(d):
    """Of a row: d/2 bytes of elements, d/32 of scales."""
    return d // 2 + d // 32


def fp4_quantise(x):
    """x [.., d] fp64 as rows [.., d/2 + d/32] uint8.  Of 32 elements the scale is
    2^e with the largest magnitude in (3.5, 7] * 2^e, e + 127 clamped to [2, 252]; an
    element goes to the nearest value, ties to the even code, beyond 6 to 6.  A
    block with an infinity or NaN has the scale byte 255."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    out = np.zeros(x.shape[:-1] + (fp4_row_bytes(d),), dtype=np.uint8)
    flat, rows = x.reshape(-1, d), out.reshape(-1, fp4_row_bytes(d))
    mid = [(a + b) / 2 for a, b in zip(GRID, GRID[1:])]
    for r in range(flat.shape[0]):
        codes = np.zeros(d, dtype=np.uint8)
        for blk in range(d // 32):
            y = flat[r, 32 * blk:32 * blk + 32]
            if not np.all(np.isfinite(y)):
                rows[r, d // 2 + blk] = 255
                continue
            top = np.max(np.abs(y))
            e = -125
            if top > 0:
                e = int(np.floor(np.log2(top))) - 3      # at or below the one sought
                while top > 7 * 2.0 ** e:
                    e += 1
            e = min(max(e, -125), 125)
            rows[r, d // 2 + blk] = e + 127
            a = np.abs(y) / 2.0 ** e
            c = np.zeros(32, dtype=np.uint8)
            for i, m in enumerate(mid):        # past a midpoint, or at it where the upper code is even
                c += (a > m) | ((a == m) & ((i + 1) % 2 == 0))
            codes[32 * blk:32 * blk + 32] = c | (np.signbit(y).astype(np.uint8) << 3)
        rows[r, :d // 2] = codes[0::2] | codes[1::2] << 4
    return out


def fp4_numbers(rows):
    """What rows [.., d/2 + d/32] stand for, fp64."""
    rows = np.asarray(rows, dtype=np.uint8)
    d = rows.shape[-1] * 32 // 17
    data, scale = rows[..., :d // 2], rows[..., d // 2:]
    code = np.stack([data & 15, data >> 4], -1).reshape(*data.shape[:-1], d)
    val = np.array(GRID + tuple(-g for g in GRID))[code]
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return val * np.repeat(s, 32, axis=-1)


def fp4_blocks(pool):
    """A model's pool [nl, n_pages, G, P, row bytes] as the blocks of the cache: the
    rows of a page, then their scales."""
    d = pool.shape[-1] * 32 // 17
    lead = pool.shape[:3]
    return np.concatenate([pool[..., :d // 2].reshape(*lead, -1), pool[..., d // 2:].reshape(*lead, -1)], -1)


def read(model, slots, rows, row_len):
    """[n_layers, sum rows, G, row_len] of the last rows, zero where there is none."""
    nl, _, G = model.k.shape[:3]
    k = np.zeros((nl, sum(rows), G, row_len), dtype=model.k.dtype)
    v, r = np.zeros_like(k), 0
    for b, T in zip(slots, rows):
        for j in range(T):
            t = int(model.len[b]) - T + j
            w = model.at(b, t) if t >= 0 else None
            if w is not None:
                k[:, r], v[:, r] = model.k[:, w[0], :, w[1]], model.v[:, w[0], :, w[1]]
            r += 1
    return k, v


def weights(model, slot, q, lse, see, to_f64, layer):
    """sum_{i, h: i sees t} exp(q . k_t / sqrt(d) - lse) for each cached token t:
    q [T, H, d], lse [T, H] (fp64), see [T, n].  Also the largest sum_j |q_j k_j| /
    sqrt(d) + |lse| among what was added to each token."""
    T, H, d = q.shape
    n, G = int(model.len[slot]), model.k.shape[2]
    add, size = np.zeros(n), np.zeros(n)
    with np.errstate(all="ignore"):
        for t in range(n):
            w = model.at(slot, t)
            if w is None:
                continue
            k = np.repeat(to_f64(model.k[layer, w[0], :, w[1]]), H // G, axis=0)       # [H, d]
            use = see[:, t][:, None] & (lse > -np.inf)         # (nor NaN)
            if not use.any():
                continue
            x = np.einsum("thd,hd->th", q, k) / np.sqrt(d)
            add[t] = np.sum(np.exp(x - lse)[use])
            size[t] = np.max((np.einsum("thd,hd->th", np.abs(q), np.abs(k)) / np.sqrt(d) + np.abs(lse))[use])
    return add, size


def evict(model, slots, mass, keep, sinks, recent):
    """mass [n_layers, n_slots, cap] is changed in place.  Returns idx
    [n_layers, n, sinks + keep] and the statuses."""
    nl = model.k.shape[0]
    idx = np.full((nl, len(slots), sinks + keep), -1, dtype=np.int32)
    counts, grown = [], []
    new = {}
    for i, b in enumerate(slots):
        n = int(model.len[b])
        grown.append(OK if n > sinks + keep + recent else SHORT)
        counts.append(0)
        if grown[-1] == SHORT:
            continue
        for l in range(nl):
            here = [t for t in range(n - recent) if model.at(b, t) is not None]
            m = mass[l, b]
            weigh = lambda t: (np.inf, 0) if np.isnan(m[t]) else (m[t], -1)     # NaN above infinity
            rest = sorted((t for t in here if t >= sinks), key=lambda t: (-weigh(t)[0], -weigh(t)[1], t))
            kept = [t for t in here if t < sinks] + sorted(rest[:keep])
            idx[l, i, :len(kept)] = kept
            counts[-1] = len(kept)
            new[l, i] = np.concatenate([m[kept], m[n - recent:n]])
    # the model's compaction takes tokens of the span [0, n - recent)
    status = model.compact(slots, np.where(idx < 0, 1 << 30, idx), tail=recent,
                           counts=np.array(counts), grown=np.array(grown))
    for (l, i), m in new.items():
        if status[i] == OK:
            mass[l, slots[i], :len(m)] = m
    return idx, status
