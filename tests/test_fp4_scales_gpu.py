"""Scale bytes that pages_write does not make, in a pool that the caller filled: 0 and 1,
whose elements are subnormal or small, and 253 and 254, of whose elements those that bf16
does not hold, 2^128 and more, count as infinities.  Bounds as in the tests of the
attentions over 4 bits; infinities and NaN as the reference has them."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import fp4_cache as F  # noqa: E402
from oracle import evict_oracle as EO  # noqa: E402
from oracle import paged_oracle as PO  # noqa: E402
from paper_2606_01790_amd import paged as pg  # noqa: E402
from test_fp4_attend_gpu import U, Case, say, tree_masks  # noqa: E402

pytestmark = pytest.mark.gpu


def numbers(rows):
    x = EO.fp4_numbers(rows)
    return np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x)


def test_every_scale_and_code():
    """Read back: bf16 has every number below 2^128 exactly."""
    d, P = 64, 256
    m = F.empty_model(1, 2, 1, P, d, 1, 2)
    m.table[0], m.refs[:], m.len[0] = [1, 0], 1, 2 * P
    rows = np.zeros((2 * P, EO.fp4_row_bytes(d)), dtype=np.uint8)
    rows[:, :d // 2] = (np.arange(d) % 16)[0::2] | (np.arange(d) % 16)[1::2] << 4
    rows[:, d // 2] = np.arange(2 * P) % 256
    rows[:, d // 2 + 1] = 255 - np.arange(2 * P) % 256
    m.k[0, [1, 0], 0] = rows.reshape(2, P, -1)
    m.v[0, [1, 0], 0] = rows[::-1].reshape(2, P, -1)
    c = F.cache_of(m, 2, d)
    k = torch.full((1, 2 * P, 1, d), 7.0, device="cuda", dtype=torch.bfloat16)
    v = k.clone()
    pg.pages_read(c, [0], [2 * P], k, v, pg.rows_layout(k))
    torch.cuda.synchronize()
    for got, want in ((k, numbers(rows)), (v, numbers(rows[::-1]))):
        got = got[0, :, 0].double().cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True), np.argwhere((got != want) & ~np.isnan(want))[:5]


def magnitudes(c, b, see):
    """sum_t |v_t| over the tokens that a row sees, [T, H, d]"""
    V = np.array([np.abs(numbers(c.m.v[0, p, :, row])) for p, row in (c.m.at(b, t) for t in range(see.shape[1]))])
    V = V.repeat(c.H // V.shape[1], axis=1)
    return np.array([V[row].sum(0) for row in see])


def check(c, tag, mask=None, window=0, sinks=0):
    c.call(mask=mask, window=window, sinks=sinks)
    torch.cuda.synchronize()
    got, at, odd, worst = c.out.double().cpu().numpy(), 0, 0, 0.0
    for n, T, b in zip(c.lens, c.rows, c.slots):
        q = c.q[0, at:at + T]
        see = PO.see_tree(n, T, mask[at:at + T]) if mask is not None else PO.see_window(n, T, window, sinks)
        with np.errstate(all="ignore"):
            o, _, mass, size = PO.attend(c.m, b, q, see, numbers, 0)
        mine, fine = got[at:at + T], np.isfinite(o)
        assert np.array_equal(mine[~fine], o[~fine], equal_nan=True), f"{tag}: infinities and NaN, slot {b}"
        # Sums are float32 and divided at the end, of weights relative to the largest so far, in
        # the kernel for more than 32 rows of a group to one that may be behind by 2^8: a weight
        # is 1 there, or 2^8, at most, and so is a sum sum_t |v_t| times that.  Where this is 2^128
        # or more (here 2^8 times an element of 2^127.6) it may overflow before the division.
        lag = 256 if T * c.H // c.m.k.shape[2] > 32 else 1
        held = fine & (magnitudes(c, b, see) * lag * 1.01 < 2.0 ** 128)
        assert np.isfinite(mine[held]).all(), f"{tag}: finite places, slot {b}"
        held |= fine & np.isfinite(mine)
        E = (2 * (c.d + 8) * U * (size + 1) + 3 * (n + 64) * U)[..., None]
        with np.errstate(all="ignore"):
            tol = (E * mass + 2.0 ** -8 * (np.abs(o) + mass)) * (1 + 2.0 ** -7) + 1e-30
        worst = max(worst, float((np.abs(mine[held] - o[held]) / np.broadcast_to(tol, o.shape)[held]).max()))
        odd += int((~fine).sum())
        at += T
    assert worst <= 1, f"{tag}: {worst:.2f} of the bound"
    say(f"{tag}: ok, {odd} infinities and NaN, {worst:.3f} of the bound")
    return odd


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 4, 40])
@pytest.mark.parametrize("byte", [253, 254])
def test_large_scales_in_masked_places(byte, T, d):
    """Blocks of V of which some elements are infinite, some are large and most are zero,
    of tokens that some rows see and others do not."""
    c = Case(byte + T, [60, 150], [T, T], 4, 2, d, 16)
    inf, big = (7, 5) if byte == 253 else (5, 3)       # 6 and 3 times 2^126; 3 and 1.5 times 2^127
    for b, n in zip(c.slots, c.lens):
        places = sorted({n - 1, n - 2, n - T + 1 if T > 1 else n - 3, n - T - 10, 0})
        for i, t in enumerate(places):
            p, row = c.m.at(b, t)
            blk = i % (d // 32)
            codes = np.zeros(32, dtype=np.uint8)
            codes[2 * i], codes[2 * i + 10] = inf | (8 if i % 2 else 0), big       # a column of each token's own
            codes[31] = inf | (8 if i // (d // 32) % 2 else 0)                     # and one of both signs
            block = c.m.v[0, p, :, row]                                            # [G, row bytes], a copy
            block[:, 16 * blk:16 * blk + 16] = codes[0::2] | codes[1::2] << 4
            block[:, d // 2 + blk] = byte
            c.m.v[0, p, :, row] = block
    c.upload()
    assert check(c, f"causal {byte} T {T}") > 0
    assert check(c, f"window {byte} T {T}", window=25, sinks=3) > 0
    check(c, f"tree {byte} T {T}", mask=tree_masks(c.r, [T, T], 1))
