"""Logits of minus infinity that come from K itself: such a token has no
weight, and a row that sees no other gives what one gives that sees nothing."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from test_attend_gpu import Case, U, to_f64, to_store  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,T", [(50, 3), (50, 40), (1500, 2), (1500, 33)])
def test_tokens_of_logit_minus_infinity(dtype, n, T):
    """Every 7th token has logit 0, and then none: equal weights over those,
    bounds as in test_attend_gpu.py with X = 0 (their products are exact)."""
    c = Case(n + T, [n], [T], 4, 2, 64, 16, dtype)
    q = np.zeros(64)
    q[0] = 8.0
    c.q[...] = to_store(q, dtype)
    f, slot = to_f64(dtype), c.slots[0]
    for some in (True, False):
        k = np.zeros(64)
        for t in range(n):
            p, row = c.m.at(slot, t)
            k[0] = 0 if some and t % 7 == 0 else -np.inf
            c.m.k[0, p, :, row] = to_store(k, dtype)
        c.upload()
        c.call()
        torch.cuda.synchronize()
        got, lse = c.out.double().cpu().numpy(), c.lse.double().cpu().numpy()
        if not some:
            assert (got[:T] == 0).all() and np.isneginf(lse[:T]).all()
            continue
        v = np.stack([f(c.m.v[0, c.m.at(slot, t)[0], :, c.m.at(slot, t)[1]]) for t in range(0, n, 7)])
        E = 2 * 72 * U + 3 * (n + 64) * U
        for i in range(T):
            m = (n - T + i) // 7 + 1
            want, mass = v[:m].mean(0).repeat(2, 0), np.abs(v[:m]).mean(0).repeat(2, 0)
            low = 2.0 ** -8 if dtype == "bf16" else U          # the weights are 1, exactly
            assert np.all(np.abs(got[i] - want) <= E * mass + low * np.abs(want))
            assert np.all(np.abs(lse[i] - np.log(m)) <= E + 2 * U * np.log(m))
