"""The bounds of head_sharp.py themselves, on the CPU: they hold the 64-bit rows, and tell
statistics that are rounded to fp32."""
import numpy as np
import pytest

import head_sharp as sharp


@pytest.mark.parametrize("V,k,tau", ((700, 9, 1.0), (5003, 33, 2.0), (20011, 64, 0.7)))
def test_the_bounds_tell_fp32_statistics(V, k, tau):
    rng = np.random.default_rng(V)
    rows = 64
    s, t, top, rest = sharp.case(rng, rows, V, k, tau)
    weight = rng.uniform(0.5, 3.0, rows).astype(np.float32)
    tau = float(np.float32(tau))
    told = np.zeros(2, dtype=int)
    for r in range(rows):
        loss, grad, loss_bound, grad_bound = sharp.bounds(s[r], t[r], top[r], tau, float(rest[r]), float(weight[r]), 24, 40)
        assert 0 < loss_bound < 0.3 * sharp.U * tau * tau and (grad_bound[top[r][0]] < 0.05 * sharp.U * tau * weight[r])
        assert loss > loss_bound                        # a few parts in 10^7: not lost beside it
        l32, g32 = sharp.fp32_row(s[r], t[r], top[r], tau, float(rest[r]), float(weight[r]))
        told += (abs(l32 - loss) > loss_bound, abs(g32 - grad[top[r][0]]) > grad_bound[top[r][0]])
    assert told.min() > rows // 2, told
