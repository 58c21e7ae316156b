"""The tests' plain sampling and distillation themselves, on the CPU: whole-number weights
against the exponential, draws against real probabilities, gradients against differences."""
import math

import numpy as np
import pytest

import head_reference as ref


def test_weights_are_the_exponential_to_24_bits():
    rng = np.random.default_rng(0)
    l = np.sort(np.concatenate([rng.uniform(-30, 0, 20000), [0.0]]).astype(np.float32))
    w, _ = ref.weights(l, 1.0)
    z = l * ref.LOG2E                                # fp32, as the definition has it
    real = np.where(z >= -41, np.exp2(z.astype(np.float64)) * 2.0 ** 40, 0.0)
    # three parts: the polynomial's 9.2e-8, its roundings in fp32, and the truncation
    # (one unit of 2^-24 at the top, then whole numbers)
    assert np.all(np.abs(w - real) <= real * 3e-7 + 1.0)
    assert w[-1] == 1 << 40
    assert np.all(np.diff(w) >= 0)


@pytest.mark.parametrize("T,top_k,top_p,min_p", [(1.0, 0, 1.0, 0.0), (0.5, 0, 0.8, 0.0), (2.0, 7, 1.0, 0.0),
                                                 (1.3, 20, 0.6, 0.0), (1.0, 0, 1.0, 0.1), (0.9, 50, 0.9, 0.02)])
def test_draws_follow_the_real_probabilities(T, top_k, top_p, min_p):
    """The token is the one the real numbers give, except where u or a cut lies within
    2e-6 of a boundary."""
    rng = np.random.default_rng(1)
    T, top_p, min_p = (float(np.float32(x)) for x in (T, top_p, min_p))       # as the call takes them
    off = 0
    for _ in range(200):
        l = (rng.standard_normal(60) * 2).astype(np.float32)
        u = np.float32(rng.integers(0, 1 << 24) / 2 ** 24)
        p = np.exp((l.astype(float) - l.max()) / T)
        order = np.argsort(-l, kind="stable")
        keep = np.zeros(60, bool)
        keep[order[:top_k or 60]] = True
        mass = np.cumsum(p[order] * keep[order]) / (p * keep).sum()
        close = False
        if top_p < 1:
            first = np.concatenate([[0.0], mass[:-1]])
            keep[order[~(first < top_p)]] = False
            close = np.abs(first - top_p).min() < 2e-6
        close = close or (min_p > 0 and np.abs(p - min_p).min() < 2e-6)
        keep &= p >= min_p
        run = np.cumsum(np.where(keep, p, 0.0)) / (p * keep).sum()
        close = close or np.abs(run - u).min() < 2e-6
        want = int(np.argmax(run > u))
        got, logp = ref.sample_row(l, u, T, top_k, top_p, min_p)
        if got != want:
            assert close
            off += 1
        else:
            assert abs(logp - math.log(p[want] / (p * keep).sum())) < 1e-9 or close
    assert off <= 2


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("tau", [0.7, 1.0, 3.0])
def test_gradient_is_the_loss_difference(rest, tau):
    rng = np.random.default_rng(2)
    for V, k in ((2, 1), (5, 5), (40, 7)):
        if rest and k == V:
            continue
        s = rng.standard_normal(V) * 2
        slots = list(zip(rng.permutation(V)[:k].tolist(), (rng.standard_normal(k) * 2).tolist()))
        slots.append((slots[0][0], 9.0))             # a repeated entry and an empty slot count nothing
        slots.append((-1, 50.0))
        r = float(rng.standard_normal()) if rest else None
        loss, g = ref.distill_row(s, slots, tau, r)
        assert loss >= 0
        for i in range(V):
            h = 1e-5
            hi, lo = s.copy(), s.copy()
            hi[i] += h
            lo[i] -= h
            d = (ref.distill_row(hi, slots, tau, r)[0] - ref.distill_row(lo, slots, tau, r)[0]) / (2 * h)
            assert abs(d - g[i]) < 1e-8


def test_masked_rows_of_the_reference():
    assert ref.sample_row([-np.inf] * 3, 0.5) == (-1, 0.0)
    assert ref.sample_row([1, 3, 3], 0.9, T=0.0) == (1, 0.0)
    loss, g = ref.distill_row([1.0, np.nan], [(-1, 0.0)], 1.0)
    assert loss == 0 and not g.any()
    loss, g = ref.distill_row([-np.inf, 0.0], [(0, 1.0)], 2.0)
    assert loss == np.inf and np.array_equal(g, [-2.0, 2.0])
