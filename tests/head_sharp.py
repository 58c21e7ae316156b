"""Rows in which one entry holds nearly all of the student and of its teacher: the sharpest
test of the statistics that a row's loss and gradient are differences of.

Let R be the part that the entries other than that one hold (of the student or of the
teacher, whichever is larger).  The entry's own exponential is e^0, exactly 1 on both
sides, so only parts of R carry errors.  An exponential of argument x, |x| <= X, is off by
3 |x| 2^-24 (difference, scale, product) and 2 2^-24 (one unit in the last place); each of
at most n additions a thread makes, and the change of its running maximum before it, adds
3 2^-24, pairs and joins 8 2^-24: at most E = (3 X + 10 + 3 n) 2^-24 of itself.  So with
statistics of more than fp32 where they meet,
  loss       tau^2 R E (D + 3)         D the largest |ln p - ln q| of a value with mass
  gradient   tau w R E (4 q or p, and 1) at the large entry, E of the others' parts
beside the rounding of the result itself (2^-24 of a loss, its type's for a gradient).
fp32 statistics would be off by 2^-24 of 1, hundreds of times that."""
import numpy as np

import head_reference as ref

U = 2.0 ** -24


def case(rng, rows, V, k, tau):
    """Student and teacher logits [rows, V] in fp32, each row's large entry first of its k
    listed ones, and the teacher's rest in fp32 (None where every entry is listed)."""
    s = (rng.standard_normal((rows, V)) - tau * (np.log(V) + 9.0)).astype(np.float32)
    at = rng.integers(0, V, rows)
    s[np.arange(rows), at] = 5.25
    t = (s + 0.2 * tau * rng.standard_normal((rows, V))).astype(np.float32)
    t[np.arange(rows), at] = 4.5
    top = np.argsort(-t, axis=1, kind="stable")[:, :k]
    listed = np.take_along_axis(t, top, axis=1)
    if k == V:
        return s, listed, top, None
    left = t.astype(np.float64) / tau
    np.put_along_axis(left, top, -np.inf, axis=1)
    most = left.max(axis=1, keepdims=True)
    rest = (most[:, 0] + np.log(np.exp(left - most).sum(axis=1))).astype(np.float32)
    return s, listed, top, rest


def bounds(s, t, top, tau, rest, weight, bits, adds):
    """(loss, gradient, bound of the loss's error, bounds of the gradient's) of one row."""
    slots = list(zip(top.tolist(), t.tolist()))
    loss, grad = ref.distill_row(s, slots, tau, rest, weight)
    x = s.astype(np.float64) / tau
    values = t.astype(np.float64) / tau if rest is None else np.append(t.astype(np.float64) / tau, rest)
    q = np.exp(x - x.max())
    q /= q.sum()
    p = np.exp(values - values.max())
    p /= p.sum()
    other = np.ones(len(s), dtype=bool)
    other[top] = False
    qs = q[top] if rest is None else np.append(q[top], q[other].sum())
    R = max(1.0 - q.max(), 1.0 - p.max())
    X = max(np.ptp(x), np.ptp(values))
    E = (3 * X + 10 + 3 * adds) * U
    D = np.abs(np.log(p) - np.log(qs)).max()
    loss_bound = tau * tau * R * E * (D + 3) + U * loss * 2
    mine = np.zeros(len(s))                                  # p, and p_r q_i / q_r
    mine[top] = p[:len(top)]
    if rest is not None:
        mine[other] = p[-1] * q[other] / qs[-1]
    big = np.zeros(len(s), dtype=bool)
    big[top[0]] = True
    grad_bound = tau * abs(weight) * np.where(big, 4 * R * E, (q + mine) * 2 * E)
    grad_bound += np.abs(grad) * 2.0 ** -bits + (2.0 ** -25 if bits == 11 else 0.0)
    return loss, grad, loss_bound, grad_bound


def fp32_row(s, t, top, tau, rest, weight):
    """Loss and the large entry's gradient with the row's statistics rounded to fp32 as they
    meet: what the bounds are there to tell."""
    f = np.float32
    values = np.append((t / f(tau)).astype(f), f(rest))
    e_t = np.exp((values - values.max()).astype(f)).astype(f)
    x = ((s - s.max()) / f(tau)).astype(f)
    e_s = np.exp(x).astype(f)
    other = np.ones(len(s), dtype=bool)
    other[top] = False
    apart = f(e_s[other].astype(np.float64).sum())
    sum_t, whole = f(e_t.astype(np.float64).sum()), f(f(e_s[top].astype(np.float64).sum()) + apart)
    p = (e_t / sum_t).astype(f)
    log_p = ((values - values.max()) - np.log(sum_t)).astype(f)
    log_q = np.append((x[top] - np.log(whole)).astype(f), np.log(f(apart / whole)))
    loss = f(tau * tau) * f((p * (log_p - log_q)).astype(f).sum(dtype=np.float64))
    weighted = f(tau) * f(weight)
    inv_t, listed = f(1) / sum_t, weighted * (f(1) / whole)
    return float(loss), float(f(e_s[top[0]] * listed) - f(f(e_t[0] * inv_t) * weighted))


def even_case(rng, rows, V, tau, kind):
    """One listed entry, and all others equal: their exponentials against their own largest are
    1, their sum is exact, and so is the listed entry's e^0 on both sides.  What is left to be
    off is e^((mu - m) / tau) and e^(rest - t / tau), one each.  `kind` rounds to the logits'
    type.  Returns logits [rows, V], teacher [rows, 1], index [rows, 1] and rest, about a
    thousandth from the student's own."""
    at = rng.integers(0, V, rows)
    g = rng.uniform(0.1, 2.0, rows)
    low = kind((5.25 - tau * (np.log(V - 1.0) + g)).astype(np.float32))
    s = np.repeat(low[:, None], V, axis=1)
    s[np.arange(rows), at] = 5.25
    t = np.full((rows, 1), 4.5, np.float32)
    rest = 4.5 / tau + (low.astype(np.float64) - 5.25) / tau + np.log(V - 1.0) + 1e-3 * rng.standard_normal(rows)
    return s, t, at[:, None], rest.astype(np.float32)


def even_bounds(s, t, top, tau, rest, weight, bits):
    """As bounds(): the two exponentials within 3e-9 of themselves, each a part of its sum, so
    6e-9 (D + 1) tau^2, D the rest's |x - y| against the mean's."""
    loss, grad = ref.distill_row(s, [(int(top[0]), float(t[0]))], tau, rest, weight)
    x = s.astype(np.float64) / tau
    q = np.exp(x - x.max())
    q /= q.sum()
    D = abs((float(t[0]) / tau - rest) - (x[top[0]] - (x[top[0] - 1] + np.log(len(s) - 1.0))))
    # an unlisted entry: its factor's rounding, and its product's
    grad_bound = tau * abs(weight) * 2e-8 * q + np.abs(grad) * (2 * U + 2.0 ** -bits) + (2.0 ** -25 if bits == 11 else 0.0)
    return loss, grad, tau * tau * 6e-9 * (D + 1) + 2 * U * loss, grad_bound
