"""Plain implementations of the output head's operators for the tests: sampling with
whole-number weights row by row, distillation in 64 bits."""
from __future__ import annotations

import math

import numpy as np

LOG2E = np.float32(1.4426950408889634)
POLY = [np.float32(float.fromhex(c) * 2.0 ** 24) for c in
        ("0x1p0", "0x1.62e42ap-1", "0x1.ebf9bcp-3", "0x1.c6b754p-5", "0x1.3cea84p-7", "0x1.5bb994p-10")]


def weights(l, T):
    """(weights as Python-int-safe int64, scaled logits z) of a row of float32 logits."""
    l = np.asarray(l, dtype=np.float32)
    l = np.where(np.isnan(l), np.float32(-np.inf), l)
    m = l.max()
    with np.errstate(all="ignore"):
        c = np.float32(LOG2E / np.float32(T))
        z = np.where(l == m, np.float32(0), (l - m) * c).astype(np.float32)
        live = (z >= np.float32(-41.0)) & (l > -np.inf)
    z = np.where(live, z, np.float32(0))
    n = np.rint(z)
    f = z - n
    P = POLY[5] * np.ones_like(f)
    for i in (4, 3, 2, 1, 0):
        P = P * f + POLY[i]
    w = (P.astype(np.int64) << 16) >> (-n).astype(np.int64)
    return np.where(live, w, 0), z


def sample_row(l, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability, size of the kept probability mass) of one row."""
    l = np.asarray(l, dtype=np.float32)
    l = np.where(np.isnan(l), np.float32(-np.inf), l)
    V = len(l)
    T, top_p, min_p, u = (np.float32(x) for x in (T, top_p, min_p, u))
    if not (l > -np.inf).any():
        return -1, 0.0
    m = l.max()
    if not T > 0 or top_k == 1 and V > 1:
        return int(np.argmax(l == m)), 0.0
    w, _ = weights(l, T)
    order = sorted(range(V), key=lambda i: (-l[i], i)) if V < 4096 else np.lexsort((np.arange(V), -l)).tolist()
    k = top_k if 0 < top_k < V else V
    ranked = order[:k]
    if top_p < 1:
        whole = sum(int(w[i]) for i in ranked)
        target = (whole * int(np.float32(max(top_p, np.float32(0))) * np.float32(2 ** 24))) >> 24
        before, kept = 0, []
        for i in ranked:
            if kept and before >= target:
                break
            kept.append(i)
            before += int(w[i])
        ranked = kept
    if min_p > 0:
        least = int(np.float32(min(min_p, np.float32(1))) * np.float32(2.0 ** 40))
        ranked = [i for i in ranked if int(w[i]) >= least]
    keep = np.zeros(V, dtype=bool)
    keep[ranked] = True
    keep &= w > 0
    index = np.flatnonzero(keep)
    whole = sum(int(w[i]) for i in index)
    u = np.float32(0) if not u > 0 else min(u, np.float32(1 - 2.0 ** -24))
    target = (whole * int(u * np.float32(2 ** 24))) >> 24
    running = 0
    for token in index:
        running += int(w[token])
        if running > target:
            break
    with np.errstate(all="ignore"):
        x = np.where(l[index] == m, 0.0, (l[index].astype(np.float64) - np.float64(m)) / np.float64(T))
        at = 0.0 if l[token] == m else (float(l[token]) - float(m)) / float(T)
        return int(token), float(at - np.log(np.exp(x).sum()))


def logp_tolerance(logp, x):
    """Bound on the error of a float32 log-probability logp = x - ln(sum), x <= 0: one
    rounding each of difference, quotient and subtraction; the weights' relative error 2e-7
    and the sum's conversion in the logarithm, and the logarithm's own 2^-22 of its value."""
    return 2.0 ** -22 * (abs(x) + abs(logp - x)) + 2.0 ** -24 * abs(logp) + 4e-7


def distill_row(s, slots, tau, rest=None, weight=1.0):
    """(loss, gradient, tolerance data) of one row in 64 bits.  slots: (entry, logit)."""
    s = np.asarray(s, dtype=np.float64)
    V = len(s)
    seen = {}
    for i, t in slots:
        if 0 <= i < V and int(i) not in seen:
            seen[int(i)] = float(t) / tau
    values = list(seen.values()) + ([] if rest is None else [float(rest)])
    if not values or (max(values) == -math.inf and not any(math.isnan(v) for v in values)):
        return 0.0, np.zeros(V)
    with np.errstate(all="ignore"):
        t = np.array(values)
        mt = t.max()
        lp = t - mt - np.log(np.exp(t - mt).sum())
        x = s / tau
        m = x.max()
        lq = np.full(V, -np.inf) if m == -np.inf else x - m - np.log(np.exp(x - m).sum())
        entries = list(seen)
        p = np.exp(lp)
        div = lambda a, b, c: 0.0 if a == 0 else a * (b - c)  # noqa: E731
        loss = sum(div(p[j], lp[j], lq[i]) for j, i in enumerate(entries))
        q = np.exp(lq)
        g = q.copy()
        if rest is not None:
            other = np.ones(V, dtype=bool)
            other[entries] = False
            top = lq[other].max() if other.any() else -np.inf
            lr = -np.inf if top == -np.inf else top + np.log(np.exp(lq[other] - top).sum())
            loss += div(p[-1], lp[-1], lr)
            if lr > -np.inf or np.isnan(lr):
                g[other] = q[other] - p[-1] * np.exp(lq[other] - lr)     # q_r itself may underflow
        for j, i in enumerate(entries):
            g[i] -= p[j]
    return tau * tau * loss, (g * (tau * weight) if weight else np.zeros(V))


def distill_tolerance(s, slots, tau, rest, weight, dtype_bits):
    """Bounds on the errors of float32 arithmetic for distill_row's loss and gradient.

    An exponential's argument carries three roundings (|x| 3 2^-24), the unit one ulp; a
    thread adds at most 160 of them in a row and the workgroup's tree 32 more, so a sum
    of n is within (3 X + 2 + min(n, 192)) 2^-24 of itself, X the largest |x|.  A
    probability adds its own exponential and a division, a logarithm 2^-22 of its
    value.  Gradients are rounded once to dtype_bits of significand (and at the least to
    the 16-bit types' subnormals)."""
    eps = 2.0 ** -24
    s = np.asarray(s, dtype=np.float64)
    V = len(s)
    seen = {}
    for i, t in slots:
        if 0 <= i < V and int(i) not in seen:
            seen[int(i)] = float(t) / tau
    values = np.array(list(seen.values()) + ([] if rest is None else [float(rest)]))
    t = values[np.isfinite(values)]
    x = s[np.isfinite(s)] / tau
    if not len(t):
        return 0.0, np.zeros(V)
    if not len(x):
        x = np.zeros(1)                              # a row of -inf: q = 0, the loss infinite
    Xt, Xs = t.max() - t.min() + np.abs(t).max(), x.max() - x.min() + np.abs(x).max()
    ep = 2 * (3 * Xt + 4 + min(len(values), 192)) * eps
    eq = 2 * (3 * Xs + 4 + min(V, 192)) * eps
    lp = values - t.max() - np.log(np.exp(t - t.max()).sum())
    p = np.exp(lp)
    lq = s / tau - x.max() - np.log(np.exp(x - x.max()).sum())
    q = np.exp(lq)
    entries = list(seen)
    lqs = [lq[i] for i in entries]
    other = np.ones(V, dtype=bool)
    other[entries] = False
    if rest is not None:
        far = x.max() if not other.any() else lq[other].max()
        lr = far + np.log(np.exp(lq[other] - far).sum()) if np.isfinite(far) and other.any() else -np.inf
        lqs.append(lr)
    part = np.zeros(V)                               # p_r q_i / q_r
    if rest is not None and lqs[-1] > -np.inf:
        part[other] = p[-1] * np.exp(lq[other] - lqs[-1])
    terms = [(pj, a, b) for pj, a, b in zip(p, lp, lqs) if pj > 0 and np.isfinite(b)]
    loss = tau * tau * sum(pj * ((ep + 8 * eps) * abs(a - b) + ep + eq + 8 * eps * (abs(a) + abs(b) + 1)) for pj, a, b in terms)
    pl = np.zeros(V)
    for j, i in enumerate(entries):
        pl[i] = p[j]
    g = tau * abs(weight) * (q * (eq + 4 * eps) + pl * (ep + 4 * eps) + part * (ep + 2 * eq + 4 * eps))
    _, exact = distill_row(s, slots, tau, rest, weight)
    low = {24: 0.0, 8: 0.0, 11: 2.0 ** -25}[dtype_bits]
    return loss + 1e-37, g * (1 + 2.0 ** -dtype_bits) + np.abs(exact) * 2.0 ** -dtype_bits + low + 1e-37
