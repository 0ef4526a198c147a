"""The definitions of stagefrontier_train.h in 64 bits, as plain numpy, with the
error that each operator's 32-bit steps may leave.  They share no code with the
kernels or the binding.

Error bounds take u = 2^-24, the rounding of a 32-bit operation, and count
roundings from the formulas: differences, products and sums round once each, an
exponential is within 2 u of the true one plus its argument's error, a sum of n
terms is within n u of the terms' absolute sum.
"""
import math

import numpy as np

U = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -125, "bf16": 2.0 ** -125, "f16": 2.0 ** -25}


def row_stats(x, inv_t):
    """(m, s, u) of a row in 64 bits, z = x * inv_t, relative to its maximum."""
    z = np.asarray(x, dtype=np.float64) * inv_t
    m = z.max()
    if m == -np.inf:
        return m, 0.0, 0.0
    with np.errstate(invalid="ignore"):
        t = z - m
    e = np.exp(t)
    t[e == 0] = 0.0
    return m, e.sum(), (e * t).sum()


def token_logp(x, t, inv_t):
    """logp, lse, entropy of one row and the bounds of their errors.

    The exponents' error is 3 u of their size (difference, scale, constant),
    which the terms weigh by their probability; 2 u of each exponential; the
    sum's terms meet at most len(x) / 64 + 64 others one after the other.
    """
    V = len(x)
    if not 0 <= t < V:
        return (0.0, 0.0, 0.0), (0.0, 0.0, 0.0)
    m, s, u = row_stats(x, inv_t)
    if m == -np.inf:
        return (-np.inf, -np.inf, 0.0), (0.0, 0.0, 0.0)
    ls, zt = math.log(s) if s == s else np.nan, float(x[t]) * inv_t
    depth = -u / s
    logp, lse, h = zt - m - ls, m + ls, ls + depth
    steps = V / 64 + 64
    err_s = U * (steps + 4 + 4 * (depth + 1))
    e_logp = err_s + 4 * U * abs(zt - m if zt > -np.inf else 0.0) + U * (abs(ls) + abs(logp if logp > -np.inf else 0.0))
    e_lse = err_s + 2 * U * abs(m) + 2 * U * abs(lse) + U * abs(ls)
    e_h = (err_s + 4 * U) * (2 + 2 * depth) + 2 * U * (abs(ls) + abs(h)) + 4 * U * depth
    return (logp, lse, h), (e_logp, e_lse, e_h)


def token_logp_grad(x, t, inv_t, lse, entropy, g, h, kind):
    """The gradient of one row, and the bound of its error as stored in ``kind``."""
    x = np.asarray(x, dtype=np.float64)
    V = len(x)
    if not 0 <= t < V or lse == -np.inf:
        return np.zeros(V), np.zeros(V)
    q = x * inv_t - lse
    p = np.exp(q)
    live = p > 0
    qf = np.where(live, q, 0.0)
    y = -p * (g + h * (qf + entropy))
    y = np.where(live, y, 0.0)
    hot = np.zeros(V)
    hot[t] = g
    y = (y + hot) * inv_t
    size = p * (abs(g) + abs(h) * (np.abs(qf) + abs(entropy))) * inv_t
    # the exponent: one rounding of itself, of its constant and of its product;
    # then the products and sums of the formula
    err = U * size * (3 * np.abs(qf) + 12) + U * 6 * np.abs(hot) * inv_t
    return y, err + HALF_ULP[kind] * (np.abs(y) + err) + TINY[kind]


def policy(logp, old, ref, adv, per_token, mask, start, reduction, scale, lo, hi, beta):
    """terms, grad and the bounds of their errors.  reduction: 0 mean over
    tokens, 1 over sequences, 2 sum."""
    N, B = len(logp), len(start) - 1
    seq = np.full(N, -1)
    for b in range(B):
        seq[start[b]:start[b + 1]] = b
    on = (seq >= 0) & (np.ones(N, bool) if mask is None else np.asarray(mask) != 0)
    w = np.zeros(N)
    if reduction == 0 and on.any():
        w[on] = scale / on.sum()
    elif reduction == 1 and on.any():
        count = np.bincount(seq[on], minlength=B)
        w[on] = scale / (count[seq[on]] * (count > 0).sum())
    elif reduction == 2:
        w[on] = scale
    terms, size, grad, bound = np.zeros(4), np.zeros(4), np.zeros(N), np.zeros(N)
    big = float(np.finfo(np.float32).max)
    for i in np.nonzero(on)[0]:
        a = float(adv[i] if per_token else adv[seq[i]])
        d = float(logp[i]) - float(old[i])
        r = min(math.exp(min(d, 700.0)), big)
        over, under = a > 0 and d > math.log1p(hi), a < 0 and d < math.log1p(-lo)
        surr = -a * ((1 + hi) if over else (1 - lo) if under else r)
        gr = 0.0 if over or under else surr
        kl = em1 = x = 0.0
        if ref is not None:
            x = float(ref[i]) - float(logp[i])
            if x > 88.72:
                kl = em1 = big
            else:
                em1 = math.expm1(x)
                kl = em1 - x
        terms += w[i] * np.array([surr + beta * kl, surr, kl, float(over or under)])
        grad[i] = w[i] * (gr - beta * em1)
        # d and x are differences of two 32-bit numbers: u of their size; the
        # exponential 2 u; products and the weight 4 u.  kl near 0 is x^2 / 2
        # and more, so the error of x counts twice.
        e_surr = abs(surr) * U * (abs(d) + 8)
        e_kl = U * (10 * abs(kl) + 2 * abs(em1 * x) + (2 * abs(x) if abs(x) > 0.5 else 0.0))
        e_em1 = U * (10 * abs(em1) + math.exp(min(x, 88.0)) * abs(x))
        bound[i] = abs(w[i]) * (abs(gr) * U * (abs(d) + 8) + abs(beta) * e_em1) + 2 * U * abs(grad[i])
        size += abs(w[i]) * np.array([e_surr + abs(beta) * e_kl, e_surr, e_kl, 4 * U])
    return terms, size + 2 * U * np.abs(terms), grad, bound


def norms(tensors):
    """Per tensor and in all, in 64 bits, and the counts of entries that are
    not finite."""
    per = [float(np.sqrt(np.sum(np.asarray(t, np.float64) ** 2))) for t in tensors]
    wrong = [int((~np.isfinite(np.asarray(t, np.float64))).sum()) for t in tensors]
    return per, float(np.sqrt(np.sum(np.square(np.array(per, np.float64))))), wrong
