"""The definitions of stagefrontier_draw.h, as plain numpy in extended precision
and Python's whole numbers, with the error that each operator's last steps may
leave.  They share no code with the kernels or the binding.

Tokens are held to the definition's, but where the uniform number lies within
MARGIN of a border between two: the kernels' powers of two are within 2^-39.7,
sums of them as near, plus 2^-53 for each addition on the longest path, and a
place in the cumulative sums is a quotient of two of them: 2^-38.7 in all.
"""
import math

import numpy as np

U = 2.0 ** -24
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}
MARGIN = 2.0 ** -38
LEAST = 2.0 ** -30
TINIEST = np.longdouble(2.0) ** -700
LOST = "p and q of a draft are both too small to tell"
WORD = (1 << 32) - 1


def philox(counter, key):
    """Philox4x32-10 of one counter of four words, by Python's whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & WORD, (a >> 32) ^ c[3] ^ k[1], a & WORD]
        k = [(k[0] + 0x9E3779B9) & WORD, (k[1] + 0xBB67AE85) & WORD]
    return c


def words(seed, step, site, block, kind):
    return philox((block & WORD, (block >> 32) | kind << 31, site, step & WORD), (seed & WORD, (seed >> 32) & WORD))


def uniform(seed, step, site, first, n):
    return np.array([(words(seed, step, site, i // 4, 1)[i % 4] >> 8) * 2.0 ** -24 for i in range(first, first + n)])


def threshold(p):
    return math.floor(float(np.float32(p)) * 65536.0 + 0.5)


def kept(seed, step, site, p, indexes):
    """Whether each index is kept."""
    t, made, out = threshold(p), {}, []
    for e in np.asarray(indexes).reshape(-1).tolist():
        if e // 8 not in made:
            made[e // 8] = words(seed, step, site, e // 8, 0)
        out.append((made[e // 8][e % 8 // 2] >> 16 * (e % 2) & 0xFFFF) >= t)
    return np.array(out).reshape(np.shape(indexes))


def dropout(x, keep, p, residual, kind):
    """Outputs and the bounds of their errors: the scale, the product added to
    the residual and the type round once each."""
    t = threshold(p)
    scale = 65536.0 / (65536 - t) if t < 65536 else 0.0
    xs = np.where(keep, np.asarray(x, np.float64), 0.0) * scale
    y = xs if residual is None else xs + np.asarray(residual, np.float64)
    return y, U * np.abs(xs) + (U + HALF_ULP[kind]) * (1 + 2 * U) * np.abs(y) + U * U * np.abs(xs) + 1.01 * TINY[kind]


def softmax(x, inv_t):
    """p in extended precision; None for nothing but -inf, NaN where +inf or NaN is."""
    x = np.asarray(x, np.float64)
    if not (x < np.inf).all():
        return np.nan
    if x.max() == -np.inf:
        return None
    # products of a float and a float are exact in 64 bits
    z = (x * float(np.float32(inv_t))).astype(np.longdouble)
    e = np.exp(z - z.max())
    return e / e.sum()


def pick(weights, u, margin=MARGIN):
    """The token of a uniform number and those that a border within ``margin`` leaves."""
    c = np.cumsum(weights)
    c = c / c[-1]
    t = int(np.searchsorted(c, np.longdouble(u), side="right"))
    t = min(t, int(np.nonzero(weights)[0][-1]))
    near = {int(j) for j in np.nonzero((c > u - margin) & (c - weights / weights.sum() < u + margin) & (weights > 0))[0]}
    return t, near | {t}


def log_p(p):
    return float(np.log(p)) if p > 0 else -math.inf


def sample(x, u, inv_t):
    """(token, tokens allowed, logp of a token)."""
    if not 0.0 <= u < 1.0:
        return -1, {-1}, lambda t: 0.0
    p = softmax(x, inv_t)
    if p is None:
        return -1, {-1}, lambda t: -math.inf
    if np.ndim(p) == 0:
        return -1, {-1}, lambda t: math.nan
    return pick(p, u) + (lambda t: log_p(p[t]),)


def logp_bound(want):
    """One rounding, and the 64-bit steps before it."""
    return U * abs(want) + 2.0 ** -38 * (1 + abs(want)) if math.isfinite(want) else 0.0


def verify(target, drafts, draft, u, inv_t, draft_inv_t):
    """One sequence: target [n + 1, V], drafts [n, V] or None, draft [n], u
    [n + 1].  (accepted, tokens, tokens allowed at the last, function of its
    logp, log-probabilities of the accepted); None where a comparison is within
    MARGIN, and either answer is right."""
    n, logps = len(draft), []
    for k in range(n + 1):
        p = softmax(target[k], inv_t)
        V = len(target[k])
        if not 0.0 <= u[k] < 1.0:
            return k, {-1}, lambda t: 0.0, logps
        if p is None:
            return k, {-1}, lambda t: -math.inf, logps
        if np.ndim(p) == 0:
            return k, {-1}, lambda t: math.nan, logps
        weights = p
        if k < n and 0 <= draft[k] < V:
            d = draft[k]
            if drafts is None:
                q = np.zeros(V, np.longdouble)
                q[d] = 1.0
            else:
                q = softmax(drafts[k], draft_inv_t)
                if q is not None and np.ndim(q) == 0:
                    return k, {-1}, lambda t: math.nan, logps
                if q is None:
                    q = np.zeros(V, np.longdouble)
            # (what lies below 2^-700 of a row's largest may count as 0)
            if p[d] < TINIEST * p.max() and (u[k] == 0.0 or q[d] < TINIEST * max(q.max(), p.max())):
                return LOST
            if p[d] > 0 and abs(u[k] * q[d] - p[d]) < MARGIN * p[d]:
                return None
            if u[k] * q[d] < p[d]:
                logps.append(log_p(p[d]))
                continue
            weights = np.maximum(p - q, 0)
        if not 0.0 <= u[n] < 1.0:
            return k, {-1}, lambda t: 0.0, logps
        # what p and q leave of each other is only as good as they are: each is within 2^-38.7 of its size,
        # so cumulative sums of the differences within 2^-37.7, relative to the share that is left
        share = float(weights.sum())
        if share < LEAST:
            weights, share = p, 1.0
        t, near = pick(weights, u[n], 2 * MARGIN / share)
        return k, near, lambda t: log_p(p[t]), logps
