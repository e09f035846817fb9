"""Plain implementations of the operators of include/gwtf_learn.h in numpy,
written from their formulas: 64 bits or more, except where 8-bit states follow
32-bit arithmetic bit for bit.  They share no code with the HIP library.
"""
import numpy as np

from .stage import philox4x32

BLOCK = 128
_MOST = {"e4m3": 448.0, "e5m2": 57344.0}
_MANTISSA = {"e4m3": 3, "e5m2": 2}
_LEAST = {"e4m3": 2.0 ** -9, "e5m2": 2.0 ** -16}


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log probability, tokens that stay, margin) of one row of logits:
    margin is how near u or top_p lie to the next border, relative to the sums."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any() or (x == np.inf).any():
        return -1, np.nan, 0, np.inf
    if not (0 <= temperature < np.inf and top_p >= 0 and 0 <= min_p <= 1):
        return -1, np.nan, 0, np.inf
    live = np.flatnonzero(x > -np.inf)
    if len(live) == 0:
        return -1, -np.inf, 0, np.inf
    order = live[np.argsort(-x[live], kind="stable")]
    margin = np.inf
    if temperature == 0:
        order = order[:1]
        w = np.ones(1, np.longdouble)
    else:
        w = np.exp(((x[order] - x[order[0]]) / np.float64(temperature)).astype(np.longdouble))
        first = len(order) if top_k <= 0 else min(top_k, len(order))
        n = first
        if top_p < 1:
            c = np.cumsum(w[:first])
            # The product is a 64-bit number, as the sums are: 0.9 in 64 bits times 40 equal weights is 36 + 8.9e-16,
            # which 64 bits hold as 36, and 36 tokens reach it.
            target = np.float64(top_p) * np.float64(c[-1])
            n = min(first, int((c < target).sum()) + 1)
            margin = float(np.abs(c - target).min() / c[-1])
        if min_p > 0:
            n = min(n, int((w >= min_p).sum()))
            margin = min(margin, float(np.abs(w - np.longdouble(min_p)).min()))
        order, w = order[:n], w[:n]
    by_index = np.argsort(order)
    order, w = order[by_index], w[by_index]
    c = np.cumsum(w)
    u = 0.0 if not u >= 0 else u
    above = np.flatnonzero(c > u * c[-1])
    at = above[0] if len(above) else int(np.flatnonzero(w > 0)[-1])
    margin = min(margin, float(np.abs(c - u * c[-1])[:-1].min() / c[-1])) if len(c) > 1 else margin
    return int(order[at]), float(np.log(w[at] / c[-1])), len(order), margin


def grad_norm(grads, max_norm=np.inf, scale=1.0):
    norm = scale * np.sqrt(sum(np.sum(np.asarray(g, np.float64) ** 2) for g in grads))
    if not norm < 2.0 ** 128 - 2.0 ** 103:  # infinite in 32 bits
        return norm, np.nan
    return norm, scale * (min(1.0, max_norm / norm) if norm > 0 else 1.0)


def adamw(p, g, m, v, lr, step, betas, eps, decay, factor=1.0):
    """(p, m, v) in 64 bits."""
    b1, b2 = betas
    g = g * factor
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p - lr * (m / (1 - b1 ** step) / (np.sqrt(v / (1 - b2 ** step)) + eps) + decay * p), m, v


def moments32(g, m, v, betas, factor=1.0):
    """The new m and v in 32-bit arithmetic, each operation rounded by itself."""
    f = np.float32
    g = g.astype(f) * f(factor)
    m = m.astype(f) * f(betas[0]) + g * f(1 - betas[0])
    return m, v.astype(f) * f(betas[1]) + g * g * f(1 - betas[1])


def draws(size, seed, site, step, first=0):
    """16 random bits for each of a tensor's values from number `first` on, a multiple of eight."""
    n = -(-size // 8)
    i = np.arange(first // 8, first // 8 + n, dtype=np.uint64)
    counter = np.stack((i, np.full(n, site, np.uint64), np.full(n, step & 0xFFFFFFFF, np.uint64),
                        np.full(n, step >> 32, np.uint64)), -1)
    words = philox4x32(counter, (seed & 0xFFFFFFFF, seed >> 32))
    return np.stack((words & np.uint64(0xFFFF), words >> np.uint64(16)), -1).reshape(-1)[:size].astype(np.float64)


def narrow(x, r, kind):
    """(values in units of the scale, scales) that 8 bits hold of x: the magnitude in steps, and a remainder of
    (r + 1/2) 2^-16 steps, cut down to whole steps; the sum is one of 32 bits where steps are the smallest."""
    x = np.asarray(x, np.float64)
    scales = np.empty(-(-len(x) // BLOCK), np.float32)
    out = np.empty(len(x))
    for b in range(len(scales)):
        y = x[b * BLOCK:(b + 1) * BLOCK]
        most = np.abs(y).max() if np.isfinite(y).all() else np.nan
        if not np.isfinite(most):
            scales[b], out[b * BLOCK:(b + 1) * BLOCK] = np.nan, 0.0
            continue
        e = -126
        while most * 2.0 ** -e > _MOST[kind]:
            e += 1
        a = np.abs(y) * 2.0 ** -e
        step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(a, 1e-300))) - _MANTISSA[kind]), _LEAST[kind])
        total = a / step + (r[b * BLOCK:(b + 1) * BLOCK] + 0.5) / 65536
        normal = _LEAST[kind] * 2.0 ** _MANTISSA[kind]
        q = np.floor(np.where(a < normal, total.astype(np.float32), total)) * step
        if kind == "e5m2":
            q[(a > 0) & (q == 0)] = _LEAST[kind]
        scales[b], out[b * BLOCK:(b + 1) * BLOCK] = 2.0 ** e, np.where(y < 0, -q, q)
    return out, scales
