"""Plain 64-bit implementations of the operators of include/gwtf_stage.h, in
numpy, written from their formulas.  They share no code with the HIP library.

Arrays are float64 (inputs already rounded to the type under test); tokens,
targets and identities are int64.
"""
import numpy as np

F8_MAX = 448.0
SCALE_MIN = 2.0 ** -126
BLOCK = 128


def philox4x32(counter, key):
    """Ten rounds of Philox4x32 for arrays of counters (.., 4) and one key
    (2,): four 32-bit words (.., 4) as uint64."""
    mask = np.uint64(0xFFFFFFFF)
    c = [np.asarray(counter, dtype=np.uint64)[..., i] for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        a = c[0] * np.uint64(0xD2511F53)
        b = c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & mask,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1)


def embed(tokens, table, scale=1.0):
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[i] = scale * table[t]
    return out


def embed_grad(tokens, dout, vocab, scale=1.0):
    out = np.zeros((vocab, dout.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < vocab:
            out[t] += scale * dout[i]
    return out


def dropout_keep(rows, width, p, seed, site):
    """The mask [N][width] and the factor of kept values."""
    limit = int(np.rint(p * 65536))
    rows = np.asarray(rows, dtype=np.int64).astype(np.uint64)
    steps = (width + 7) // 8
    counter = np.zeros((len(rows), steps, 4), np.uint64)
    counter[..., 0] = np.arange(steps, dtype=np.uint64)
    counter[..., 1] = site
    counter[..., 2] = (rows & np.uint64(0xFFFFFFFF))[:, None]
    counter[..., 3] = (rows >> np.uint64(32))[:, None]
    words = philox4x32(counter, (seed & 0xFFFFFFFF, seed >> 32))
    u = np.stack((words & np.uint64(0xFFFF), words >> np.uint64(16)), -1).reshape(len(rows), steps * 8)
    return u[:, :width] >= limit, 65536.0 / (65536 - limit)


def dropout(x, p, seed, site, rows=None, residual=None):
    rows = np.arange(x.shape[0]) if rows is None else rows
    keep, factor = dropout_keep(rows, x.shape[1], p, seed, site)
    y = np.where(keep, x * factor, 0.0)
    return y if residual is None else residual + y


def norm(x, weight, eps, residual=None):
    """(h, rstd, y) before any rounding."""
    h = x if residual is None else x + residual
    rstd = 1.0 / np.sqrt(np.mean(h * h, 1) + eps)
    return h, rstd, h * rstd[:, None] * weight


def scales(y, quant):
    """One scale a row ("row") or for each 128 columns ("block")."""
    if quant == "row":
        m = np.abs(y).max(1, keepdims=True)
    else:
        m = np.stack([np.abs(y[:, c:c + BLOCK]).max(1) for c in range(0, y.shape[1], BLOCK)], 1)
    s = np.maximum(m / F8_MAX, SCALE_MIN)
    return np.where(np.isfinite(m), s, np.nan)


def spread(s, width, quant):
    """Scales by column."""
    return np.repeat(s, width if quant == "row" else BLOCK, 1)[:, :width]


def norm_grad(dy, h, weight, rstd, dh=None):
    xhat = h * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - xhat * np.mean(g * xhat, 1, keepdims=True))
    return (dx if dh is None else dx + dh), (dy * xhat).sum(0)


def logprob(logits, targets=None, top=0):
    """(logp, entropy, lse, top_logp, top_ids); rows without NaN or +infinity."""
    n, v = logits.shape
    lse = np.full(n, -np.inf)
    entropy = np.zeros(n)
    lp = np.full((n, v), -np.inf)
    for i, x in enumerate(logits):
        m = x.max()
        if m == -np.inf:
            continue
        e = np.exp(x - m)
        lse[i] = m + np.log(e.sum())
        lp[i] = x - lse[i]
        p = np.exp(lp[i])
        entropy[i] = -np.sum(p[p > 0] * lp[i][p > 0])
    logp = None
    if targets is not None:
        logp = np.array([lp[i, t] if 0 <= t < v else 0.0 for i, t in enumerate(targets)])
    ids = np.argsort(-logits, axis=1, kind="stable")[:, :top]
    return logp, entropy, lse, np.take_along_axis(lp, ids, 1), ids


def logprob_grad(logits, targets, lse, entropy, dlogp=None, dentropy=None):
    n, v = logits.shape
    out = np.zeros((n, v))
    for i, x in enumerate(logits):
        if lse[i] == -np.inf:
            continue
        lp = x - lse[i]
        p = np.exp(lp)
        if dentropy is not None:
            some = p > 0
            out[i][some] -= dentropy[i] * p[some] * (lp[some] + entropy[i])
        if dlogp is not None and 0 <= targets[i] < v:
            out[i] -= dlogp[i] * p
            out[i][targets[i]] += dlogp[i]
    return out
