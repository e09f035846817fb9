"""Log probabilities where logits are finite and large: masks by values such as
-1e10, whole rows of them, and entries that are as large above 0.

The 64-bit values are computed from the differences to a row's maximum, which
64 bits hold exactly for these inputs where they count.  Bounds as in
test_gpu_stage.py; beyond 1e5, where 32 bits of lse do not resolve a probability,
logp is held to the difference of the logit and the row's maximum.
"""
import numpy as np
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_stage import E, close, f64, ids, matrix, ops, torch_

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

KINDS = 8


def rows_of(r, n, v, size):
    """Row i is of kind i % KINDS."""
    a = r.standard_normal((n, v)) * 3
    unit, lane = np.arange(v) // 16, np.arange(v) // 16 % 256
    for i in range(n):
        kind = i % KINDS
        if kind == 0:  # the first columns of several lanes, and single units later
            a[i, (unit % 7 == 0) | (unit < 3)] = -size
        elif kind == 1:  # lanes that see nothing else
            a[i, lane < 200] = -size
            a[i, -1] = 0.5
        elif kind == 2:
            a[i, r.random(v) < 0.5] = -size
        elif kind == 3:  # one word is left
            a[i] = -size
            a[i, int(r.integers(v))] = 1.25
        elif kind == 4:
            a[i] = -size
        elif kind == 5:
            a[i] = size
        elif kind == 6:
            a[i] = -size * (1 + 0.125 * r.integers(0, 3, v))
        else:
            a[i, int(r.integers(v))] = size
    return a


def from_maximum(x):
    m = x.max(1, keepdims=True)
    d = x - m
    e = np.exp(d)
    s = e.sum(1, keepdims=True)
    p, ln_s = e / s, np.log(s)
    lp = d - ln_s
    entropy = -np.where(p > 0, p * lp, 0).sum(1)
    chain = 16 * (x.shape[1] // 4096 + 1) + 3 * 20
    d1, d2 = (p * np.abs(d)).sum(1), (p * d * d).sum(1)
    b = (chain + 8 + 2 * d1) * E
    ent_b = b + (chain + 8) * E * d1 + 2 * E * d2 + b * d1 + 4 * E * np.abs(entropy)
    return m[:, 0], lp, (m + ln_s)[:, 0], entropy, p, b, ent_b


SIZES = [("float16", 5e4)] + [(t, z) for t in ("float32", "bfloat16")
                              for z in (8e4, 1.5e5, 3e6, 1e9, 5e9, 1e10, 1e18, 1e20, 1e30)]


@pytest.mark.parametrize("dtype, size", SIZES)
@pytest.mark.parametrize("n, v, top", [(9, 37, 3), (16, 5003, 8), (8, 70001, 20), (600, 700, 2), (520, 9000, 5), (9, 4500, 40)])
def test_logprob_of_large_finite_values(dtype, size, n, v, top):
    torch = torch_()
    r = np.random.default_rng(v)
    x, xv = matrix(r, n, v, dtype, a=rows_of(r, n, v, size), pad=v % 3)
    tok = r.integers(0, v, n)
    m, lp, lse, entropy, p, b, ent_b = from_maximum(xv)
    dlogp, dent = r.standard_normal(n), r.standard_normal(n)
    dev = lambda a: torch.from_numpy(a).to("cuda", torch.float32)  # noqa: E731
    with ops(n, 1, v) as s:
        got = s.logprob(x, ids(tok), top=top)
        grad = s.logprob_grad(x, ids(tok), got[2], got[1], dev(dlogp), dev(dent))
    close(f64(got[2]), lse, b + 3 * E * np.abs(lse), "lse")
    close(f64(got[1]), entropy, ent_b, "entropy")
    # of a probability: that of lse, or beyond 1e5 that of the differences
    off = b + 3 * E * np.where(np.abs(m) > 1e5, 0, np.abs(lse))
    want = lp[np.arange(n), tok]
    close(f64(got[0]), want, off + 4 * E * np.abs(want), "logp")
    order = np.argsort(-xv, axis=1, kind="stable")[:, :top]
    assert (got[4].cpu().numpy() == order).all()
    want = np.take_along_axis(lp, order, 1)
    close(f64(got[3]), want, off[:, None] + 4 * E * np.abs(want), "top_logp")
    # gradients: finite everywhere, the formula's where lse resolves p
    assert bool(torch.isfinite(grad).all())
    some = np.abs(m) < 100
    d = np.maximum(xv - f64(got[2])[:, None], -1e4)[some]
    q, ge, gl, e = np.exp(d), f64(dev(dent))[some, None], f64(dev(dlogp))[some, None], f64(got[1])[some, None]
    want = -q * (gl + ge * (d + e))
    want[np.arange(len(want)), tok[some]] += gl[:, 0]
    u = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[dtype]
    size_ = np.abs(gl) + np.abs(ge) * (np.abs(d) + np.abs(e))
    close(f64(grad)[some], want, (10 + 4 * np.abs(d)) * E * q * size_ + (u + 2 * E) * np.abs(want) + 2.0 ** -25 * 2.0 ** -100
          * size_ + {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}[dtype], "dlogits")
