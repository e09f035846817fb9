"""Microbatch operators on the GPU against the plain 64-bit implementations of
oracle/stage.py.

Tolerances.  U is the unit roundoff of the output's type and E = 2^-24 that of
32-bit sums.  A sum of n terms in any order is off by at most n * E * sum of the
magnitudes; an elementary step (product, root, quotient, exponential) by a few
E; the output's own rounding by U of the value (plus half the least subnormal
number).  Each test adds these up along its formula.
"""
import numpy as np
import pytest

from oracle import stage as O
from tests.gpu_util import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

E = 2.0 ** -24
U = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}
TYPES = list(U)
SENTINEL = 77.0


def torch_():
    import torch
    return torch


def dt(name):
    return getattr(torch_(), name)


def ops(n, h=1, v=1, **kw):
    from paper_2509_21221_amd.stage import StageOps
    return StageOps(max(n, 1), h, v, **kw)


def matrix(r, n, w, dtype, std=1.0, pad=0, a=None):
    """(device tensor with rows w + pad apart, the same values in float64)."""
    torch = torch_()
    a = r.standard_normal((n, w)) * std if a is None else a
    full = torch.full((n, w + pad), SENTINEL, dtype=dt(dtype), device="cuda")
    full[:, :w] = torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dt(dtype))
    return full[:, :w], full[:, :w].double().cpu().numpy()


def empty(n, w, dtype, pad=0):
    """Output rows w + pad apart in a buffer of sentinels."""
    full = torch_().full((n, w + pad), SENTINEL, dtype=dt(dtype), device="cuda")
    return full[:, :w], full


def f64(t):
    return t.double().cpu().numpy()


def ids(a, dtype="int64"):
    return torch_().from_numpy(np.asarray(a)).to("cuda", dt(dtype))


def untouched(full, w):
    assert bool((full[:, w:] == SENTINEL).all())


def close(got, want, bound, what=""):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} off, e.g. {got[bad][:3]} for {want[bad][:3]} (bound {np.broadcast_to(bound, got.shape)[bad][:3]})"


# ---- embedding ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, h, v, pad", [(1, 1, 1, 0), (1, 64, 7, 0), (5, 17, 11, 3), (33, 1024, 100, 0), (300, 515, 40, 1)])
def test_embed(dtype, n, h, v, pad):
    r = np.random.default_rng(n + h)
    table, tab = matrix(r, v, h, dtype, pad=pad)
    tok = r.integers(-2, v + 2, n)
    for kind in ("int32", "int64"):
        out, full = empty(n, h, dtype, pad)
        with ops(n, h, v) as s:
            s.embed(ids(tok, kind), table, scale=1.7, out=out)
            want = O.embed(tok, tab, float(np.float32(1.7)))
        close(f64(out), want, (E + U[dtype]) * np.abs(want) + TINY[dtype])
        untouched(full, h)


GRAD_SHAPES = [(0, 8, 5, 0), (1, 1, 1, 0), (1, 64, 130, 0), (7, 33, 3, 5), (100, 513, 31, 0), (2047, 64, 1, 0),
               (2049, 72, 999, 0), (5000, 40, 50, 8), (9000, 520, 4000, 0), (70000, 16, 300, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, h, v, pad", GRAD_SHAPES)
def test_embed_grad(dtype, n, h, v, pad):
    r = np.random.default_rng(n + h)
    dout, g = matrix(r, n, h, dtype, pad=pad)
    tok = np.minimum(r.integers(-1, v + 1, n), r.integers(0, v + 3, n))
    want = O.embed_grad(tok, g, v, 0.5)
    size = O.embed_grad(tok, np.abs(g), v, 0.5)
    there = tok[(tok >= 0) & (tok < v)]
    most = max([1, *np.bincount(there, minlength=1)]) if len(there) else 1
    with ops(n, h, v) as s:
        for gtype in {dtype, "float32"}:
            out, full = empty(v, h, gtype, pad)
            s.embed_grad(ids(tok), dout, v, scale=0.5, out=out)
            close(f64(out), want, (most + 2) * E * size + U[gtype] * np.abs(want) + TINY[gtype])
            untouched(full, h)
            again = s.embed_grad(ids(tok, "int32"), dout, v, scale=0.5, dtype=dt(gtype))
            assert torch_().equal(again, out)
            # added to what is there; rows of absent tokens stay bit for bit
            start, st = matrix(r, v, h, gtype, pad=pad)
            kept = start.clone()
            s.embed_grad(ids(tok), dout, v, scale=0.5, out=start, accumulate=True)
            total = want + st
            close(f64(start), total, (most + 2) * E * size + (U[gtype] + E) * np.abs(total) + E * np.abs(st) + TINY[gtype])
            absent = np.setdiff1d(np.arange(v), there)
            assert torch_().equal(start[ids(absent)], kept[ids(absent)])


@pytest.mark.parametrize("n", [1, 700, 3000, 70000])
def test_embed_grad_of_a_huge_vocabulary(n):
    """Tokens of more than 21 bits: only some rows of the table are looked at."""
    torch = torch_()
    r = np.random.default_rng(n)
    v = (1 << 21) + 9
    dout, g = matrix(r, n, 4, "bfloat16")
    pool = np.array([0, 1, v - 1, v - 2, (1 << 21) - 1, 1 << 21, (1 << 21) + 1, 77, -1, v, 1 << 40])
    tok = pool[r.integers(0, len(pool), n)]
    with ops(n, 4, v) as s:
        out = s.embed_grad(ids(tok), dout, v, dtype=torch.float32)
    rows, place = np.unique(np.where((tok >= 0) & (tok < v), tok, -1), return_inverse=True)
    want = O.embed_grad(np.where(rows[place] < 0, -1, place), g, len(rows))
    size = O.embed_grad(np.where(rows[place] < 0, -1, place), np.abs(g), len(rows))
    some = rows >= 0
    close(f64(out[ids(rows[some])]), want[some], (n + 2) * E * size[some] + TINY["float32"])
    out[ids(rows[some])] = 0
    assert int(out.count_nonzero()) == 0


@pytest.mark.parametrize("n", [2048, 4096, 40000])
def test_embed_grad_of_one_token(n):
    """One run over all chunks, and runs that end on every edge of a chunk."""
    r = np.random.default_rng(n)
    dout, g = matrix(r, n, 24, "float32")
    for tok in (np.full(n, 3), np.arange(n) // 4 % 9, np.repeat(np.arange(n // 32 + 1), 32)[:n] % 50):
        with ops(n, 24, 50) as s:
            out = s.embed_grad(ids(tok), dout, 50)
        close(f64(out), O.embed_grad(tok, g, 50), (n + 2) * E * O.embed_grad(tok, np.abs(g), 50) + TINY["float32"])


def test_embed_gradient_is_the_adjoint():
    r = np.random.default_rng(3)
    table, tab = matrix(r, 50, 40, "float32")
    dout, g = matrix(r, 200, 40, "float32")
    tok = r.integers(-1, 51, 200)
    with ops(200, 40, 50) as s:
        y, dw = f64(s.embed(ids(tok), table, 2.0)), f64(s.embed_grad(ids(tok), dout, 50, 2.0))
    size = (np.abs(y) * np.abs(g)).sum()
    assert abs((y * g).sum() - (tab * dw).sum()) <= 210 * E * size


# ---- dropout ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, h, pad, p", [(1, 1, 0, 0.5), (1, 8, 0, 0.0), (3, 7, 2, 0.1), (65, 129, 0, 0.9),
                                          (40, 1024, 0, 0.1), (9, 4095, 1, 2.0 ** -16)])
def test_dropout(dtype, n, h, pad, p):
    r = np.random.default_rng(n * h)
    x, xv = matrix(r, n, h, dtype, pad=pad)
    res, rv = matrix(r, n, h, dtype, pad=pad)
    rows = r.integers(-2 ** 62, 2 ** 62, n)
    seed, site = 0xFEDCBA9876543210, 0xFFFFFFF1
    with ops(n, h) as s:
        for who in (rows, None):
            for residual in (None, res):
                out, full = empty(n, h, dtype, pad)
                s.dropout(x, p, seed, site, rows=None if who is None else ids(who), residual=residual, out=out)
                want = O.dropout(xv, p, seed, site, who, None if residual is None else rv)
                part = O.dropout(np.abs(xv), p, seed, site, who)
                close(f64(out), want, 2 * E * part + (E + U[dtype]) * np.abs(want) + TINY[dtype])
                untouched(full, h)
        whole = s.dropout(x, p, seed, site, rows=ids(rows))
        # the same rows in another call, in another order and place
        order = r.permutation(n)
        other = s.dropout(x[ids(order)], p, seed, site, rows=ids(rows[order]))
        assert torch_().equal(other, whole[ids(order)])
        # in place, onto the residual and onto x
        a, b = res.clone(), x.clone()
        both = s.dropout(x, p, seed, site, residual=res)
        assert torch_().equal(s.dropout(x, p, seed, site, residual=a, out=a), both)
        assert torch_().equal(s.dropout(b, p, seed, site, residual=res, out=b), both)


def test_dropped_nan_and_infinity_give_zero():
    torch = torch_()
    x = torch.full((4, 64), float("nan"), device="cuda")
    x[2:] = float("inf")
    keep, factor = O.dropout_keep(np.arange(4), 64, 0.5, 1, 2)
    with ops(4, 64) as s:
        y = f64(s.dropout(x, 0.5, 1, 2))
    assert (y[~keep] == 0).all() and np.isnan(y[:2][keep[:2]]).all() and np.isinf(y[2:][keep[2:]]).all()


def test_dropout_gradient_is_the_adjoint():
    r = np.random.default_rng(5)
    x, xv = matrix(r, 30, 100, "float32")
    g, gv = matrix(r, 30, 100, "float32")
    with ops(30, 100) as s:
        y, dx = f64(s.dropout(x, 0.3, 9, 1)), f64(s.dropout(g, 0.3, 9, 1))
    assert abs((y * gv).sum() - (xv * dx).sum()) <= 4 * E * (np.abs(y * gv)).sum()


# ---- norm ----

NORM_SHAPES = [(1, 1, 0), (1, 8, 0), (2, 127, 0), (5, 129, 7), (9, 512, 0), (6, 513, 0), (7, 1024, 0), (5, 1025, 3),
               (3, 2048, 0), (3, 2049, 0), (2, 4096, 8), (2, 4097, 0), (2, 8200, 1), (1, 16384, 0), (1030, 72, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, h, pad", NORM_SHAPES)
def test_norm(dtype, n, h, pad):
    torch = torch_()
    r = np.random.default_rng(n + h)
    x, xv = matrix(r, n, h, dtype, pad=pad)
    res, rv = matrix(r, n, h, dtype, std=3.0, pad=pad)
    w, wv = matrix(r, 1, h, dtype)
    w, wv, eps = w[0], wv[0], float(np.float32(1e-5))
    with ops(n, h) as s:
        for residual in (None, res):
            hv, rstd, y = O.norm(xv, wv, eps, None if residual is None else rv)
            # h by E; sum of squares (h + 2) E, its root half of that; rstd, two products
            rel = (h / 2 + 10) * E
            extra = E * np.abs(y) * (0 if residual is None else 1)
            for quant in ("none", "row", "block"):
                buf, full = empty(n, h, dtype, pad)
                hbuf, hfull = empty(n, h, dtype, pad)
                rs = torch.empty(n, dtype=torch.float32, device="cuda")
                if quant == "none":
                    s.norm(x, w, 1e-5, residual, out=(buf, None, None if residual is None else hbuf, rs))
                    close(f64(buf), y, (rel + U[dtype]) * np.abs(y) + extra + TINY[dtype], "y")
                    untouched(full, h)
                    if residual is not None:
                        close(f64(hbuf), hv, (E + U[dtype]) * np.abs(hv) + TINY[dtype], "h")
                        untouched(hfull, h)
                    close(f64(rs), rstd, rel * rstd, "rstd")
                    continue
                q, sc, kept, rs = s.norm(x, w, 1e-5, residual, quant)
                ws = O.scales(y, quant)
                close(f64(sc), ws, (rel + 3 * E) * ws, "scales")
                scale = O.spread(f64(sc), h, quant)
                # half a unit of 4 significant bits, of the least subnormal below
                close(f64(q) * scale, y, (2.0 ** -4 + 2 * rel) * np.abs(y) + 2.0 ** -10 * scale * (1 + 1e-6), "q")
                close(f64(rs), rstd, rel * rstd, "rstd")
                assert (kept is None) == (residual is None)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("std", [2.0 ** 62, 2.0 ** 90, 2.0 ** 125, 2.0 ** -45, 2.0 ** -70, 2.0 ** -120])
@pytest.mark.parametrize("h", [1, 300, 1000, 4096, 8201])
def test_norm_where_squares_leave_32_bits(dtype, std, h):
    r = np.random.default_rng(h)
    n = 6
    a = r.uniform(0.25, 1.5, (n, h)) * r.choice([-1.0, 1.0], (n, h)) * std
    a[3] /= std  # a row of its own range between the others
    x, xv = matrix(r, n, h, dtype, a=a)
    w, wv = matrix(r, 1, h, dtype)
    w, wv = w[0], wv[0]
    _, rstd, y = O.norm(xv, wv, 0.0)
    rel = (h / 2 + 16) * E
    subnormal = 2.0 ** -149  # of rstd where it is the inverse of a large value
    with ops(n, h) as s:
        got, _, _, rs = s.norm(x, w, 0.0)
        close(f64(rs), rstd, rel * rstd + subnormal, "rstd")
        close(f64(got), y, (rel + U[dtype]) * np.abs(y) + 2 * subnormal * np.abs(xv * wv) + TINY[dtype], "y")
        q, sc, _, _ = s.norm(x, w, 0.0, None, "row")
        off = 2 * subnormal * np.abs(xv * wv)
        ws = O.scales(y, "row")
        close(f64(sc), ws, (rel + 3 * E) * ws + off.max(1, keepdims=True) / 448, "scales")
        close(f64(q) * f64(sc), y, (2.0 ** -4 + 2 * rel) * np.abs(y) + 2.0 ** -10 * f64(sc) * (1 + 1e-6) + 2 * off, "q")


@pytest.mark.parametrize("quant", ["row", "block"])
def test_norm_8_bits_of_zeros_infinities_and_tiny_values(quant):
    torch = torch_()
    x = torch.randn((6, 300), device="cuda")
    x[0] = 0
    x[1, 140] = float("inf")
    x[2, 7] = float("nan")
    x[3] = 1e-30
    x[4] *= 1e-22
    w = torch.ones(300, device="cuda")
    with ops(6, 300) as s:
        q, sc, _, rstd = s.norm(x, w, 0.0 if quant == "row" else 1e-12, quant=quant)
        # without eps, a row of zeros has an infinite rstd: 0 * infinity
        zero, zs, _, _ = s.norm(x[:1], w, 1e-6, quant=quant)
    assert (f64(zero) == 0).all() and (f64(zs) == 2.0 ** -126).all()
    assert np.isnan(f64(rstd)[2])
    b = 0 if quant == "row" else 1
    assert np.isnan(f64(sc)[1, b]) and np.isnan(f64(sc)[2]).all()
    assert np.isnan(f64(q)[1, 140]) and np.isnan(f64(q)[2]).all()
    assert np.isfinite(f64(sc)[5]).all() and np.isfinite(f64(q)[5]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, h, pad", [(0, 8, 0), *NORM_SHAPES, (5000, 24, 0), (1100, 4096, 0)])
def test_norm_grad(dtype, n, h, pad):
    torch = torch_()
    r = np.random.default_rng(n + h)
    dy, dyv = matrix(r, n, h, dtype, pad=pad)
    hh, hv = matrix(r, n, h, dtype, std=2.0, pad=pad)
    dh, dhv = matrix(r, n, h, dtype, pad=pad)
    w, wv = matrix(r, 1, h, dtype)
    w, wv = w[0], wv[0]
    rstd = torch.from_numpy(1 / np.sqrt((hv * hv).mean(1) + 1e-5)).to("cuda", torch.float32)
    rv = f64(rstd)
    xhat = hv * rv[:, None]
    inner = np.abs(dyv * wv * xhat).mean(1, keepdims=True) if n else np.zeros((0, 1))
    # mean: products 3 E, sum h E; the rest a few E of each term
    size = rv[:, None] * (8 * np.abs(dyv * wv) + (h + 12) * np.abs(xhat) * inner)
    dsize = np.abs(dyv * xhat).sum(0)
    with ops(n, h) as s:
        for d in (None, dh):
            want, wdw = O.norm_grad(dyv, hv, wv, rv, None if d is None else dhv)
            out, full = empty(n, h, dtype, pad)
            dw = torch.full((h,), SENTINEL, device="cuda")
            s.norm_grad(dy, hh, w, rstd, dh=d, out=(out, dw))
            close(f64(out), want, E * size + (2 * E + U[dtype]) * np.abs(want) + TINY[dtype], "dx")
            close(f64(dw), wdw, (n + 4) * E * dsize + TINY["float32"], "dw")
            untouched(full, h)
            dx2, dw2 = s.norm_grad(dy, hh, w, rstd, dh=d)
            assert torch.equal(dx2, out) and torch.equal(dw2, dw)
        alias = dy.clone()
        s.norm_grad(alias, hh, w, rstd, dh=dh, out=(alias, None))
        assert torch.equal(alias, out)


def test_norm_gradient_against_differences():
    """Slope of the 64-bit forward pass along a direction, by differences with
    step d (off by about d^2), against the GPU's gradient."""
    torch = torch_()
    r = np.random.default_rng(8)
    n, h = 6, 200
    x, xv = matrix(r, n, h, "float32")
    w, wv = matrix(r, 1, h, "float32")
    dy, dyv = matrix(r, n, h, "float32")
    eps, d = float(np.float32(1e-5)), 1e-6
    v, vw = r.standard_normal((n, h)), r.standard_normal(h)
    with ops(n, h) as s:
        rstd = s.norm(x, w[0], eps)[3]
        dx, dw = s.norm_grad(dy, x, w[0], rstd)
    f = lambda a, b: (O.norm(a, b, eps)[2] * dyv).sum()  # noqa: E731
    slope = (f(xv + d * v, wv[0]) - f(xv - d * v, wv[0])) / (2 * d)
    assert abs((f64(dx) * v).sum() - slope) <= 400 * E * np.abs(f64(dx) * v).sum() + 1e-6
    slope = (f(xv, wv[0] + d * vw) - f(xv, wv[0] - d * vw)) / (2 * d)
    assert abs((f64(dw) * vw).sum() - slope) <= 400 * E * np.abs(f64(dw) * vw).sum() + 1e-6
    assert torch.isfinite(dx).all()


# ---- log probabilities ----

def lp_bounds(x, lse, entropy):
    """Bounds on lse and entropy.  A lane adds at most 16 terms for each 4096
    columns (2048 of a split row's least part), then 20 joins; an exponential of
    the difference d to the maximum is off by 4 + 2 |d| roundings."""
    v = x.shape[1]
    chain = 16 * (v // 4096 + 1) + 3 * 20
    m = np.where(np.isfinite(lse), np.max(x, 1), 0)
    d = np.where(np.isfinite(x), x - m[:, None], 0)
    p = np.where(np.isfinite(x) & np.isfinite(lse)[:, None], np.exp(np.minimum(x, 1e30) - np.where(np.isfinite(lse), lse, 0)[:, None]), 0)
    d1, d2 = (p * np.abs(d)).sum(1), (p * d * d).sum(1)
    b = (chain + 8 + 2 * d1) * E
    lse_b = b + 3 * E * np.abs(np.where(np.isfinite(lse), lse, 0))
    ent_b = b + (chain + 8) * E * d1 + 2 * E * d2 + b * d1 + 4 * E * np.abs(entropy)
    return lse_b, ent_b


def same(got, want, bound, what):
    """Infinities in the same places, the rest within the bound."""
    inf = np.isinf(want)
    assert (got[inf] == want[inf]).all(), what
    close(np.where(inf, 0, got), np.where(inf, 0, want), np.broadcast_to(bound, want.shape), what)


def logits_case(r, n, v, kind):
    a = r.standard_normal((n, v)) * 3
    if kind == "ties":
        a = np.round(a)
    elif kind == "masked":
        a[:, r.random(v) < 0.5] = -np.inf
        a[n // 2] = -np.inf
        if v > 3:
            a[0] = -np.inf
            a[0, v - 2] = 1.5
    elif kind == "equal":
        a[:] = -2.5
    elif kind == "rising":
        a = np.sort(a, 1)
    elif kind == "large":
        a = a * 20
    return a


LP_SHAPES = [(1, 1, 1), (1, 2, 2), (2, 63, 5), (3, 1000, 20), (5, 4097, 64), (1, 50021, 8), (2, 131072, 4), (600, 300, 3),
             (513, 4100, 0), (3, 65535, 9), (1, 65537, 30)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "equal", "rising", "large"])
@pytest.mark.parametrize("n, v, top", LP_SHAPES)
def test_logprob(dtype, kind, n, v, top):
    r = np.random.default_rng(n + v)
    pad = 0 if v % 2 else 5
    x, xv = matrix(r, n, v, dtype, pad=pad, a=logits_case(r, n, v, kind))
    tok = r.integers(-1, v + 1, n)
    with ops(n, 1, v) as s:
        got = s.logprob(x, ids(tok), top=top)
        narrow = s.logprob(x, ids(tok, "int32"), top=top)
        bare = s.logprob(x)
    logp, entropy, lse, top_logp, top_ids = O.logprob(xv, tok, top)
    lse_b, ent_b = lp_bounds(xv, lse, entropy)
    same(f64(got[2]), lse, lse_b, "lse")
    same(f64(got[1]), entropy, ent_b, "entropy")
    finite = lambda a: np.where(np.isfinite(a), np.abs(a), 0)  # noqa: E731
    same(f64(got[0]), logp, lse_b + 2 * E * finite(logp), "logp")
    if top:
        assert (got[4].cpu().numpy() == top_ids).all()
        same(f64(got[3]), top_logp, lse_b[:, None] + 2 * E * finite(top_logp), "top")
    else:
        assert got[3] is None and got[4] is None
    for a, b in zip(got, narrow):
        assert a is None or torch_().equal(a, b)
    assert bare[0] is None and torch_().equal(bare[2], got[2])


@pytest.mark.parametrize("v, top", [(20000, 3), (20001, 8), (131072, 24), (131072, 25), (300, 64)])
def test_logprob_alternatives_in_few_columns(v, top):
    """Largest entries 4096 columns apart, side by side, few, and tied over the row."""
    r = np.random.default_rng(v)
    a = np.full((520, v), -1, np.float32)  # whole rows by one workgroup
    a[:40] = r.standard_normal((40, v))
    a[0, 37::4096] = 50 + r.standard_normal(len(a[0, 37::4096]))
    a[1, 100:100 + top] = np.arange(top) + 20
    a[2] = -np.inf
    a[2, 5] = 1
    a[3] = np.where(np.arange(v) % 4096 == 17, 9, -np.inf)
    a[4] = 3
    a[5, ::16] = 30
    a[6, v - 1] = a[6, 0] = 40
    a[7, 37::4096] = 50
    for rows in (a[:8], a):
        x, xv = matrix(r, *rows.shape, "bfloat16", a=rows)
        with ops(len(rows), 1, v) as s:
            _, _, lse, top_logp, top_ids = s.logprob(x, top=top)
        want = O.logprob(xv[:41], None, top)
        assert (top_ids.cpu().numpy()[:41] == want[4]).all()
        same(f64(top_logp)[:41], want[3], 1e-4, "top")
        assert (top_ids[40:].cpu().numpy() == np.arange(top)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_logprob_of_the_types_lowest_value(dtype):
    """Masks of the lowest finite value: no probability beside others, uniform alone."""
    torch = torch_()
    x = torch.randn((3, 5000), device="cuda").to(dt(dtype))
    low = torch.finfo(dt(dtype)).min
    x[0, 100:] = low
    x[1] = low
    with ops(3, 1, 5000) as s:
        logp, entropy, lse, tl, ti = s.logprob(x, ids([7, 4999, -5]), top=3)
        plain = s.logprob(x[:1, :100].contiguous(), ids([7]), top=3)
    assert abs(f64(entropy)[1] - np.log(5000)) < 100 * E
    assert abs(f64(logp)[1] + np.log(5000)) <= 2 * abs(float(low)) * E + 1e-4
    assert ti[1].tolist() == [0, 1, 2] and ti[0].tolist() == plain[4][0].tolist()
    np.testing.assert_allclose(f64(lse)[0], f64(plain[2])[0], rtol=100 * E)
    np.testing.assert_allclose(f64(entropy)[0], f64(plain[1])[0], rtol=200 * E)
    assert f64(logp)[2] == 0


@pytest.mark.parametrize("v", [40, 9000, 90001])
def test_logprob_with_nan_and_infinity(v):
    torch = torch_()
    x = torch.randn((4, v), device="cuda")
    x[0, 3] = float("nan")
    x[1, 5] = float("inf")
    x[2] = float("nan")
    x[3, 7] = -0.0
    x[3, 9] = 0.0
    x[3, 10:] = -1.0
    x[3, :7] = x[3, 8] = -1.0
    with ops(4, 1, v) as s:
        logp, entropy, lse, tl, ti = (t.cpu() for t in s.logprob(x, ids([0, 0, 0, 0]), top=4))
    for t in (logp, entropy, lse):
        assert t[:3].isnan().all() and t[3].isfinite()
    assert tl[:3].isnan().all() and 3 not in ti[0].tolist()
    assert ti[1, 0] == 5 and ti[2].tolist() == [-1] * 4
    assert ti[3].tolist() == [7, 9, 0, 1]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["plain", "masked", "large"])
@pytest.mark.parametrize("n, v", [(1, 1), (2, 63), (3, 1001), (1, 50021), (600, 300), (2100, 40)])
def test_logprob_grad(dtype, kind, n, v):
    torch = torch_()
    r = np.random.default_rng(n + v)
    pad = 3 if v % 2 else 0
    x, xv = matrix(r, n, v, dtype, pad=pad, a=logits_case(r, n, v, kind))
    tok = r.integers(-1, v + 1, n)
    _, entropy, lse, _, _ = O.logprob(xv, tok)
    dev = lambda a: torch.from_numpy(a).to("cuda", torch.float32)  # noqa: E731
    lse_t, ent_t = dev(lse), dev(entropy)
    gl, ge = dev(r.standard_normal(n)), dev(r.standard_normal(n))
    lv, ev, glv, gev = f64(lse_t), f64(ent_t), f64(gl), f64(ge)
    with ops(n, 1, v) as s:
        for a, b in ((gl, None), (None, ge), (gl, ge)):
            out, full = empty(n, v, dtype, pad)
            s.logprob_grad(x, ids(tok), lse_t, ent_t, a, b, out=out)
            want = O.logprob_grad(xv, tok, lv, ev, None if a is None else glv, None if b is None else gev)
            ok = np.isfinite(lv)[:, None] & np.isfinite(xv)
            d = np.where(ok, xv - np.where(np.isfinite(lv), lv, 0)[:, None], 0)
            p = np.where(ok, np.exp(d), 0)
            c = np.abs(glv)[:, None] * (a is not None) + (np.abs(gev)[:, None] * (np.abs(d) + np.abs(ev)[:, None])) * (b is not None)
            bound = (10 + 4 * np.abs(d)) * E * p * c + (U[dtype] + 2 * E) * np.abs(want) + TINY[dtype] + 2.0 ** -126 * c
            close(f64(out), want, bound, "dlogits")
            untouched(full, v)
        alias = x.clone()
        s.logprob_grad(alias, ids(tok, "int32"), lse_t, ent_t, gl, ge, out=alias)
        assert torch.equal(alias, out)


def test_logprob_gradient_against_differences():
    r = np.random.default_rng(12)
    torch = torch_()
    n, v, d = 5, 3001, 1e-5
    x, xv = matrix(r, n, v, "float32", std=2.0)
    tok = np.array([0, 3000, 17, -1, 2999])
    gl, ge, dirn = r.standard_normal(n), r.standard_normal(n), r.standard_normal((n, v))
    dev = lambda a: torch.from_numpy(a).to("cuda", torch.float32)  # noqa: E731
    with ops(n, 1, v) as s:
        _, entropy, lse, _, _ = s.logprob(x, ids(tok))
        g = f64(s.logprob_grad(x, ids(tok), lse, entropy, dev(gl), dev(ge)))
    gl, ge = np.float64(np.float32(gl)), np.float64(np.float32(ge))

    def loss(z):
        lp, e, *_ = O.logprob(z, tok)
        return (lp * gl).sum() + (e * ge).sum()
    slope = (loss(xv + d * dirn) - loss(xv - d * dirn)) / (2 * d)
    # each entry by (10 + 4 * 20) E of its terms, which are at most (2 + 30) p
    assert abs((g * dirn).sum() - slope) <= 100 * E * (np.abs(g * dirn).sum() + 32 * n) + 1e-6


# ---- calls larger than the caches ----

def parts_of(n, pieces=5):
    step = -(-n // pieces)
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


@pytest.mark.parametrize("dtype, h", [("bfloat16", 4096), ("float32", 2056), ("float16", 1000)])
def test_large_calls_match_small_ones(dtype, h):
    """A row's result does not depend on the call's size: calls of more than 256
    MB against the same rows in pieces, bit for bit."""
    torch = torch_()
    size = 4 if dtype == "float32" else 2
    n = (300 << 20) // (2 * size * h)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    new = lambda: torch.randn((n, h), device="cuda", generator=gen).to(dt(dtype))  # noqa: E731
    x, res, w = new(), new(), torch.randn(h, device="cuda", generator=gen).to(dt(dtype))
    tok = torch.randint(-1, 4000, (n,), device="cuda", generator=gen)
    ident = torch.arange(n, device="cuda") * 7919
    with ops(n, h, 4000) as s:
        table = x[:4000]
        calls = [lambda r: (s.embed(tok[r], table, 1.5),),
                 lambda r: (s.dropout(x[r], 0.3, 11, 2, rows=ident[r]),),
                 lambda r: (s.dropout(x[r], 0.3, 11, 2, rows=ident[r], residual=res[r]),)]
        calls += [lambda r, q=q: [t for t in s.norm(x[r], w, 1e-5, res[r], q) if t is not None] for q in ("none", "row", "block")]
        rstd = s.norm(x, w)[3]
        calls.append(lambda r: (s.norm_grad(x[r], res[r], w, rstd[r], dh=x[r])[0],))
        for call in calls:
            whole = call(slice(0, n))
            pieces = [call(r) for r in parts_of(n)]
            for i, t in enumerate(whole):
                assert torch.equal(t.view(torch.uint8), torch.cat([p[i] for p in pieces]).view(torch.uint8))


def test_large_embedding_gradient():
    torch = torch_()
    n, h, v = 9000, 4096, 32000
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    dout = torch.randn((n, h), device="cuda", generator=gen).to(torch.bfloat16)
    tok = torch.randint(-1, v, (n,), device="cuda", generator=gen) % 9001 - 1
    there = tok >= 0
    want = torch.zeros((v, h), device="cuda", dtype=torch.float64).index_add_(0, tok[there], dout[there].double())
    size = torch.zeros((v, h), device="cuda", dtype=torch.float64).index_add_(0, tok[there], dout[there].double().abs())
    with ops(n, h, v) as s:
        got = s.embed_grad(tok, dout, v, dtype=torch.float32)
        again = s.embed_grad(tok, dout, v, dtype=torch.float32)
    most = int(torch.bincount(tok[there]).max())
    assert bool(((got.double() - want).abs() <= (most + 2) * E * size).all())
    assert torch.equal(got, again)


# ---- refusals, streams, graphs ----

def test_refusals():
    torch = torch_()
    from paper_2509_21221_amd.mcf import GwtfError
    x = torch.zeros((4, 16), device="cuda")
    w = torch.ones(16, device="cuda")
    t = ids([0, 1, 2, 3])
    with ops(4, 16, 8) as s:
        table = torch.zeros((8, 16), device="cuda")
        bad = [
            (TypeError, lambda: s.embed(t, [[0.0]])),
            (ValueError, lambda: s.dropout(x[0], 0.1, 0, 0)),
            (ValueError, lambda: s.norm(x[None], w)),
            (ValueError, lambda: s.embed(t, table.double())),
            (ValueError, lambda: s.embed(t.float(), table)),
            (ValueError, lambda: s.embed(t[::2], table)),
            (ValueError, lambda: s.embed(t, table.t())),
            (ValueError, lambda: s.embed(t, table.cpu())),
            (ValueError, lambda: s.embed(t, table, out=x[:2])),
            (GwtfError, lambda: s.embed(ids([0] * 5), table)),
            (GwtfError, lambda: s.embed(t, torch.zeros((9, 16), device="cuda"))),
            (GwtfError, lambda: s.embed(t, torch.zeros((8, 17), device="cuda"))),
            (ValueError, lambda: s.embed_grad(t, x, 8, accumulate=True)),
            (ValueError, lambda: s.embed_grad(t, x[:3], 8)),
            (GwtfError, lambda: s.embed_grad(t, x, 8, dtype=torch.float16)),
            (GwtfError, lambda: s.embed_grad(t, x[:1].expand(4, 16), 8)),
            (GwtfError, lambda: s.dropout(x, 1.0, 0, 0)),
            (GwtfError, lambda: s.dropout(x, 1 - 2.0 ** -20, 0, 0)),
            (GwtfError, lambda: s.dropout(x, -0.1, 0, 0)),
            (GwtfError, lambda: s.dropout(x, float("nan"), 0, 0)),
            (ValueError, lambda: s.dropout(x, 0.1, -1, 0)),
            (ValueError, lambda: s.dropout(x, 0.1, 0, 1 << 32)),
            (ValueError, lambda: s.dropout(x, 0.1, 0, 0, rows=t.int())),
            (ValueError, lambda: s.dropout(x, 0.1, 0, 0, residual=x.half())),
            (KeyError, lambda: s.norm(x, w, quant="int4")),
            (ValueError, lambda: s.norm(x, w.half())),
            (ValueError, lambda: s.norm(x, w[:8])),
            (GwtfError, lambda: s.norm(x, w, eps=-1.0)),
            (GwtfError, lambda: s.norm(x, w, eps=float("nan"))),
            (ValueError, lambda: s.norm_grad(x, x, w, w)),
            (GwtfError, lambda: s.logprob(x[:, :8].contiguous(), t, top=9)),
            (ValueError, lambda: s.logprob(x[:, :8].contiguous(), t, top=-1)),
            (ValueError, lambda: s.logprob(x[:, :8].contiguous(), t, top=65)),
            (GwtfError, lambda: s.logprob(x, t)),
            (ValueError, lambda: s.logprob(x[:, :8], t[:2])),
            (ValueError, lambda: s.logprob_grad(x[:, :8], None, w[:4].contiguous(), dlogp=w[:4].contiguous())),
            (ValueError, lambda: s.logprob_grad(x[:, :8], t, w[:4].contiguous(), dentropy=w[:4].contiguous())),
        ]
        for kind, call in bad:
            with pytest.raises(kind):
                call()
        s.embed(t, table)
    with pytest.raises(RuntimeError, match="closed"):
        s.embed(t, table)
    with ops(1, 20000) as s:
        with pytest.raises(GwtfError, match="MAX_HIDDEN"):
            s.norm(torch.zeros((1, 16385), device="cuda"), torch.zeros(16385, device="cuda"))


def test_no_tokens():
    torch = torch_()
    none = torch.zeros((0, 16), device="cuda")
    t = torch.zeros(0, dtype=torch.int64, device="cuda")
    with ops(4, 16, 8) as s:
        assert s.embed(t, torch.zeros((8, 16), device="cuda")).shape == (0, 16)
        assert (s.embed_grad(t, none, 8) == 0).all()
        assert s.dropout(none, 0.1, 0, 0).shape == (0, 16)
        assert s.norm(none, torch.ones(16, device="cuda"), quant="block")[0].shape == (0, 16)
        assert (s.norm_grad(none, none, torch.ones(16, device="cuda"), torch.zeros(0, device="cuda"))[1] == 0).all()
        assert s.logprob(none[:, :8], t, top=2)[4].shape == (0, 2)


def test_tensors_of_another_stream():
    """Inputs written, and results read, on streams other than the handle's."""
    torch = torch_()
    home, away = torch.cuda.Stream(), torch.cuda.Stream()
    v = 20000
    with ops(64, 1, v, stream=home) as s:
        for i in range(4):
            with torch.cuda.stream(away):
                big = torch.randn((4000, 4000), device="cuda")
                big = big @ big * 1e-3 + big  # keeps the stream busy before the input is there
                x = big.flatten()[:64 * v].reshape(64, v).clone()
                lse = s.logprob(x)[2]
                copy = lse * 1.0
                want = torch.logsumexp(x.double(), 1)
                del lse
                torch.randn(64, device="cuda")
            away.synchronize()
            assert (copy.double() - want).abs().max() < 1e-4


def test_graph_replays():
    """All calls in one captured graph, replayed with new inputs between the
    program's own work, against the same calls made eagerly."""
    torch = torch_()
    n, h, v = 48, 136, 9000
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream), ops(n, h, v, stream=stream) as s:
        tok = torch.zeros(n, dtype=torch.int64, device="cuda")
        table, w = torch.randn((v, h), device="cuda"), torch.rand(h, device="cuda")
        logits = torch.zeros((n, v), device="cuda")

        def step():
            e = s.embed(tok, table, 2.0)
            d = s.dropout(e, 0.2, 5, 1, residual=e)
            q, sc, hh, rstd = s.norm(d, w, residual=e, quant="block")
            dx, dw = s.norm_grad(d, hh, w, rstd, dh=e)
            g = s.embed_grad(tok, dx, v)
            logp, ent, lse, tl, ti = s.logprob(logits, tok, top=5)
            dl = s.logprob_grad(logits, tok, lse, ent, logp, ent)
            return [d, q, sc, hh, rstd, dx, dw, g, logp, ent, lse, tl, ti, dl]
        step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = step()
        for i in range(4):
            tok.copy_(torch.randint(-1, v, (n,), device="cuda"))
            logits.copy_(torch.randn((n, v), device="cuda"))
            graph.replay()
            stream.synchronize()
            got = [t.clone() for t in held]
            for a, b in zip(got, step()):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
            stream.synchronize()


# ---- more rows than one launch has threads for ----


@pytest.mark.parametrize("h, n", [(1, (1 << 26) + 5), (9, (1 << 25) + 3)])
def test_norm_of_many_rows(h, n):
    t = torch_()
    x = t.full((n, h), 3.0, dtype=t.float16, device="cuda")
    x[-1] = -2.0
    w = t.ones(h, dtype=t.float16, device="cuda")
    y = t.zeros_like(x)
    rstd = t.zeros(n, dtype=t.float32, device="cuda")
    with ops(n, h) as s:
        s.norm(x, w, eps=0.0, out=(y, None, None, rstd))
        assert bool((y[:-1] == 1).all()) and bool((y[-1] == -1).all())
        assert bool(((rstd[:-1] - 1 / 3).abs() < 1e-6).all()) and abs(rstd[-1].item() - 0.5) < 1e-6


def test_logprob_of_many_rows():
    t = torch_()
    n = (1 << 24) + 3  # one workgroup a row
    x = t.zeros((n, 2), dtype=t.bfloat16, device="cuda")
    x[-1, 1] = 4.0
    target = t.ones(n, dtype=t.int32, device="cuda")
    with ops(n, 1, 2) as s:
        logp, entropy, lse, top_logp, top_ids = s.logprob(x, target, top=1)
        d = s.logprob_grad(x, target, lse, dlogp=t.ones(n, device="cuda"))
    ln2, last = np.log(2.0), np.log1p(np.exp(-4.0))
    for got, want in ((logp, -ln2), (entropy, ln2), (lse, ln2), (top_logp[:, 0], -ln2)):
        assert bool(((got[:-1] - want).abs() < 1e-6).all())
    assert bool((top_ids[:-1] == 0).all()) and top_ids[-1].item() == 1
    assert abs(logp[-1].item() + last) < 1e-6
    assert bool((d[:-1, 0] == -0.5).all()) and bool((d[:-1, 1] == 0.5).all())
    assert abs(d[-1, 1].item() - (1 - np.exp(-last))) < 1e-3


@pytest.mark.parametrize("n", [0, 40000])
def test_embed_grad_of_the_largest_tables(n):
    t = torch_()
    v = (1 << 30) + 5  # 16 rows a wave: more than 2^32 threads
    tokens = t.full((n,), v - 2, dtype=t.int64, device="cuda")
    g = t.full((v, 1), 7.0, dtype=t.float16, device="cuda")
    with ops(max(n, 1), 1, v) as s:
        s.embed_grad(tokens, t.ones((n, 1), dtype=t.float16, device="cuda"), v, out=g)
    assert g[v - 2, 0].item() == n and g[v - 1, 0].item() == 0
    g[v - 2] = 0
    assert int(g.count_nonzero()) == 0
