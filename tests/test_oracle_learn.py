"""Pins of oracle/learn.py: enumerations, closed forms and frequencies."""
import itertools
import math

import numpy as np
import pytest

from oracle import learn as O


def shares(x, **kw):
    """Probability of each token, from draws at a fine grid of u."""
    got = np.zeros(len(x))
    grid = (np.arange(4000) + 0.5) / 4000
    for u in grid:
        got[O.sample_row(x, u, **kw)[0]] += 1 / len(grid)
    return got


def test_shares_follow_the_weights():
    x = np.array([0.3, -1.0, 2.0, 0.3])
    p = np.exp(x / 0.7) / np.exp(x / 0.7).sum()
    assert np.abs(shares(x, temperature=0.7) - p).max() < 1e-3
    token, logp, kept, _ = O.sample_row(x, 0.5, temperature=0.7)
    assert kept == 4 and abs(logp - math.log(p[token])) < 1e-12


@pytest.mark.parametrize("k,p,q", itertools.product((0, 1, 2, 5), (1.0, 0.5, 0.75, 0.0), (0.0, 0.3, 1.0)))
def test_filters_by_enumeration(k, p, q):
    x = np.array([1.0, 3.0, 3.0, -np.inf, 2.0, 0.0])
    w = np.exp(x - 3.0)
    order = [1, 2, 4, 0, 5]
    cand = order[:k] if k else order
    stays = []
    for i, j in enumerate(cand):
        before = sum(w[c] for c in cand[:i])
        if i and ((p < 1 and before >= p * sum(w[c] for c in cand)) or w[j] < q):
            break
        stays.append(j)
    token, logp, kept, _ = O.sample_row(x, 0.0, top_k=k, top_p=p, min_p=q)
    assert kept == len(stays) and token == min(stays)
    assert abs(logp - math.log(w[token] / sum(w[c] for c in stays))) < 1e-12
    assert O.sample_row(x, 1.0, top_k=k, top_p=p, min_p=q)[0] == max(stays)


def test_special_rows():
    inf = np.inf
    assert O.sample_row([-inf, -inf], 0.3)[:3] == (-1, -inf, 0)
    assert O.sample_row([0.0, np.nan], 0.3)[0] == -1 and O.sample_row([0.0, inf], 0.3)[0] == -1
    assert O.sample_row([1.0, 5.0, 5.0], 0.9, temperature=0.0)[:3] == (1, 0.0, 1)
    assert O.sample_row([1.0, 5.0], 0.9, temperature=-1.0)[0] == -1


def test_adamw_against_a_scalar_loop():
    rng = np.random.default_rng(0)
    p, m, v = 0.7, 0.0, 0.0
    q = np.array([0.7]), np.zeros(1), np.zeros(1)
    for t in range(1, 6):
        g = rng.normal()
        m, v = 0.9 * m + 0.1 * g, 0.99 * v + 0.01 * g * g
        p -= 1e-2 * (m / (1 - 0.9 ** t) / (math.sqrt(v / (1 - 0.99 ** t)) + 1e-8) + 0.1 * p)
        q = O.adamw(q[0], np.array([g]), q[1], q[2], 1e-2, t, (0.9, 0.99), 1e-8, 0.1)
    assert abs(p - q[0][0]) < 1e-14 and abs(m - q[1][0]) < 1e-14 and abs(v - q[2][0]) < 1e-14


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_narrow_keeps_8_bit_values_and_the_mean(kind):
    import torch

    dt = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[kind]
    codes = torch.arange(0, 0x7F if kind == "e4m3" else 0x7C, dtype=torch.uint8).view(dt).double().numpy()
    assert codes.max() == O._MOST[kind]
    x = np.resize(codes, 2 * 128)
    x[0] = x[128] = codes.max()
    for r in (0.0, 65535.0):  # values that 8 bits hold stay, whatever is drawn
        q, s = O.narrow(x * 8.0, np.full(256, r), kind)
        assert (s == 8.0).all() and (q == x).all()
    rng = np.random.default_rng(1)
    x = np.abs(rng.normal(size=128)) * np.exp(rng.normal(size=128) * 3)
    mean = np.mean([np.multiply(*map(np.float64, (lambda q, s: (q, s[0]))(*O.narrow(x, rng.integers(0, 65536, 128), kind)))) for _ in range(4000)], 0)
    # 4,000 roundings of at most one step: half a step / sqrt(4000), six times over
    step = np.maximum(x * 2.0 ** -O._MANTISSA[kind], O._LEAST[kind] * O.narrow(x, np.zeros(128), kind)[1][0])
    assert (np.abs(mean - x) <= 6 * 0.5 * step / math.sqrt(4000)).all()


def test_narrow_special_values():
    x = np.zeros(130)
    q, s = O.narrow(x, np.full(130, 65535.0), "e5m2")
    assert (q == 0).all() and len(s) == 2 and (s == 2.0 ** -126).all()
    x[0], x[1] = 1.0, 1e-30
    q, s = O.narrow(x, np.zeros(130), "e5m2")
    assert q[1] == 2.0 ** -16 and q[2] == 0 and q[0] * s[0] == 1.0
    assert O.narrow(x, np.zeros(130), "e4m3")[0][1] == 0
    x[129] = np.inf
    q, s = O.narrow(x, np.zeros(130), "e4m3")
    assert np.isnan(s[1]) and s[0] > 0


def test_grad_norm():
    norm, factor = O.grad_norm([np.array([3.0]), np.array([0.0, 4.0])], max_norm=1.0, scale=0.5)
    assert norm == 2.5 and factor == 0.5 / 2.5
    assert O.grad_norm([np.zeros(3)], 0.0)[1] == 1.0
    assert np.isnan(O.grad_norm([np.array([np.inf])], 1.0)[1])
