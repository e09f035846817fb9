"""How far top_p may be from what a draw keeps: by 1e-11 of the sum, or V 2^-61 of it where that is more."""
import numpy as np
import pytest

from oracle import learn as O
from tests.gpu_util import have_gpu
from tests.test_gpu_learn import HALF, dev, logits, ops, uniform  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch

    from tests.test_gpu_learn import DT


def slack(v):
    return max(1e-11, v * 2.0 ** -61)


def check_kept(x, u, got, temperature=1.0, top_k=0, top_p=1.0):
    """What stays is what a top_p within `slack` of the given one leaves, and the token and its logp are those of what
    stays."""
    x = x.double().cpu().numpy()
    ids, logp, kept = (t.cpu().numpy() for t in got)
    u = u.double().cpu().numpy()
    for i, row in enumerate(x):
        live = np.flatnonzero(row > -np.inf)
        order = live[np.argsort(-row[live], kind="stable")]
        with np.errstate(over="ignore"):
            w = np.exp(((row[order] - row[order[0]]) / np.float64(temperature)).astype(np.longdouble))
        first = min(top_k, len(order)) if top_k > 0 else len(order)
        c = np.cumsum(w[:first])
        n, p, s = int(kept[i]), np.longdouble(top_p), slack(len(row))
        assert 1 <= n <= first, (i, n, first)
        assert c[n - 1] >= (p - s) * c[-1] or n == first, (i, n, float(c[n - 1] / c[-1] - p))
        assert n == 1 or c[n - 2] < (p + s) * c[-1], (i, n, float(c[n - 2] / c[-1] - p))
        at = np.argsort(order[:n])
        stays, w = order[:n][at], w[:n][at]
        c = np.cumsum(w)
        j = int(np.flatnonzero(stays == ids[i])[0])  # the token drawn is one that stays
        # and u lies between its borders, but for the 1e-13 of 64-bit sums
        assert c[j] > (u[i] - 1e-12) * c[-1] and (j == 0 or c[j - 1] <= (u[i] + 1e-12) * c[-1]), (i, j)
        want = float(np.log(w[j] / c[-1]))
        assert abs(logp[i] - want) <= HALF["f32"] * abs(want) + 1e-12, (i, logp[i], want)


@pytest.mark.parametrize("seed", [0, 1])
@pytest.mark.parametrize("top_p", [0.9999, 0.999999])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_far_above_crowded_bins(ops, dtype, top_p, seed):  # noqa: F811
    """One token 20 above 131,071 of deviation 1, many of them equal in 16 bits: the sum ends in the bulk of the tail."""
    x = logits(24, 131072, dtype, 100 + seed, std=1.0)
    x[torch.arange(24), torch.arange(24) * 3001] = 20.0
    u = uniform(24, seed)
    got = ops.sample(x, u, top_p=top_p)
    check_kept(x, u, got, top_p=top_p)
    clear = 0
    for i in range(24):
        want = O.sample_row(x[i].double().cpu().numpy(), u[i].item(), top_p=top_p)
        if want[3] > 1e-11:
            assert (got[0][i].item(), got[2][i].item()) == (want[0], want[2]), (i, want)
            clear += 1
    assert clear > 12


# quanta of 2^-45 (131,072 columns) and 2^-41 (1.2 million) are what a sum of whole numbers in 62 bits has
@pytest.mark.parametrize("share", [0.25, 0.49, 0.51, 0.99, 1.49])
@pytest.mark.parametrize("dtype,v,top_p,bits", [("f32", 131072, 1 - 1e-9, 45), ("f32", 131072, 1 - 1e-10, 47), ("f32", 131072, 1 - 1e-8, 42),
                                                ("bf16", 131072, 1 - 1e-9, 45), ("f32", 40000, 1 - 1e-10, 46), ("f32", 1_200_007, 1 - 2.0 ** -24, 41),
                                                ("bf16", 1_200_007, 0.9999, 33)])
def test_equal_tails(ops, dtype, v, top_p, bits, share):  # noqa: F811
    """One entry of weight 1, all others of a weight near a whole or half quantum: their errors all add up."""
    x = torch.full((2, v), float(np.log(share) - bits * np.log(2.0)), device="cuda").to(DT[dtype])
    x[0, v // 3], x[1, 0] = 0.0, 0.0
    x[1, 5:9] = 0.0
    u = uniform(2, 7)
    check_kept(x, u, ops.sample(x, u, top_p=top_p), top_p=top_p)
    row = float(np.float32(top_p))
    if row < 1:
        check_kept(x, u, ops.sample(x, u, top_p=torch.full((2,), row, device="cuda")), top_p=row)
    check_kept(x, u, ops.sample(x, u, top_p=top_p, top_k=v - 1000), top_p=top_p, top_k=v - 1000)


def test_an_equal_tail_of_134_million(ops):  # noqa: F811
    v, p = 1 << 27, 0.999
    x = torch.full((1, v), float(-35.4 * np.log(2.0)), device="cuda")
    x[0, 12345] = 0.0
    w = np.exp(np.longdouble(x[0, 0].item()))
    _, _, kept = ops.sample(x, uniform(1, 1), top_p=p)
    total, n = 1 + (v - 1) * w, kept.item()
    assert 1 + (n - 1) * w >= (p - slack(v)) * total and 1 + (n - 2) * w < (p + slack(v)) * total, n


def test_tails_of_several_weights(ops):  # noqa: F811
    """Steps of equal entries, so that bins hold more than can be ranked, at all distances from the largest."""
    rng = np.random.default_rng(5)
    for dtype, v in (("f32", 50001), ("bf16", 131072), ("f32", 70001), ("f16", 3000)):
        levels = -np.sort(rng.uniform(0, 60, 24))
        pick = rng.choice(24, (4, v), p=np.exp(-0.3 * np.arange(24)) / np.exp(-0.3 * np.arange(24)).sum())
        x = dev(levels[pick].astype(np.float32), DT[dtype])
        u = uniform(4, v)
        for kw in (dict(top_p=0.5), dict(top_p=0.99), dict(top_p=1 - 1e-6), dict(top_p=1 - 1e-9, temperature=0.7), dict(top_p=0.9, top_k=v // 2),
                   dict(top_p=1 - 1e-7, top_k=1500), dict(top_p=0.9999, temperature=30.0)):
            check_kept(x, u, ops.sample(x, u, **kw), **kw)


@pytest.mark.parametrize("t", [1e-30, 1e-36, 1e-37, 1e-38, 1e-40, 1e-44, 1e-60, 1e-300, 1e20, 1e38, 1e300])
def test_temperatures_at_the_ends_of_32_bits(ops, t):  # noqa: F811
    """Logits as far apart as the temperature, where 32 bits hold such: weights of all sizes at quotients beyond 32 bits."""
    rng = np.random.default_rng(8)
    v = 4000
    near = min(t, 1e36)
    x = np.zeros((4, v))
    x[0] = -rng.exponential(5, v) * near
    x[1] = -rng.integers(0, 12, v) * near     # many equal
    x[2] = -rng.integers(0, 40, v) * 1e-45    # steps of the smallest number
    x[3] = np.where(rng.random(v) < 0.5, 0.0, -3e38)
    x[:, 17] = 0.0
    x = dev(x.astype(np.float32))
    u = uniform(4, 9)
    for kw in (dict(top_p=0.9), dict(top_p=1 - 1e-9), dict(top_p=0.7, top_k=1000), dict(top_p=0.3, top_k=3999)):
        check_kept(x, u, ops.sample(x, u, temperature=t, **kw), temperature=t, **kw)


def test_all_equal(ops):  # noqa: F811
    for dtype, v in (("bf16", 131072), ("f32", 65537), ("f32", 100_000), ("f16", 1000)):
        x = torch.full((2, v), -7.25, device="cuda", dtype=DT[dtype])
        u = uniform(2, 4)
        for p in (0.25, 0.5, 1 - 2.0 ** -20):
            got = ops.sample(x, u, top_p=p)
            check_kept(x, u, got, top_p=p)
            assert (got[2] == int(np.ceil(v * p))).all()  # v p is far from a whole number, or is one


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t", [1e30, 1e36, 2e37, 1e38, 1e39, 1e45, 1e300])
def test_distances_beyond_32_bits(ops, dtype, t):  # noqa: F811
    """Entries whose distance from the largest 32 bits do not hold, at temperatures that weigh them."""
    rng = np.random.default_rng(11)
    v = 5000
    x = np.stack((np.where(rng.random(v) < 0.3, 3e38, -3e38), rng.uniform(-3.3e38, 3.3e38, v), np.where(np.arange(v) == 9, 3.3e38, -3.3e38),
                  np.where(rng.random(v) < 0.5, 1.0, -3.3e38)))
    x = dev(x.astype(np.float32), DT[dtype])
    x[1, 100:200] = float("-inf")
    u = uniform(4, 12)
    for kw in (dict(top_p=0.5), dict(top_p=0.9), dict(top_p=1 - 1e-9), dict(top_p=0.7, top_k=1000), dict(top_p=0.7, top_k=4500)):
        check_kept(x, u, ops.sample(x, u, temperature=t, **kw), temperature=t, **kw)
