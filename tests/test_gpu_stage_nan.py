"""Alternatives of rows with NaN among masked entries: a NaN is none, and the
others go by value, then by index."""
import numpy as np
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_stage import f64, ids, matrix, ops

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]


def alternatives(x, top):
    out = np.full((len(x), top), -1)
    for i, row in enumerate(x):
        there = np.flatnonzero(~np.isnan(row))
        there = there[np.argsort(-row[there], kind="stable")][:top]
        out[i, :len(there)] = there
    return out


@pytest.mark.parametrize("n", [1, 5, 520])  # rows that are split, and rows that are not
@pytest.mark.parametrize("v, top", [(40, 3), (300, 2), (8192, 2), (8192, 24), (8195, 8), (20000, 2), (20000, 30), (70000, 5)])
def test_a_unit_of_nan_hides_no_alternative(n, v, top):
    r = np.random.default_rng(v + top)
    a = np.full((n, v), -np.inf)
    a[0, :16] = np.nan
    a[0, min(5000, v - 1)] = 1.0
    for i in range(1, min(n, 8)):
        unit = np.arange(v) // 16
        a[i, r.random(v) < 2.0 / v] = r.standard_normal()
        a[i, r.random(v // 16 + 1)[unit] < (0.05, 0.5, 0.95)[i % 3]] = np.nan
    x, xv = matrix(r, n, v, "float32", a=a)
    with ops(n, 1, v) as s:
        logp, entropy, lse, top_logp, top_ids = s.logprob(x, ids(np.zeros(n, np.int64)), top=top)
    rows = slice(0, min(n, 10))
    assert (top_ids.cpu().numpy()[rows] == alternatives(xv[rows], top)).all()
    nan = np.isnan(xv).any(1)
    for t in (logp, entropy, lse, top_logp[:, 0]):
        assert (np.isnan(f64(t)) == nan).all()
