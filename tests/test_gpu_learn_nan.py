"""Draws from rows with NaN, in forms that read a row at every look: one NaN is enough, wherever it lies and however
many lie beside it."""
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_learn import check_rows, logits, ops, uniform  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]


# widths beyond a lane's registers, whole steps of 512 columns among them, and (1,048,576 + 512) beyond the unfiltered form
@pytest.mark.parametrize("dtype,v", [("f32", 65536 + 512), ("f32", 128000), ("f32", 65537), ("bf16", 152064), ("f16", 256000),
                                     ("bf16", 131073), ("f32", 1048576 + 512), ("bf16", 1048576 + 512), ("f16", 1048576 + 500),
                                     ("bf16", 131072), ("f32", 1024)])
def test_blocks_of_nan_are_seen(ops, dtype, v):  # noqa: F811
    inf, nan = float("inf"), float("nan")
    x = logits(9, v, dtype, v)
    x[0] = nan
    x[1, :512] = nan                        # a whole step of a wave
    x[2, v // 1024 * 512:][:512] = nan
    x[3, (v - 1) // 512 * 512:] = nan       # the last one, whole or not
    x[4, 8 * 77:8 * 78] = nan               # a lane's eight
    x[5] = -inf
    x[5, 512:1024] = nan                    # among masked entries alone
    x[6, 1024 % v:] = -inf
    x[6, v - 1] = nan
    x[7, :512] = -inf                       # none: a row whose first step is masked
    for kw in (dict(), dict(top_k=20), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=1000, top_p=0.9, min_p=1e-3), dict(temperature=0.0)):
        ids, _, kept = check_rows(ops, x, uniform(9, 3), **kw)
        assert (ids[:7] == -1).all() and (kept[:7] == 0).all() and (ids[7:] >= 0).all()
