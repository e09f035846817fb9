"""A min_p of 1 leaves the largest entries alone, in every form of the draw, however near the others come."""
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_learn import ops, uniform  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch

    from tests.test_gpu_learn import DT


@pytest.mark.parametrize("dtype,v", [("f32", 3000), ("bf16", 300), ("f32", 70000), ("bf16", 40000)])
@pytest.mark.parametrize("near,t", [(1e-17, 1.0), (1e-38, 1e-20), (1.0, 1e30), (0.25, 1e300)])  # weights of 1 less 1e-17 or less
def test_min_p_of_1(ops, dtype, v, near, t):  # noqa: F811
    x = torch.full((3, v), -30.0, device="cuda").to(DT[dtype])
    x[:, 10:30] = -near
    for i, n in enumerate((1, 2, 7)):
        x[i, 50:50 + n] = 0.0
    for kw in (dict(), dict(top_k=5), dict(top_k=250), dict(top_k=290), dict(top_p=0.999999), dict(top_k=20, top_p=0.9)):
        ids, _, kept = ops.sample(x, uniform(3, 1), temperature=t, min_p=1.0, **kw)
        most = 5 if kw.get("top_k") == 5 else 7
        # (top_p of twenty equal weights and more leaves all of the largest)
        assert kept.tolist() == [1, 2, most], (kw, kept)
        assert all(50 <= j < 50 + n for j, n in zip(ids.tolist(), (1, 2, most))), (kw, ids)
