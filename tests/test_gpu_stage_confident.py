"""Rows that are sure of one word: no probability above one, no entropy below zero."""
import numpy as np
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_stage import E, TINY, TYPES, dt, f64, ops, torch_

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("std", [1e-3, 0.3, 3.0, 30.0, 3000.0, 60000.0])
@pytest.mark.parametrize("n, v, top", [(2000, 1, 1), (900, 5, 2), (300, 40, 3), (600, 9000, 30), (40, 70000, 4)])
def test_log_probabilities_and_entropies_keep_their_sign(dtype, std, n, v, top):
    torch = torch_()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(v)
    best = torch.rand(n, device="cuda", generator=gen) * std * (torch.randint(0, 2, (n,), device="cuda", generator=gen) * 2 - 1)
    at = torch.randint(0, v, (n,), device="cuda", generator=gen)
    x = torch.randn((n, v), device="cuda", generator=gen)
    x += best[:, None] - torch.tensor([120.0, 30.0, 12.0, float("inf")], device="cuda").repeat(n)[:n, None]
    x[torch.arange(n), at] = best
    x = x.to(dt(dtype))
    with ops(n, 1, v) as s:
        logp, entropy, lse, top_logp, _ = s.logprob(x, at, top=top)
    most = x.float().amax(1)
    assert bool((lse >= most).all())
    assert bool((logp <= 0).all()) and bool((top_logp <= 0).all()) and bool((entropy >= 0).all())
    # one word left: certain to the rounding of lse
    sure = np.arange(n) % 4 == 3
    off = 80 * E + 3 * E * np.abs(f64(most))
    assert (np.abs(f64(logp)) <= off + TINY["float32"])[sure].all() and (f64(entropy) <= 80 * E)[sure].all()
