"""Norms of gradients beyond 32 bits are infinite, and so have no factor."""
import math

import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_learn import ops  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch

MOST = 2.0 ** 128 - 2.0 ** 104  # the largest number of 32 bits


@pytest.mark.parametrize("n", [4, 4_000_000])  # joined by the last to arrive, and by a launch of its own
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_norm_beyond_32_bits(ops, n, dtype):  # noqa: F811
    g = torch.full((n,), 2.0 ** 127, device="cuda", dtype=getattr(torch, dtype))
    p = torch.ones(n, device="cuda", dtype=g.dtype)
    group = ops.parameters([p], [g])
    keep = [t.clone() for t in group.tensors]
    norm, factor = ops.grad_norm(group, 1.0)       # 2^127 sqrt(n) in 64 bits
    assert norm.item() == math.inf and math.isnan(factor.item())
    ops.adamw(group, 1e-2, 1, factor=factor)
    assert all(torch.equal(a, b) for a, b in zip(group.tensors, keep))
    _, factor = ops.grad_norm(group, 1.0, out=(None, torch.empty(1, device="cuda")))
    assert math.isnan(factor.item())
    norm, factor = ops.grad_norm(group, math.inf)
    assert norm.item() == math.inf and math.isnan(factor.item())
    norm, factor = ops.grad_norm(group, 1.0, scale=2.0 ** -20)
    want = 2.0 ** 107 * math.sqrt(n)
    assert abs(norm.item() / want - 1) < 2 ** -23
    # 2^-20 / (2^107 sqrt(n)), 2^-128 or 2^-138, lies below the normal numbers, whose steps are 2^-149: one rounding is 2^-150
    assert abs(factor.item() - 2.0 ** -20 / want) <= 2.0 ** -150


def test_norm_at_the_largest_number(ops):  # noqa: F811
    """A norm that rounds to the largest number of 32 bits is one, the next is none."""
    one = ops.parameters(None, [torch.full((1,), MOST, device="cuda")])
    norm, factor = ops.grad_norm(one, MOST / 4)
    assert norm.item() == MOST and factor.item() == 0.25
    norm, factor = ops.grad_norm(one, MOST / 4, scale=1 + 2.0 ** -26)  # by less than half a step more
    assert norm.item() == MOST and abs(factor.item() - 0.25) <= 2.0 ** -24
    norm, factor = ops.grad_norm(one, MOST / 4, scale=1 + 2.0 ** -24)  # by half a step and a little more
    assert norm.item() == math.inf and math.isnan(factor.item())
