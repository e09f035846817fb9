"""Step numbers, rates and other numbers that a step cannot be taken with."""
import itertools
import math

import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_learn import group_of, ops, state  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch

    from paper_2509_21221_amd.learn import LearnOps
    from paper_2509_21221_amd.mcf import GwtfError


@pytest.mark.parametrize("bits,master", itertools.product((32, 8), (False, True)))
@pytest.mark.parametrize("step,lr", [(0, 1e-2), (-1, 1e-2), (-2 ** 63, 1e-2), (3, math.nan), (3, math.inf), (3, -math.inf), (0, math.nan)])
def test_device_numbers_out_of_range_write_nothing(ops, bits, master, step, lr):  # noqa: F811
    s = state([5000, 5], "bf16", "f32", bits, master, 21)
    group = group_of(ops, s, weight_decay=0.1)
    before = [t.clone().view(torch.uint8) for t in group.tensors]
    step_at, lr_at = torch.tensor([step], device="cuda"), torch.tensor([lr], device="cuda")
    factor = torch.ones(1, device="cuda")
    if math.isfinite(lr):
        ops.adamw(group, lr, step_at, factor=factor)
    if step >= 1:
        ops.adamw(group, lr_at, step)
    ops.adamw(group, lr_at, step_at, factor=factor)
    assert all(torch.equal(a.view(torch.uint8), b) for a, b in zip(group.tensors, before))
    ops.adamw(group, lr_at.fill_(1e-2), step_at.fill_(1), factor=factor)
    assert not all(torch.equal(a.view(torch.uint8), b) for a, b in zip(group.tensors, before))


def test_captured_counter_that_moves_after_the_step():
    """A counter of 0 at the first replay: it leaves everything, the ones after it are steps 1, 2, .."""
    side = torch.cuda.Stream()
    runs = []
    for how in ("graph", "eager"):
        s = state([5000, 33], "bf16", "f32", 8, True, 32)
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side), LearnOps(stream=side) as o:
            group = group_of(o, s)
            if how == "graph":
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    o.adamw(group, 1e-2, step, seed=7)
                    step.add_(1)
                before = [t.clone().view(torch.uint8) for t in group.tensors]
                graph.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(a.view(torch.uint8), b) for a, b in zip(group.tensors, before))
                for _ in range(3):
                    s["grads"][0].mul_(1.5)
                    graph.replay()
                    torch.cuda.synchronize()
                del graph
            else:
                for t in (1, 2, 3):
                    s["grads"][0].mul_(1.5)
                    o.adamw(group, 1e-2, torch.tensor([t], device="cuda"), seed=7)
            torch.cuda.synchronize()
            runs.append([t.clone().view(torch.uint8) for t in group.tensors])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_numbers_that_are_infinite_in_32_bits_are_refused(ops):  # noqa: F811
    s = state([64], "bf16", "f32", 32, False, 24)
    group = group_of(ops, s)
    before = [t.clone().view(torch.uint8) for t in group.tensors]
    most = 2.0 ** 128 - 2.0 ** 104
    for kw, match in ((dict(lr=1e39), "lr"), (dict(lr=-1e39), "lr"), (dict(lr=2.0 ** 128), "lr"), (dict(eps=1e39), "eps"),
                      (dict(eps=most * (1 + 2.0 ** -24)), "eps")):
        with pytest.raises(GwtfError, match=match):
            ops.adamw(group, **{**dict(lr=1e-3, step=1), **kw})
    with pytest.raises(GwtfError, match="scale"):
        ops.grad_norm(group, 1.0, scale=1e39)
    with pytest.raises(GwtfError, match="weight_decay"):
        group_of(ops, s, weight_decay=1e39)
    assert all(torch.equal(a.view(torch.uint8), b) for a, b in zip(group.tensors, before))
    ops.adamw(group, 1e-3, 1, eps=most)  # the largest number is one: a step of nothing but the decay
    assert torch.equal(s["params"][0].view(torch.uint8), before[0])
    ops.grad_norm(group, 1e300, scale=most)
