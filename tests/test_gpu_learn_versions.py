"""What a call writes in place is seen by autograd: a graph that has kept the old values refuses its backward pass."""
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_learn import logits, ops, uniform  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch


def test_backward_after_an_update_is_refused(ops):  # noqa: F811
    w, b = (torch.nn.Parameter(torch.randn(n, device="cuda")) for n in ((8, 8), (8,)))
    w.grad, b.grad = torch.randn_like(w), torch.randn_like(b)
    grads = [w.grad, b.grad]
    group = ops.parameters([w, b], grads)
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    kept = torch.tanh(x @ w + b).sum()      # keeps w
    ops.adamw(group, 1e-2, 1)
    with pytest.raises(RuntimeError, match="inplace"):
        kept.backward()
    torch.tanh(x @ w + b).sum().backward()  # of the new weights
    assert w.grad is grads[0] and torch.isfinite(x.grad).all()


def test_versions_of_what_is_written(ops):  # noqa: F811
    flat = torch.randn(100, device="cuda")
    inner = torch.randn(5, 5, device="cuda")
    p = [flat[:50], flat[50:99].view(7, 7), inner, torch.randn(3, device="cuda").bfloat16()]
    g = [torch.randn(t.shape, device="cuda", dtype=t.dtype) for t in p]
    master = [t.float() * 1 for t in p]
    for group in (ops.parameters(p, g), ops.parameters(p, g, bits=8, master=master)):
        versions = [t._version for t in (*p, *g)]
        ops.adamw(group, 1e-3, 1)
        now = [t._version for t in (*p, *g)]
        assert all(a > b for a, b in zip(now[:4], versions)) and now[4:] == versions[4:]
    versions = [t._version for t in master]
    ops.adamw(group, 1e-3, 2)
    assert all(t._version > v for t, v in zip(master, versions))
    versions = [t._version for t in p]
    ops.grad_norm(group)
    assert versions == [t._version for t in p]


def test_versions_of_results_given(ops):  # noqa: F811
    x, u = logits(4, 700, "f32", 15), uniform(4, 15)
    out = ops.sample(x, u)
    scale = torch.ones(4, device="cuda", requires_grad=True)
    kept = (scale * out[1]).sum()
    assert ops.sample(x, u, top_k=3, out=out) is out
    with pytest.raises(RuntimeError, match="inplace"):
        kept.backward()
    group = ops.parameters(None, [torch.ones(5, device="cuda")])
    norm, factor = ops.grad_norm(group)
    scale = torch.ones(1, device="cuda", requires_grad=True)
    kept = (scale * factor).sum()
    ops.grad_norm(group, 0.5, out=(None, factor))
    with pytest.raises(RuntimeError, match="inplace"):
        kept.backward()
    ops.sample(x, u, out=(out[0], None, None))


def test_inference_tensors(ops):  # noqa: F811
    """Tensors without a version are written as they are."""
    with torch.inference_mode():
        x, u = logits(4, 700, "f32", 16), uniform(4, 16)
        out = ops.sample(x, u)
        ops.sample(x, u, out=out)
        p, g = torch.ones(9, device="cuda"), torch.ones(9, device="cuda")
        group = ops.parameters([p], [g])
        ops.adamw(group, 1e-2, 1)
    ops.adamw(group, 1e-2, 2)
    ops.sample(x, u, out=out)
    assert p.is_inference() and (p < 0.99).all()


def test_versions_of_copies_that_the_list_makes(ops):  # noqa: F811
    p, g = torch.ones(9, device="cuda").bfloat16(), torch.ones(9, device="cuda")
    group = ops.parameters([p], [g], master=True)
    scale = torch.ones(9, device="cuda", requires_grad=True)
    kept = (scale * group.master[0]).sum()
    ops.adamw(group, 1e-2, 1)
    with pytest.raises(RuntimeError, match="inplace"):
        kept.backward()
    empty = ops.parameters([], [])
    ops.adamw(empty, 1e-2, 1)
    assert empty.versions == ()
