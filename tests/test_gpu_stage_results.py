"""Results of a call are tensors of their own."""
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_stage import ids, ops, torch_

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]


@pytest.mark.parametrize("top", [0, 3])
def test_results_of_log_probabilities_share_nothing(top):
    torch = torch_()
    x = torch.randn((6, 500), device="cuda")
    with ops(6, 1, 500) as s:
        logp, entropy, lse, top_logp, top_ids = s.logprob(x, ids([0, 1, 2, 3, 4, 5]), top=top)
    there = [t for t in (logp, entropy, lse, top_logp, top_ids) if t is not None]
    assert len({t.untyped_storage().data_ptr() for t in there}) == len(there)
    for t in there:
        assert t.untyped_storage().nbytes() == t.numel() * t.element_size()
    # one result changed in place while another is kept for a backward pass
    z = torch.ones(6, device="cuda", requires_grad=True)
    loss = (z * lse).sum()
    logp.mul_(2.0)
    entropy += z.detach()
    loss.backward()
    assert torch.equal(z.grad, lse)
    # and one that takes part in a graph itself
    entropy.mul_(z)
    assert entropy.requires_grad and not lse.requires_grad
