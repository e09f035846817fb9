"""A call's status is that of its own work."""
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_stage import ids, ops, torch_

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]


def test_an_earlier_error_of_the_thread_is_not_a_calls_own():
    from paper_2509_21221_amd.mcf import load_library
    torch = torch_()
    hip = load_library()  # and the runtime that it is linked with
    x = torch.randn((40, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    t = ids([i % 64 for i in range(40)])
    with ops(40, 64, 64) as s:
        _, entropy, lse, _, _ = s.logprob(x)
        calls = [lambda: s.embed(t, x), lambda: s.embed_grad(t, x, 64), lambda: s.dropout(x, 0.1, 1, 2), lambda: s.norm(x, w),
                 lambda: s.norm_grad(x, x, w, lse), lambda: s.logprob(x, t, top=2),
                 lambda: s.logprob_grad(x, t, lse, entropy, lse, lse)]
        for call in calls:
            try:
                assert hip.hipSetDevice(1 << 20) != 0  # refused on the host; the runtime keeps the error
                call()
            finally:
                hip.hipGetLastError()
    torch.cuda.synchronize()
