"""States that a list makes itself are ordered with the object's stream, whatever stream they are asked for on."""
import itertools

import pytest

from tests.gpu_util import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch

    from paper_2509_21221_amd.learn import LearnOps


def bits_of(group):
    return [t.clone().view(torch.uint8) for one in (group.params, group.m, group.v, group.m_scales, group.v_scales, group.master) if one for t in one]


@pytest.mark.parametrize("bits,master", itertools.product((32, 8), (False, True)))
def test_list_made_on_a_busy_stream(bits, master):
    own, busy = torch.cuda.Stream(), torch.cuda.Stream()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    start = [(torch.randn(n, device="cuda", generator=gen) * 0.02).bfloat16() for n in (3_000_000, 77, 1)]
    grads = [torch.randn(t.numel(), device="cuda", generator=gen).bfloat16() for t in start]
    big = torch.randn(4096, 4096, device="cuda")
    found = {}
    for how in ("in order", "apart"):
        params = [t.clone() for t in start]
        torch.cuda.synchronize()
        with LearnOps(stream=own) as o:
            if how == "apart":
                # memory that an earlier tensor has left behind, to be filled only after the products
                with torch.cuda.stream(busy):
                    left = [torch.full((3_000_000,), 3.0, device="cuda") for _ in range(5)]
                    for _ in range(20):
                        big = big @ big * 1e-3
                    del left
                    group = o.parameters(params, grads, bits=bits, master=master, weight_decay=0.1)
            else:
                group = o.parameters(params, grads, bits=bits, master=master, weight_decay=0.1)
                torch.cuda.synchronize()
            with torch.cuda.stream(own):
                for t in (1, 2):
                    o.adamw(group, 1e-3, t, seed=4)
            torch.cuda.synchronize()
            found[how] = bits_of(group)
    assert all(torch.equal(a, b) for a, b in zip(found["in order"], found["apart"]))


def test_list_made_after_a_step_on_the_other_stream():
    """Copies in 32 bits are of the weights that the object's pending work leaves; who asked for them can read them."""
    own, here = torch.cuda.Stream(), torch.cuda.Stream()
    p, g = torch.ones(2_000_000, device="cuda"), torch.ones(2_000_000, device="cuda")
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with LearnOps(stream=own) as o:
        with torch.cuda.stream(own):
            first = o.parameters([p], [g])
            for _ in range(20):
                big = big @ big * 1e-3
            o.adamw(first, 0.5, 1)
        with torch.cuda.stream(here):
            second = o.parameters([p], [g], master=True)
            copy, zeros = second.master[0] * 1, second.m[0] * 1
        torch.cuda.synchronize()
        assert torch.equal(copy, p) and (p != 1).all() and (zeros == 0).all()
