"""8-bit states below a code's smallest normal number: the remainder and the random bits are added up in 32 bits."""
import numpy as np
import pytest

from oracle import learn as O
from tests.gpu_util import have_gpu
from tests.test_gpu_learn import ops  # noqa: F401

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch

N, SEED, STEP, SITE = 128 * 512, 5, 3, 7


def borders(steps, least):
    """Values whose remainder and random part come to a whole step, to a number of 32 bits below it and to one above,
    among `steps` steps of size `least`; and the random bits."""
    r = O.draws(N, SEED, SITE, STEP)
    at = np.arange(N)
    exact = at // 3 % steps + 1 - (r + 0.5) / 65536
    x = exact.astype(np.float32)
    assert (x == exact).all()  # 3 + 17 bits
    return np.choose(at % 3, [x, np.nextafter(x, np.float32(0)), np.nextafter(x, np.float32(99))]) * np.float32(least), r


def check(ops, g, x, r, which, code):  # noqa: F811
    """With both betas 0 the states are g and g^2."""
    group = ops.parameters([torch.zeros(N, device="cuda")], [torch.from_numpy(g).cuda()], bits=8, sites=[SITE])
    ops.adamw(group, 0.0, STEP, betas=(0.0, 0.0), seed=SEED)
    got, scale = (group.m[0], group.m_scales[0]) if which == "m" else (group.v[0], group.v_scales[0])
    q, z = O.narrow(x, r, code)
    assert (z == 1).all() and np.array_equal(scale.cpu().numpy(), z)
    assert np.array_equal(got.double().cpu().numpy(), q)


def test_first_moment(ops):  # noqa: F811
    x, r = borders(8, 2.0 ** -9)
    x[::128] = 448.0  # of which the scale is 1
    check(ops, x, x, r, "m", "e4m3")
    check(ops, -x, -x, r, "m", "e4m3")


def test_second_moment(ops):  # noqa: F811
    x, r = borders(4, 2.0 ** -16)
    g = np.sqrt(x.astype(np.float64)).astype(np.float32)
    g[::128] = 224.0
    check(ops, g, g * g, r, "v", "e5m2")


def test_second_moment_far_below_its_block_stays_above_0(ops):  # noqa: F811
    """Values that the block's scale takes below the least number of 32 bits, beside 0."""
    g = np.zeros(N, np.float32)
    g[::128], g[1::128], g[2::128], g[3::128] = 1e18, 1e-6, 1e-18, 2.0 ** -74  # of 2^-148 the square is one step of 32 bits
    group = ops.parameters([torch.zeros(N, device="cuda")], [torch.from_numpy(g).cuda()], bits=8, sites=[SITE])
    ops.adamw(group, 0.0, STEP, betas=(0.0, 0.0), seed=SEED)
    v = group.v[0].float().view(-1, 128)
    assert (v[:, 0] > 28672).all() and (v[:, 1:4] == 2.0 ** -16).all() and (v[:, 4:] == 0).all()
    q, z = O.narrow(g * g, O.draws(N, SEED, SITE, STEP), "e5m2")
    assert np.array_equal(group.v_scales[0].cpu().numpy(), z) and np.array_equal(group.v[0].double().cpu().numpy(), q)
