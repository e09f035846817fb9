"""GPU tests of include/gwtf_learn.h beyond 2^31 values: offsets of 64 bits in logits, gradients and states."""
import math

import numpy as np
import pytest

from oracle import learn as O
from tests.gpu_util import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

if have_gpu():
    import torch

    from paper_2509_21221_amd.learn import LearnOps

N = 2 ** 31 + 1029


def test_sample_rows_beyond_32_bits():
    n, v = 17000, 131072
    with LearnOps() as ops:
        x = torch.zeros(n, v, device="cuda", dtype=torch.bfloat16)
        rows = [0, 4095, 4096, 16383, 16384, n - 1]
        for i in rows:
            x[i] = torch.randn(v, device="cuda") * 2.5
        u = torch.rand(n, device="cuda", dtype=torch.float64)
        for kw in (dict(), dict(top_p=0.9), dict(top_k=30)):
            ids, _, kept = ops.sample(x, u, **kw)
            for i in rows:
                want = O.sample_row(x[i].double().cpu().numpy(), u[i].item(), **kw)
                assert (ids[i].item(), kept[i].item()) == (want[0], want[2]), (i, kw)
        # rows of equal logits: token floor(u V), since every border is a multiple of 1 / V
        ids, _, kept = ops.sample(x, u)
        even = torch.ones(n, dtype=torch.bool, device="cuda")
        even[rows] = False
        assert torch.equal(ids[even].long(), (u * v).floor().long()[even]) and (kept == v).all()


def test_norm_beyond_32_bits():
    with LearnOps() as ops:
        g = torch.full((N,), 0.5, device="cuda", dtype=torch.bfloat16)
        g[-1] = 4096.0
        norm, factor = ops.grad_norm(ops.parameters(None, [g]), 1.0)
        want = math.sqrt((N - 1) * 0.25 + 4096.0 ** 2)
        assert abs(norm.item() - want) <= 2.0 ** -24 * want * 1.01 and abs(factor.item() * want - 1) < 2e-7


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_beyond_32_bits(bits):
    tail, seed, step = 2 * 128 + 1029 % 128, 99, 3  # whole blocks and the last, shorter one
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    with LearnOps() as ops:
        p = torch.full((N,), 0.5, device="cuda", dtype=torch.bfloat16)
        g = torch.zeros(N, device="cuda", dtype=torch.bfloat16)
        g[-tail:] = torch.randn(tail, device="cuda", generator=gen).bfloat16()
        group = ops.parameters([p], [g], bits=bits)
        ops.adamw(group, 0.1, step, betas=(0.9, 0.95), seed=seed)
        zero = np.zeros(tail)
        grad = g[-tail:].double().cpu().numpy()
        want, m, v = O.adamw(zero + 0.5, grad, zero, zero, 0.1, step, (0.9, 0.95), 1e-8, 0.0)
        # one rounding to bf16, after the step's 32-bit ones
        assert (np.abs(p[-tail:].double().cpu().numpy() - want) <= 2.0 ** -8 * (np.abs(want) + 1e-6) + 1e-6).all()
        assert (p[: N - tail] == 0.5).all()
        m32, v32 = O.moments32(grad, zero, zero, (0.9, 0.95))
        if bits == 32:
            assert np.array_equal(group.m[0][-tail:].cpu().numpy(), m32) and np.array_equal(group.v[0][-tail:].cpu().numpy(), v32)
            return
        r = O.draws(tail, seed, 0, step, N - tail)
        for got, scale, x, kind in ((group.m[0], group.m_scales[0], m32, "e4m3"), (group.v[0], group.v_scales[0], v32, "e5m2")):
            q, z = O.narrow(x, r, kind)
            assert np.array_equal(scale[-len(z):].cpu().numpy(), z)
            assert np.array_equal(got[-tail:].double().cpu().numpy(), q)
