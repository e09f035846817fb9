"""Loops, launches and aliases of the microbatch operators that take many rows or
wide ones: gradients of log probabilities in whole steps, through and past the
caches, several rows a workgroup in the norm's gradient, results on inputs."""
import numpy as np
import pytest

from tests import test_gpu_stage as T
from tests.gpu_util import have_gpu
from tests.test_gpu_stage import E, TINY, TYPES, U, dt, ids, ops, torch_

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]


def placed(n, w, dtype, first, stride, gen=None, std=2.5):
    """n rows of w columns, `stride` apart, the first `first` elements after a boundary."""
    torch = torch_()
    flat = torch.full((n * stride + first,), T.SENTINEL, device="cuda", dtype=dt(dtype))
    view = flat[first:].view(n, stride)[:, :w]
    if gen is not None:
        view.copy_(torch.randn((n, w), device="cuda", generator=gen) * std)
    return flat, view


# whole steps are taken by workgroups that have 4,096 columns at least, so 512 rows and more
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, v, place, to", [
    (520, 4096, (0, 4096), (0, 4096)), (520, 9001, (0, 9001), (0, 9001)), (515, 9001, (3, 9011), (1, 9003)),
    (513, 12289, (5, 12290), (0, 12296)),
    (2048, 32001, (0, 32001), (0, 32001)), (2048, 32000, (0, 32000), (0, 32000)),  # past the caches
    (1500, 32001, (1, 32003), (7, 32008))])
def test_logprob_grad_in_whole_steps(dtype, n, v, place, to):
    torch = torch_()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(v)
    _, x = placed(n, v, dtype, *place, gen=gen)
    x[:, torch.rand(v, device="cuda", generator=gen) < 0.1] = float("-inf")
    x[n // 2] = float("-inf")
    # targets before the first step, on both sides of the steps' ends, in the last columns, outside
    edges = sorted({c for k in range(0, v + 2048, 2048) for c in range(k - 9, k + 9) if -2 <= c <= v + 1})
    tok = torch.tensor([edges[i % len(edges)] for i in range(n)], device="cuda")
    x64 = x.double()
    lse, gl, ge = torch.logsumexp(x64, 1).float(), torch.randn(n, device="cuda", generator=gen), torch.randn(n, device="cuda", generator=gen)
    live = torch.isfinite(lse)
    d = torch.where(torch.isfinite(x64) & live[:, None], x64 - torch.where(live, lse, 0).double()[:, None], -1e9)
    p = d.exp()
    entropy = -(p * d.clamp_min(-1e4)).sum(1).float()
    e64, gl64, ge64 = (t.double()[:, None] for t in (entropy, gl, ge))
    there = (tok >= 0) & (tok < v) & live
    gl64 = torch.where(there[:, None], gl64, 0)
    pl = p * (d.clamp_min(-1e4) + e64)
    want = -gl64 * p - ge64 * pl
    want.scatter_add_(1, tok.clamp(0, v - 1)[:, None], gl64)
    size = p * (gl64.abs() + ge64.abs() * (d.clamp_min(-1e4).abs() + e64.abs()))
    bound = (10 + 4 * d.clamp_min(-1e4).abs()) * E * size + (U[dtype] + 2 * E) * want.abs() + TINY[dtype] + 2.0 ** -126 * (
        gl64.abs() + 1e3 * ge64.abs())
    del x64, pl, size, p, d
    flat, out = placed(n, v, dtype, *to)
    with ops(n, 1, v) as s:
        s.logprob_grad(x, tok, lse, entropy, gl, ge, out=out)
        off = ~((out.double() - want).abs() <= bound)
        assert not bool(off.any()), (int(off.sum()), off.nonzero()[0].tolist())
        gaps = flat.clone()
        gaps[to[0]:].view(n, to[1])[:, :v] = T.SENTINEL
        assert bool((gaps == T.SENTINEL).all())
        kept = out.clone()
        s.logprob_grad(x, tok.int(), lse, entropy, gl, ge, out=x)
        # another alignment, the same values
        assert torch.equal(x, kept)


@pytest.mark.parametrize("dtype, n, h", [("float32", 1100, 4100), ("bfloat16", 1025, 5000), ("float32", 1030, 8200),
                                         ("bfloat16", 1100, 8193), ("float16", 600, 16384), ("float32", 513, 16383)])
def test_norm_grad_of_many_wide_rows(dtype, n, h):
    """Workgroups of 8 and 16 waves that take more than one row."""
    T.test_norm_grad(dtype, n, h, 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, h", [(1, 5), (7, 100), (9, 1000), (6, 1025), (5, 4095), (5, 8191), (3, 16001)])
def test_norm_writes_the_sum_onto_an_input(dtype, n, h):
    torch = torch_()
    r = np.random.default_rng(h)
    x, _ = T.matrix(r, n, h, dtype)
    res, _ = T.matrix(r, n, h, dtype)
    w = T.matrix(r, 1, h, dtype)[0][0]
    with ops(n, h) as s:
        for quant in ("none", "row", "block"):
            y, scales, kept, rstd = s.norm(x, w, residual=res, quant=quant)
            for onto in ("x", "residual"):
                a, b = x.clone(), res.clone()
                to = a if onto == "x" else b
                again = s.norm(a, w, residual=b, quant=quant,
                               out=(torch.empty_like(y), None if scales is None else torch.empty_like(scales), to, torch.empty_like(rstd)))
                for got, want in zip(again, (y, scales, kept, rstd)):
                    assert want is None or torch.equal(got.view(torch.uint8), want.view(torch.uint8))
                assert torch.equal(b if onto == "x" else a, res if onto == "x" else x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n, h", [(1, 5), (7, 100), (1030, 1000), (520, 1025), (600, 4095), (530, 8191), (515, 16001)])
def test_norm_grad_writes_onto_an_input(dtype, n, h):
    torch = torch_()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(h)
    dy, hh, dh = (torch.randn((n, h), device="cuda", generator=gen).to(dt(dtype)) for _ in range(3))
    w = torch.randn(h, device="cuda", generator=gen).to(dt(dtype))
    rstd = torch.rand(n, device="cuda", generator=gen) + 0.5
    with ops(n, h) as s:
        dx, dw = s.norm_grad(dy, hh, w, rstd, dh=dh)
        for onto in ("dy", "dh"):
            a, b = dy.clone(), dh.clone()
            got = s.norm_grad(a, hh, w, rstd, dh=b, out=(a if onto == "dy" else b, torch.empty_like(dw)))
            assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
            assert torch.equal(b if onto == "dy" else a, dh if onto == "dy" else dy)


@pytest.mark.parametrize("n", [1, 700, 5000])
def test_embed_grad_of_a_table_whose_absent_rows_are_not_kept(n):
    """More than 2^22 rows, tokens few enough to look through: all zeros in the first launch."""
    torch = torch_()
    v, h = (1 << 22) + 77, 5
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    dout = torch.randn((n, h), device="cuda", generator=gen)
    tok = torch.randint(-1, v + 1, (n,), device="cuda", generator=gen)
    tok[::3] = v - 1
    grad = torch.full((v, h), T.SENTINEL, device="cuda")
    with ops(n, h, v) as s:
        s.embed_grad(tok, dout, v, out=grad)
    there = (tok >= 0) & (tok < v)
    want = torch.zeros((v, h), device="cuda", dtype=torch.float64).index_add_(0, tok[there], dout[there].double())
    size = torch.zeros((v, h), device="cuda", dtype=torch.float64).index_add_(0, tok[there], dout[there].double().abs())
    assert bool(((grad.double() - want).abs() <= (n // 3 + 4) * E * size).all())


@pytest.mark.parametrize("dtype, v", [("float16", 1000), ("bfloat16", (1 << 21) + 3)])
def test_embed_grad_of_tokens_that_merge_three_times(dtype, v):
    """More than 2^21 tokens."""
    torch = torch_()
    n, h = (1 << 21) + 70001, 9
    gen = torch.Generator(device="cuda")
    gen.manual_seed(v)
    dout = torch.randn((n, h), device="cuda", generator=gen).to(dt(dtype))
    tok = (torch.rand(n, device="cuda", generator=gen) ** 4 * (v + 1)).long() - 1
    with ops(n, h, v) as s:
        got = s.embed_grad(tok, dout, v, dtype=torch.float32)
        assert torch.equal(got, s.embed_grad(tok.int(), dout, v, dtype=torch.float32))
    there = tok >= 0
    want = torch.zeros((v, h), device="cuda", dtype=torch.float64).index_add_(0, tok[there], dout[there].double())
    size = torch.zeros((v, h), device="cuda", dtype=torch.float64).index_add_(0, tok[there], dout[there].double().abs())
    count = torch.bincount(tok[there], minlength=v).double()[:, None]
    assert bool(((got.double() - want).abs() <= (count + 2) * E * size).all())
