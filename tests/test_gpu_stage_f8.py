"""8-bit values of the norm bit for bit.  With x = 1 and eps = 0 the norm is 1 and
y is the weight exactly, so that 32-bit quotients y / s and their nearest e4m3
values are known."""
import numpy as np
import pytest

from tests.gpu_util import have_gpu
from tests.test_gpu_stage import dt, ops, torch_

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]


def quotients(w, group):
    """(e4m3 values as bytes, scales) by 32-bit division on the CPU."""
    torch = torch_()
    q, scales = [], []
    for c in range(0, len(w), group):
        part = w[c:c + group]
        s = max(np.float32(np.abs(part).max() / np.float32(448)), np.float32(2.0 ** -126))
        q.append(np.clip(part / s, np.float32(-448), np.float32(448)))
        scales.append(s)
    return torch.from_numpy(np.concatenate(q)).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), np.array(scales, np.float32)


def ties():
    """Numbers below 448 half way between two e4m3 values."""
    return np.array([t for e in range(-6, 6) for m in range(8) if (t := (8 + m + 0.5) * 2.0 ** e) < 448])


def weights(kind, h, r):
    if kind == "ties":  # 448 k is each 128 columns' largest: s = k
        w = r.choice(ties(), h) * r.choice([-1, 1], h)
        k = 1 + 2 * r.integers(0, 70, (h + 127) // 128)  # 448 k is a 16-bit number too
        if h > 128:
            k[:] = k[0]  # one scale for the row form too
        w = w * np.repeat(k, 128)[:h]
        w[::128] = 448 * k
    elif kind == "near ties":
        w = r.choice(ties(), h) * 7 * (1 + r.integers(-2, 3, h) * 2.0 ** -23)
        w[::128] = 448 * 7
    else:
        w = r.standard_normal(h)
    return w


SCALES = [1.0, 2.0 ** 100, 2.0 ** -60, 2.0 ** -90, 2.0 ** -110, 2.0 ** -122, 2.0 ** -128, 2.0 ** -133]


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("kind", ["ties", "near ties", "random"])
@pytest.mark.parametrize("h", [1, 100, 640, 1500, 4096, 10000])
def test_values_are_the_nearest_to_the_quotients(dtype, kind, h):
    torch = torch_()
    r = np.random.default_rng(h)
    for scale in SCALES if dtype != "float16" else SCALES[:1]:
        w = torch.from_numpy(weights(kind, h, r) * scale).to(torch.float32).to(dt(dtype))
        wide = w.float().numpy()
        x = torch.ones((3, h), dtype=dt(dtype), device="cuda")
        with ops(3, h) as s:
            for quant, group in (("row", h), ("block", 128)):
                q, scales, _, rstd = s.norm(x, w.cuda(), 0.0, quant=quant)
                want, ws = quotients(wide, group)
                assert (rstd == 1).all()
                assert (scales.cpu().numpy() == ws).all()
                got = q.view(torch.uint8).cpu().numpy()
                bad = got != want
                assert not bad.any(), (quant, scale, bad.sum(), wide[bad[0]][:3], got[bad][:3])
