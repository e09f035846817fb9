"""Pins of the plain 64-bit operators (oracle/stage.py): published answers of
the generator, closed forms, and gradients against differences."""
import numpy as np
import pytest

from oracle import stage as O


@pytest.mark.parametrize("counter, key, words", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator_gives_the_published_answers(counter, key, words):
    assert tuple(int(w) for w in O.philox4x32(np.array(counter), key)) == words


def test_dropout_mask_follows_the_row_and_not_its_place():
    rows = np.array([7, (3 << 32) | 5, 7, -1])
    keep, factor = O.dropout_keep(rows, 37, 0.25, 11, 4)
    assert (keep[0] == keep[2]).all() and not (keep[0] == keep[1]).all()
    assert factor == 65536 / (65536 - 16384)
    again, _ = O.dropout_keep(rows[::-1], 40, 0.25, 11, 4)
    assert (again[::-1, :37] == keep).all()
    assert not (O.dropout_keep(rows, 37, 0.25, 11, 5)[0] == keep).all()
    many, _ = O.dropout_keep(np.arange(400), 512, 0.25, 3, 0)
    # 204,800 draws: four standard deviations are 0.0038
    assert abs(many.mean() - 0.75) < 0.004


def test_uniform_and_masked_rows():
    x = np.zeros((3, 8))
    x[1, 2:] = -np.inf
    x[2] = -np.inf
    logp, entropy, lse, top_logp, ids = O.logprob(x, np.array([3, 5, -1]), 3)
    np.testing.assert_allclose(lse, [np.log(8), np.log(2), -np.inf])
    np.testing.assert_allclose(entropy, [np.log(8), np.log(2), 0], atol=1e-15)
    np.testing.assert_allclose(logp, [-np.log(8), -np.inf, 0])
    assert (ids == [[0, 1, 2]] * 3).all() and top_logp[1, 2] == -np.inf


def _slope(f, x, v, d=1e-6):
    return (f(x + d * v) - f(x - d * v)) / (2 * d)


def test_gradients_against_differences():
    r = np.random.default_rng(0)
    x, w, dy, dh, v = (r.standard_normal(s) for s in ((4, 9), 9, (4, 9), (4, 9), (4, 9)))
    rstd = O.norm(x, w, 1e-5)[1]
    dx, dw = O.norm_grad(dy, x, w, rstd, dh)
    f = lambda z: (O.norm(z, w, 1e-5)[2] * dy).sum() + (z * dh).sum()  # noqa: E731
    np.testing.assert_allclose((dx * v).sum(), _slope(f, x, v), rtol=1e-7)
    vw = r.standard_normal(9)
    np.testing.assert_allclose((dw * vw).sum(), _slope(lambda u: (O.norm(x, u, 1e-5)[2] * dy).sum(), w, vw), rtol=1e-7)
    t, gl, ge = np.array([0, 3, 9, -1]), r.standard_normal(4), r.standard_normal(4)
    _, entropy, lse, _, _ = O.logprob(x, t)
    g = O.logprob_grad(x, t, lse, entropy, gl, ge)

    def loss(z):
        lp, e, *_ = O.logprob(z, t)
        return (lp * gl).sum() + (e * ge).sum()
    np.testing.assert_allclose((g * v).sum(), _slope(loss, x, v), rtol=1e-7)
    tok = np.array([2, 0, 2, -1])
    np.testing.assert_allclose((O.embed_grad(tok, dy, 5, 3.0) * np.ones((5, 9))).sum(), 3 * dy[:3].sum())
