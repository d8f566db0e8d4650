"""The float64 statements of norm, activation, 8-bit values and loss: gradients against differences, and the properties of the 8-bit form."""
import numpy as np
import pytest

from oracle import training_rest as rest


def _differences(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


@pytest.mark.parametrize("width", [1, 2, 5, 9])
def test_norm(width):
    rng = np.random.default_rng(width)
    s, w, b, dy = rng.standard_normal((3, width)), rng.standard_normal(width), rng.standard_normal(width), rng.standard_normal((3, width))
    f = lambda s, w, b: (rest.layer_norm(s, w, b, 1e-2)[0] * dy).sum()  # noqa: E731
    ds, dw, db = rest.layer_norm_bwd(s, w, 1e-2, dy)
    # differences of step 1e-5: off by 1e-10 of third derivatives, which eps keeps below 1e4, and 1e-11 of rounding
    np.testing.assert_allclose(ds, _differences(lambda x: f(x, w, b), s), atol=1e-6)
    np.testing.assert_allclose(dw, _differences(lambda x: f(s, x, b), w), atol=1e-6)
    np.testing.assert_allclose(db, _differences(lambda x: f(s, w, x), b), atol=1e-6)


@pytest.mark.parametrize("erf", [False, True])
def test_gelu(erf):
    x = np.linspace(-9, 9, 181)
    y, slope = rest.gelu(x, erf)
    np.testing.assert_allclose(slope, (rest.gelu(x + 1e-5, erf)[0] - rest.gelu(x - 1e-5, erf)[0]) / 2e-5, atol=1e-8)
    assert y[90] == 0 and slope[90] == 0.5 and abs(y[-1] - 9) < 1e-15 and abs(y[0]) < 1e-15
    # the two forms differ by less than 5e-4 everywhere
    assert np.abs(y - rest.gelu(x, not erf)[0]).max() < 5e-4


def test_loss():
    rng = np.random.default_rng(1)
    h, E = rng.standard_normal((5, 4)), rng.standard_normal((7, 4))
    labels, d = np.array([3, -1, 6, 7, 3]), rng.standard_normal(5)
    loss, lse = rest.vocab_loss(h, E, labels)
    assert loss[1] == lse[1] == loss[3] == lse[3] == 0
    dh, dE, dz = rest.vocab_loss_bwd(h, E, labels, d)
    f = lambda h, E: (rest.vocab_loss(h, E, labels)[0] * d).sum()  # noqa: E731
    np.testing.assert_allclose(dh, _differences(lambda x: f(x, E), h), atol=1e-8)
    np.testing.assert_allclose(dE, _differences(lambda x: f(h, x), E), atol=1e-8)
    assert (dh[1] == 0).all() and (dz[3] == 0).all()
    np.testing.assert_allclose(dz.sum(1), 0, atol=1e-15)
    h[1] = np.nan                                                   # a token without a label counts for nothing
    assert np.isfinite(rest.vocab_loss_bwd(h, E, labels, d)[1]).all()


@pytest.mark.parametrize("width", [1, 127, 128, 129, 300])
def test_eight_bits(width):
    rng = np.random.default_rng(width)
    x = (rng.standard_normal((6, width)) * 10.0 ** rng.uniform(-30, 30, (6, 1))).astype(np.float32)
    x[4] = 0
    x[5] = np.float32(1e-42)                                        # below 2^-126
    codes, units = rest.keep(x)
    back = rest.kept(codes, units)
    assert np.abs(codes.astype(int)).max() <= 127 and (back[4] == 0).all()
    unit = np.repeat(units, 128, 1)[:, :width].astype(np.float64)
    # half a unit; the reciprocal, the product and the way back are off by 2^-24 each of at most 127 units
    assert (np.abs(back.astype(np.float64) - x) <= unit * (0.5 + 127 * 3 * 2.0 ** -24)).all()
    again, u2 = rest.keep(back)
    np.testing.assert_allclose(rest.kept(again, u2), back, rtol=4 * 2.0 ** -24, atol=2.0 ** -126)
