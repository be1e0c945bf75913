"""The fp64 oracle of the dense sublayer: gradients against central
differences, checkpoints against their definition."""

import numpy as np
import pytest

from oracle import layer as O

H = 1e-6


def numeric(f, x, g):
    """Central differences of sum(f(x) * g) by every element of x."""
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        lo, hi = x.copy(), x.copy()
        lo[i] -= H
        hi[i] += H
        out[i] = ((f(hi) - f(lo)) * g).sum() / (2 * H)
    return out


# central differences: truncation of order H^2 and rounding of order 1e-16 / H
# for values of order 10, so 1e-8 absolute
@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
def test_linear_gradients(name):
    rng = np.random.default_rng(3)
    a, w, b, r, g = (rng.normal(size=s) for s in ((4, 5), (6, 5), (6,), (4, 6), (4, 6)))
    z, _ = O.linear(a, w, b, r, name)
    assert np.abs(z).min() > 10 * H      # no difference across relu's corner
    da, dw, db, _ = O.linear_backward(g, a, w, z, name)
    assert np.allclose(da, numeric(lambda t: O.linear(t, w, b, r, name)[1], a, g), atol=1e-8)
    assert np.allclose(dw, numeric(lambda t: O.linear(a, t, b, r, name)[1], w, g), atol=1e-8)
    assert np.allclose(db, numeric(lambda t: O.linear(a, w, t, r, name)[1], b, g), atol=1e-8)


@pytest.mark.parametrize("center", [True, False])
def test_norm_gradients(center):
    rng = np.random.default_rng(4)
    s, g, gam, bet = (rng.normal(size=t) for t in ((3, 7), (3, 7), (7,), (7,)))
    _, mean, rstd = O.layer_norm(s, gam, bet, center)
    dx, dg, db = O.layer_norm_backward(g, s, mean, rstd, gam, None, center)
    assert np.allclose(dx, numeric(lambda t: O.layer_norm(t, gam, bet, center)[0], s, g), atol=1e-8)
    assert np.allclose(dg, numeric(lambda t: O.layer_norm(s, t, bet, center)[0], gam, g), atol=1e-8)
    assert np.allclose(db, numeric(lambda t: O.layer_norm(s, gam, t, center)[0], bet, g), atol=1e-8)


def test_checkpoint_is_the_nearest_code():
    """Every restored value is within half a step of a 3-bit mantissa (2^-4
    of the value), or of the smallest step 2^-9 2^e, and the largest of a
    block uses the upper half of the codes' range."""
    rng = np.random.default_rng(5)
    x = rng.normal(size=(9, 101)) * np.exp(4 * rng.normal(size=(9, 101)))
    codes, scales = O.checkpoint(x)
    v = O.restore(codes, scales)
    e = np.repeat(scales.astype(int), 32, axis=1)[:, :101] - 127
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** (e - 10))).all()
    for b in range(4):
        top = np.abs(x[:, 32 * b:32 * b + 32]).max(1) / 2.0 ** (scales[:, b].astype(int) - 127)
        assert (top <= 448).all() and (top > 224).all()


def test_checkpoint_of_zeros_and_non_finite_blocks():
    x = np.zeros((2, 64))
    x[1, 40], x[1, 3] = np.inf, -0.0
    codes, scales = O.checkpoint(x)
    assert scales.tolist() == [[10, 10], [10, 255]] and codes[1, 3] == 128
    assert (codes[0] == 0).all() and np.isnan(O.restore(codes, scales)[1, 32:]).all()
