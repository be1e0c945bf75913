"""The bounds on fp32 errors are tight enough: an oracle that keeps fewer bits
than fp32 somewhere is outside of them at the sizes where they are used."""

import numpy as np
import pytest

from oracle import layer as O
from tests import _bounds as B
from tests._bounds import BACKWARD, FORWARD, SUBLAYER, rel


def bits(x, keep):
    """x rounded to `keep` significant bits (8: bf16, 11: a 10-bit mantissa)."""
    m, e = np.frexp(x)
    return np.ldexp(np.round(np.ldexp(m, keep)), e - keep)


def normals(seed, *shapes):
    rng = np.random.default_rng(seed)
    return [rng.normal(size=s) for s in shapes]


@pytest.mark.parametrize("m,n,k,parts", sorted({c[:4] for c in FORWARD}))
def test_products(m, n, k, parts):
    a, w = normals(m + n + k, (m, k), (n, k))
    want, bound, h = a @ w.T, B.product(k, parts), k // 2
    assert rel(bits(a, 8) @ bits(w, 8).T, want) > 2 * bound
    assert rel(bits(a, 11) @ bits(w, 11).T, want) > 2 * bound
    assert rel(bits(want, 8), want) > 2 * bound
    assert rel(bits(a[:, :h] @ w[:, :h].T, 8) + a[:, h:] @ w[:, h:].T, want) > 2 * bound
    assert rel(want.astype(np.float32), want) < bound


@pytest.mark.parametrize("m,n,k,act,_", BACKWARD)
def test_gradients(m, n, k, act, _):
    a, z, g, w = normals(m + n + k, (m, k), (m, n), (m, n), (n, k))
    da, dw, db, dz = O.linear_backward(g, a, w, z, act)
    extra = 0 if act in ("none", "relu") else 2 * 2.0 ** -20
    for keep in (8, 11):
        assert rel(bits(dz, keep) @ bits(w, keep), da) > 2 * (B.product(n) + extra)
        assert rel(bits(dz, keep).T @ bits(a, keep), dw) > 2 * (B.product(m) + extra)
        assert rel(bits(dz, keep).sum(0), db) > B.product(m) + extra


@pytest.mark.parametrize("n,d,f,act", SUBLAYER)
def test_sublayer(n, d, f, act):
    x, dout, w1, w2 = normals(n, (n, d), (n, d), (f, d), (d, f))
    w1, w2 = w1 / d ** 0.5, w2 / f ** 0.5

    def run(cut):
        h, mean, rstd = O.layer_norm(x)
        h = cut(h)
        z, u = O.linear(h, cut(w1), name=act)
        u = cut(u)
        out = O.linear(u, cut(w2), residual=x)[1]
        du, dw2, _, _ = O.linear_backward(dout, u, cut(w2))
        dh, dw1, _, _ = O.linear_backward(cut(du), h, cut(w1), cut(z), act)
        return out, dw2, dw1, O.layer_norm_backward(cut(dh), x, mean, rstd, None, dout)[0]

    want, less = run(lambda t: t), run(lambda t: bits(t, 8))
    assert rel(less[0], want[0]) > 4 * B.sublayer_forward(d, f)
    for p, q in zip(less[1:], want[1:]):
        assert rel(p, q) > 2 * B.sublayer_backward(n, d, f)
