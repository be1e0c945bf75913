"""Pins of the attention oracle: rotations against complex numbers and their
properties, scaled frequencies by hand, attention against torch's in fp64."""

import math

import numpy as np
import pytest
import torch

import paper_2511_11505_amd as fs
from oracle import attention as O


def rng(seed):
    return np.random.default_rng(seed)


def test_rotary_is_a_product_with_complex_numbers():
    r = rng(1)
    x, pos, f = r.standard_normal((5, 3, 12)), np.array([0, 1, 7, 1000, 12345]), O.frequencies(8)
    t = np.exp(1j * pos[:, None] * f)[:, None]
    got = O.rotary(x, pos, f, "pairs", 2)
    z = (x[..., 2:10:2] + 1j * x[..., 3:10:2]) * t
    assert np.allclose(got[..., 2:10:2], z.real) and np.allclose(got[..., 3:10:2], z.imag)
    got = O.rotary(x, pos, f, "halves", 4)
    z = (x[..., 4:8] + 1j * x[..., 8:12]) * t
    assert np.allclose(got[..., 4:8], z.real) and np.allclose(got[..., 8:], z.imag)
    assert np.array_equal(got[..., :4], x[..., :4])


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_rotary_backward_is_the_transpose(layout):
    r = rng(2)
    x, y, f = r.standard_normal((4, 2, 16)), r.standard_normal((4, 2, 16)), O.frequencies(16)
    pos = [3, 0, 99, 70000]
    a = (O.rotary(x, pos, f, layout, 0, 1.3) * y).sum()
    b = (x * O.rotary(y, pos, f, layout, 0, 1.3, back=True)).sum()
    assert abs(a - b) < 1e-12 * max(1.0, abs(a))
    # scores depend on the distance only
    q, k = x[:1], y[:1]
    s = [(O.rotary(q, [p + 5], f, layout) * O.rotary(k, [p], f, layout)).sum() for p in (0, 17, 4000)]
    assert np.allclose(s, s[0])


def test_frequencies():
    f = O.frequencies(8, 10000.0)
    assert np.allclose(f, [1, 0.1, 0.01, 0.001])
    assert np.allclose(O.frequencies(8, 10000.0, "linear", 4.0), f / 4)
    b = O.frequencies(8, 10000.0, "base", 4.0)
    assert np.allclose(b[0], 1) and np.allclose(b[-1], f[-1] / 4)
    # 1000 trained positions: 159, 15.9, 1.59 and 0.159 turns
    p = O.frequencies(8, 10000.0, "parts", 4.0, 1000.0, 1.0, 4.0)
    g = (10 / (2 * math.pi) - 1) / 3
    assert np.allclose(p, [f[0], f[1], f[2] * (g + (1 - g) / 4), f[3] / 4])


@pytest.mark.parametrize("rot", [0, 2, 6, 64, 512])
@pytest.mark.parametrize("kw", [dict(), dict(base=5e5), dict(scaling="linear", factor=3.5),
                                dict(scaling="base", factor=8.0),
                                dict(scaling="parts", factor=32.0, trained_len=8192.0, low=1.0, high=32.0)])
def test_the_librarys_frequencies(rot, kw):
    """Host code of the library: to 4 roundings of 64 bits (pow and exp log differ
    by the logarithm's rounding times its size, at most 14)."""
    if rot == 2 and kw.get("scaling") == "base":
        return
    want = O.frequencies(rot, **{{"trained_len": "trained"}.get(k, k): v for k, v in kw.items()})
    got = fs.fs_rope_frequencies(rot, **kw).numpy()
    assert np.all(np.abs(got - want) <= 64 * 2.0 ** -53 * want)


def test_append():
    r = rng(3)
    cache, rows = r.standard_normal((4, 2, 3, 8)), r.standard_normal((5, 2, 8))
    table = np.array([[2, -1], [0, 4]])
    got = O.append(cache, rows, [0, 0, 1, 1, 2], [1, 4, 0, 5, 0], table)
    assert np.array_equal(got[2, :, 1], rows[0]) and np.array_equal(got[0, :, 0], rows[2])
    got[2, :, 1], got[0, :, 0] = cache[2, :, 1], cache[0, :, 0]
    assert np.array_equal(got, cache)


@pytest.mark.parametrize("window", [0, 1, 4])
@pytest.mark.parametrize("new", [1, 3])
def test_attention_against_torch(new, window):
    r = rng(4 + new + window)
    kv, group, d, size, lens = 2, 3, 8, 4, [9, 2, 0, 13]
    pages = 12
    k, v = r.standard_normal((pages, kv, size, d)), r.standard_normal((pages, kv, size, d))
    table = np.full((4, 4), -1)
    order = iter(r.permutation(pages))
    for b, n in enumerate(lens):
        for j in range((n + size - 1) // size):
            table[b, j] = next(order)
    q = r.standard_normal((4 * new, kv * group, d))
    out, lse, mass, _ = O.attention(q, k, v, lens, table, new, 0.3, window)
    for b, n in enumerate(lens):
        kk, vv = (torch.from_numpy(np.stack([x[table[b, j // size], :, j % size] for j in range(n)], 1)
                                   if n else np.zeros((kv, 0, d))).repeat_interleave(group, 0) for x in (k, v))
        for i in range(new):
            at = n - new + i
            seen = [j for j in range(n) if j <= at and (not window or j > at - window)]
            t = b * new + i
            if not seen:
                assert (out[t] == 0).all() and np.isneginf(lse[t]).all()
                continue
            s = 0.3 * (kk[:, seen] @ torch.from_numpy(q[t])[..., None])[..., 0]
            want = (torch.softmax(s, 1)[:, None] @ vv[:, seen])[:, 0]
            assert np.allclose(out[t], want.numpy()) and np.allclose(lse[t], torch.logsumexp(s, 1).numpy())
            assert (mass[t] + 1e-12 >= np.abs(out[t])).all()


def test_holes_are_not_seen():
    r = rng(8)
    k, v, q = r.standard_normal((3, 1, 2, 8)), r.standard_normal((3, 1, 2, 8)), r.standard_normal((1, 1, 8))
    whole = O.attention(q, k, v, [2], np.array([[1]]))
    hole = O.attention(q, k, v, [4], np.array([[7, 1]]))
    assert np.allclose(whole[0], hole[0]) and np.allclose(whole[1], hole[1])
    none = O.attention(q, k, v, [4], np.array([[-1, 3]]))
    assert (none[0] == 0).all() and np.isneginf(none[1]).all()
