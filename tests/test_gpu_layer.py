"""The dense sublayer's operators on the GPU against the fp64 oracle.

Tolerances are bounds, from the operations that round.  A sum of K fp32
products errs by at most K * 2^-23 of the sum of their absolute values (a
product and an add each round once, 2^-24); a stored value by half a step of
its type (bf16 2^-8 of it, fp32 2^-24); the activations' hardware exponential
and reciprocal by at most 2^-20 of the value.  |act'| is at most 1.13."""

import numpy as np
import pytest
import torch

import paper_2511_11505_amd as fs
from oracle import layer as O
from paper_2511_11505_amd import _lib as L
from tests import _bounds as B
from tests import _linear_rules as R
from tests._bounds import BACKWARD, FORWARD, SUBLAYER, rel
from tests._util import f64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]
DEV = "cuda"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": L.FS_F32, "bf16": L.FS_BF16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -23
ACT = 2.0 ** -20


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def mat(g, m, n, dtype, pad=0, scale=1.0, poison=float("nan"), lead=0):
    """[m, n] view with row stride n + pad; what is around it is NaN, so that a
    read past a row's end shows."""
    full = torch.full((m + 2, n + pad), poison, dtype=TORCH[dtype], device=DEV)
    v = full.view(-1)[lead:lead + (m + 1) * (n + pad)].view(m + 1, n + pad)[:m, :n]
    v.copy_(scale * torch.randn((m, n), generator=g, device=DEV))
    return v


class Out:
    """An output [m, n] inside a buffer of a sentinel, which has to stay."""

    def __init__(self, m, n, dtype, pad=0):
        self.full = torch.full((m + 2, n + pad), -77.0, dtype=TORCH[dtype], device=DEV)
        self.view = self.full[1:m + 1, :n]
        self.m, self.n = m, n

    def get(self):
        rest = self.full.clone()
        rest[1:self.m + 1, :self.n] = -77.0
        assert bool((rest == -77.0).all()), "wrote outside the output"
        return f64(self.view)


class Codes:
    def __init__(self, m, n):
        self.pair = fs.checkpoint_buffers(m, n)
        for t in self.pair:
            t.fill_(0x5A)

    def get(self):
        return tuple(t.cpu().numpy() for t in self.pair)


def workspace(nbytes):
    """Exactly nbytes of 0xFF (NaNs), with a guard behind."""
    ws = torch.full((nbytes + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    return ws, (ws.data_ptr(), nbytes)


def guard(ws, pair):
    assert bool((ws[pair[1]:] == 0xFF).all()), "wrote past the workspace"


def near(got, want, tol):
    bad = np.abs(got - want) > tol
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], np.asarray(tol)[bad][:4])
    assert np.isfinite(got).all()


def act_tol(z, zerr, name, value):
    """Error of act(z) from z's and its own."""
    return zerr if name == "none" else 1.13 * zerr + ACT * (np.abs(value) + np.abs(z) * 1e-3)


# ------------------------------------------------------------------- linear
SIZES = [(1, 1, 1), (1, 64, 64), (3, 5, 7), (17, 33, 31), (64, 64, 64), (65, 129, 130), (1, 300, 4096),
         (8, 96, 520), (130, 72, 1000), (200, 264, 96), (5, 1000, 2049), (257, 520, 328), (520, 260, 200)]


def check_linear(m, n, k, dtype, act, bias, residual, pad, seed=0, lead=0, scale_w=None, save=True):
    g = gen(seed + m + 3 * n + 7 * k)
    a = mat(g, m, k, dtype, pad, lead=lead)
    w = mat(g, n, k, dtype, pad, scale_w or k ** -0.5, lead=lead)
    b = torch.randn((n,), generator=g, device=DEV) if bias else None
    r = mat(g, m, n, dtype, pad) if residual else None
    desc = fs.linear_desc(m, n, k, dtype, act)
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR))
    out, z, zc, oc = Out(m, n, dtype, pad), Out(m, n, dtype, pad), Codes(m, n), Codes(m, n)
    save_z = fs.fs_saved(z.view.data_ptr(), z.view.stride(0), zc.pair[0].data_ptr(), zc.pair[1].data_ptr())
    fs.fs_linear(desc, a, w, b, r, out.view, wp, save_z=save_z if save else None,
                 save_out=oc.pair if save else None)
    torch.cuda.synchronize()
    guard(ws, wp)
    A, W = f64(a), f64(w)
    Z, want = O.linear(A, W, None if b is None else f64(b), None if r is None else f64(r), act)
    zerr = (k + 2) * U * (np.abs(A) @ np.abs(W).T + (0 if b is None else np.abs(f64(b))))
    value = O.act(Z, act)
    tol = act_tol(Z, zerr, act, value) + (0 if r is None else U * np.abs(want)) + HALF[dtype] * np.abs(want)
    near(out.get(), want, tol + HALF[dtype] * tol)
    if save:
        near(z.get(), Z, zerr + HALF[dtype] * (np.abs(Z) + zerr))
        # the checkpoints are those of the stored rows, code for code
        for rows, c in ((z, zc), (out, oc)):
            want_c = O.checkpoint(f64(rows.view))
            assert all(np.array_equal(x, y) for x, y in zip(c.get(), want_c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear(m, n, k, dtype):
    check_linear(m, n, k, dtype, "none", False, False, 0)


# sizes that fill the large tiles: whole tiles, ragged rows and columns, K that
# ends inside a block, the least K, one and several tiles per workgroup
# (and the 64 x 128 tiles: ragged edges, K in slices)
# (and operands that have to be copied first)
LARGE = [(900, 1501, 1409, 0), (3001, 2003, 777, 0), (2050, 2050, 301, 1), (1000, 1992, 520, 0), (520, 2056, 2056, 8), (70, 4104, 4104, 0), (513, 1000, 1992, 0), (4096, 2048, 256, 0), (3000, 2600, 328, 8), (6100, 1992, 200, 0), (2047, 4104, 520, 0),
         (9000, 2900, 264, 0)]


@pytest.mark.parametrize("m,n,k,pad", LARGE)
def test_linear_large(m, n, k, pad):
    check_linear(m, n, k, "bf16", "none", False, False, pad, save=False)


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_linear_large_epilogue(act):
    check_linear(2500, 2824, 264, "bf16", act, True, True, 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("m,n,k,pad", [(33, 70, 45, 0), (33, 70, 45, 3), (96, 128, 192, 8), (2, 40, 2048, 0)])
def test_linear_epilogue(m, n, k, pad, act, dtype):
    check_linear(m, n, k, dtype, act, True, True, pad)


@pytest.mark.parametrize("m,n,k", [(64, 128, 128), (3, 40, 1000), (300, 130, 264)])
def test_linear_unaligned_base(m, n, k):
    """Bases that only their element aligns."""
    check_linear(m, n, k, "bf16", "silu", True, False, 0, lead=1)
    check_linear(m, n, k, "f32", "silu", True, False, 0, lead=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_adds_into_the_residual(dtype):
    """out may be the residual itself, split over K or not."""
    for m, n, k in ((4, 40, 4096), (70, 96, 64)):
        g = gen(m)
        a, w, r = mat(g, m, k, dtype), mat(g, n, k, dtype, 0, k ** -0.5), mat(g, m, n, dtype)
        desc = fs.linear_desc(m, n, k, dtype)
        ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR))
        want = torch.empty_like(r)
        fs.fs_linear(desc, a, w, None, r, want, wp)
        got = r.clone()
        fs.fs_linear(desc, a, w, None, got, got, wp)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(5, 70, 100), (300, 520, 264)])
def test_linear_keeps_non_finite_values_in_their_rows(m, n, k, dtype):
    """A NaN or infinity in one token or output reaches its own row or column
    only, and reaches all of that."""
    g = gen(1)
    a, w = mat(g, m, k, dtype), mat(g, n, k, dtype, 0, k ** -0.5)
    a[m - 1, k - 1] = float("nan")
    w[n - 2, 0] = float("inf")
    desc = fs.linear_desc(m, n, k, dtype)
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR))
    out, oc = Out(m, n, dtype), Codes(m, n)
    fs.fs_linear(desc, a, w, None, None, out.view, wp, save_out=oc.pair)
    torch.cuda.synchronize()
    o = out.get()
    assert np.isnan(o[m - 1]).all() and np.isinf(o[:m - 1, n - 2]).all()
    assert np.isfinite(np.delete(o[:m - 1], n - 2, axis=1)).all()
    assert all(np.array_equal(x, y) for x, y in zip(oc.get(), O.checkpoint(o)))


def check_backward(m, n, k, dtype, act, pad, coded, seed=0, lead=0):
    g = gen(seed + m + 3 * n + 7 * k)
    a, z, dout = mat(g, m, k, dtype, pad, lead=lead), mat(g, m, n, dtype, pad, 1.3, lead=lead), mat(g, m, n, dtype, pad, lead=lead)
    w = mat(g, n, k, dtype, pad, n ** -0.5, lead=lead)
    desc = fs.linear_desc(m, n, k, dtype, act)
    A, Z = f64(a), f64(z)
    sa, sz = a, z
    if coded:
        sa, sz = Codes(m, k), Codes(m, n)
        fs.fs_checkpoint_fp8(CODE[dtype], m, k, a, *sa.pair)
        fs.fs_checkpoint_fp8(CODE[dtype], m, n, z, *sz.pair)
        A, Z = O.restore(*sa.get()), O.restore(*sz.get())
        sa, sz = sa.pair, sz.pair
    da, dw = Out(m, k, dtype, pad), Out(n, k, dtype, pad)
    db = torch.full((n,), float("nan"), device=DEV)
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR_BACKWARD))
    fs.fs_linear_backward(desc, dout, sa, w, None if act == "none" else sz, da.view, dw.view, db, wp)
    torch.cuda.synchronize()
    guard(ws, wp)
    G, W = f64(dout), f64(w)
    wa, ww, wb, dz = O.linear_backward(G, A, W, Z, act)
    # dz: the slope's error (its terms are at most 1 + |z|), then the rounding
    serr = 0.0 if act == "none" else ACT * (1 + np.abs(Z)) * np.abs(G)
    zerr = serr if act == "none" else serr + HALF[dtype] * (np.abs(dz) + serr)
    zerr = zerr + np.zeros_like(dz)
    hd = HALF[dtype]
    ta = zerr @ np.abs(W) + (n + 2) * U * (np.abs(dz) @ np.abs(W))
    tw = zerr.T @ np.abs(A) + (m + 2) * U * (np.abs(dz).T @ np.abs(A))
    near(da.get(), wa, ta * (1 + hd) + hd * np.abs(wa))
    near(dw.get(), ww, tw * (1 + hd) + hd * np.abs(ww))
    near(f64(db), wb, (serr + np.zeros_like(dz)).sum(0) + (m + 2) * U * np.abs(dz).sum(0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear_backward(m, n, k, dtype):
    check_backward(m, n, k, dtype, "none", 0, False)


@pytest.mark.parametrize("m,n,k,act,pad,coded", [
    (4096, 1024, 2048, "none", 0, False), (3000, 2600, 2504, "silu", 8, True),
    (1501, 1409, 2003, "none", 0, False), (1501, 1408, 2003, "silu", 0, False), (2003, 1409, 1504, "none", 0, False),
    (3000, 1001, 2002, "gelu", 1, True), (600, 2056, 2504, "silu", 0, False), (130, 1999, 4104, "relu", 0, True), (2500, 264, 520, "none", 8, False),
    (2047, 1999, 4104, "gelu", 0, False), (300, 4104, 3000, "relu", 0, True), (5000, 200, 6104, "none", 0, True),
    (6100, 3001, 1992, "silu", 0, True)])
def test_linear_backward_large(m, n, k, act, pad, coded):
    check_backward(m, n, k, "bf16", act, pad, coded)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("m,n,k,pad", [(33, 70, 45, 3), (96, 128, 192, 8), (130, 40, 2048, 0), (1, 33, 40, 0)])
def test_linear_backward_epilogue(m, n, k, pad, coded, act, dtype):
    check_backward(m, n, k, dtype, act, pad, coded)


def test_linear_backward_unaligned_base():
    check_backward(70, 136, 264, "bf16", "gelu", 0, False, lead=1)
    check_backward(70, 136, 264, "f32", "gelu", 0, False, lead=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_backward_parts(dtype):
    """Each gradient alone is what it is beside the others."""
    m, n, k = 70, 136, 200
    g = gen(9)
    a, z, dout, w = mat(g, m, k, dtype), mat(g, m, n, dtype), mat(g, m, n, dtype), mat(g, n, k, dtype)
    desc = fs.linear_desc(m, n, k, dtype, "silu")
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR_BACKWARD))

    def run(ia, iw, ib):
        da, dw = torch.empty((m, k), dtype=TORCH[dtype], device=DEV), torch.empty((n, k), dtype=TORCH[dtype], device=DEV)
        db = torch.empty((n,), device=DEV)
        fs.fs_linear_backward(desc, dout, a if iw else None, w if ia else None, z, da if ia else None,
                              dw if iw else None, db if ib else None, wp)
        return da, dw, db

    every = run(1, 1, 1)
    for i in range(3):
        assert torch.equal(run(*(int(i == j) for j in range(3)))[i], every[i])


def test_linear_backward_without_tokens():
    desc = fs.linear_desc(0, 40, 24, "bf16", "gelu")
    dw, db = torch.ones((40, 24), dtype=torch.bfloat16, device=DEV), torch.ones((40,), device=DEV)
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR_BACKWARD))
    fs.fs_linear_backward(desc, None, None, None, None, None, dw, db, wp)
    torch.cuda.synchronize()
    assert float(dw.float().abs().sum() + db.abs().sum()) == 0.0


# --------------------------------------------------------------- layer norm
NORM_SIZES = [(1, 1), (3, 7), (5, 64), (2, 515), (9, 1000), (4, 2048), (7, 2056), (3, 5120), (6, 7169),
              (2, 12345), (3, 20001), (1, 32768)]


def depth(d):
    """Adds in the longest chain of a row's sum: a thread's 8 columns of at
    most 4 chunks, the lanes, the waves."""
    return 32 + 6 + 16


def check_norm(m, d, dtype, center, add, affine, pad, offset=0.0, eps=1e-5):
    g = gen(m + d)
    x = mat(g, m, d, dtype, pad)
    x += offset
    e = mat(g, m, d, dtype, pad) if add else None
    gam = 1 + 0.3 * torch.randn((d,), generator=g, device=DEV) if affine else None
    bet = torch.randn((d,), generator=g, device=DEV) if affine else None
    desc = fs.norm_desc(m, d, dtype, center, eps)
    s, y = Out(m, d, dtype, pad), Out(m, d, dtype, pad)
    mean, rstd = torch.full((m,), float("nan"), device=DEV), torch.full((m,), float("nan"), device=DEV)
    xc, yc = Codes(m, d), Codes(m, d)
    fs.fs_layer_norm(desc, x, e, gam, bet, s.view, y.view, mean, rstd, save_in=xc.pair, save_y=yc.pair)
    torch.cuda.synchronize()
    S = s.get()
    if add:
        exact = f64(x) + f64(e)
        near(S, exact, HALF[dtype] * np.abs(exact) + U * np.abs(exact))
    else:
        assert np.array_equal(S, f64(x))
    G, B = (None if t is None else f64(t) for t in (gam, bet))
    Y, M, R = O.layer_norm(S, G, B, center, eps)
    # mean: its sum's chain; then var, from differences that err by the mean's
    # error and a rounding; rstd by half of var's relative error and three
    # roundings
    merr = (depth(d) * U * np.abs(S).mean(1) + U * np.abs(M)) if center else np.zeros(m)
    dev = S - M[:, None]
    derr = merr[:, None] + U * np.abs(dev)
    verr = (2 * np.abs(dev) * derr + derr ** 2).mean(1) + (depth(d) + 2) * U * (dev ** 2).mean(1)
    rrel = 0.5 * verr * R ** 2 + verr ** 2 * R ** 4 + 4 * U
    near(f64(mean), M if center else np.zeros(m), merr + 1e-30)
    near(f64(rstd), R, rrel * R)
    yerr = (derr * R[:, None] + np.abs(dev) * (R * rrel)[:, None]) * (1 if G is None else np.abs(G))
    yerr = yerr + 3 * U * (np.abs(Y) + (0 if B is None else 2 * np.abs(B)))
    near(y.get(), Y, yerr * (1 + HALF[dtype]) + HALF[dtype] * np.abs(Y))
    for rows, c in ((S, xc), (y.get(), yc)):
        assert all(np.array_equal(p, q) for p, q in zip(c.get(), O.checkpoint(rows)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,d", NORM_SIZES)
def test_norm(m, d, dtype):
    check_norm(m, d, dtype, True, True, True, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("add,affine,pad", [(False, True, 0), (True, False, 1), (False, False, 8)])
def test_norm_forms(add, affine, pad, center, dtype):
    for m, d in ((5, 77), (3, 4096)):
        check_norm(m, d, dtype, center, add, affine, pad)


def test_norm_of_far_and_flat_rows():
    """A mean a thousand times the spread, and rows without spread."""
    check_norm(4, 1000, "f32", True, False, True, 0, offset=1000.0)
    for dtype in ("f32", "bf16"):
        x = torch.full((3, 100), 2.5, dtype=TORCH[dtype], device=DEV)
        x[1] = 0
        y, rstd = torch.empty_like(x), torch.empty((3,), device=DEV)
        fs.fs_layer_norm(fs.norm_desc(3, 100, dtype, True, 1e-2), x, None, None, None, None, y, None, rstd)
        torch.cuda.synchronize()
        assert float(y.float().abs().max()) == 0.0
        assert np.allclose(f64(rstd), 10.0, rtol=1e-6)


def test_norm_in_place_and_non_finite_rows():
    g = gen(2)
    for m, d in ((5, 200), (4, 3000)):
        x, e = mat(g, m, d, "bf16"), mat(g, m, d, "bf16")
        desc = fs.norm_desc(m, d, "bf16")
        s, y = torch.empty_like(x), torch.empty_like(x)
        fs.fs_layer_norm(desc, x, e, None, None, s, y, None, None)
        x2, e2 = x.clone(), e.clone()
        fs.fs_layer_norm(desc, x2, e2, None, None, x2, e2, None, None)
        torch.cuda.synchronize()
        assert torch.equal(x2, s) and torch.equal(e2, y)
        x[1, 3], x[2, 0] = float("inf"), float("nan")
        bad = torch.empty_like(x)
        fs.fs_layer_norm(desc, x, e, None, None, None, bad, None, None)
        torch.cuda.synchronize()
        assert bool(bad[1:3].isnan().all())
        keep = [0, *range(3, m)]
        assert torch.equal(bad[keep], y[keep])


def check_norm_backward(m, d, dtype, center, coded, dres, affine, pad):
    g = gen(m + d)
    x, dy = mat(g, m, d, dtype, pad), mat(g, m, d, dtype, pad)
    r = mat(g, m, d, dtype, pad) if dres else None
    gam = 1 + 0.3 * torch.randn((d,), generator=g, device=DEV) if affine else None
    S = f64(x)
    sx = x
    if coded:
        c = Codes(m, d)
        fs.fs_checkpoint_fp8(CODE[dtype], m, d, x, *c.pair)
        S, sx = O.restore(*c.get()), c.pair
    _, M, R = O.layer_norm(f64(x), None, None, center)
    mean, rstd = (torch.tensor(t, dtype=torch.float32, device=DEV) for t in (M, R))
    M, R = f64(mean), f64(rstd)
    desc = fs.norm_desc(m, d, dtype, center)
    dx = Out(m, d, dtype, pad)
    dg, db = torch.full((d,), float("nan"), device=DEV), torch.full((d,), float("nan"), device=DEV)
    ws, wp = workspace(fs.fs_layer_norm_workspace(desc))
    fs.fs_layer_norm_backward(desc, dy, sx, mean if center else None, rstd, gam, r, dx.view, dg, db, wp)
    torch.cuda.synchronize()
    guard(ws, wp)
    DY, RES = f64(dy), None if r is None else f64(r)
    G = None if gam is None else f64(gam)
    wx, wg, wb = O.layer_norm_backward(DY, S, M, R, G, RES, center)
    h = (S - M[:, None]) * R[:, None]
    u = DY if G is None else DY * G
    herr, uerr = 2 * U * (np.abs(h) + np.abs(M * R)[:, None]), U * np.abs(u)
    chain = (depth(d) + 2) * U
    m1, m2 = np.abs(u).mean(1), (np.abs(u * h)).mean(1)
    e1 = chain * m1
    e2 = chain * m2 + (herr * np.abs(u) + uerr * np.abs(h)).mean(1)
    terr = uerr + e1[:, None] + herr * m2[:, None] + np.abs(h) * e2[:, None]
    terr = terr + 4 * U * (np.abs(u) + m1[:, None] + np.abs(h) * m2[:, None])
    xerr = terr * R[:, None] + 2 * U * (np.abs(wx) + (0 if RES is None else np.abs(RES)))
    near(dx.get(), wx, xerr * (1 + HALF[dtype]) + HALF[dtype] * np.abs(wx))
    near(f64(dg), wg, (m + 34) * U * np.abs(DY * h).sum(0) + (np.abs(DY) * herr).sum(0))
    near(f64(db), wb, (m + 34) * U * np.abs(DY).sum(0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("m,d", NORM_SIZES + [(700, 40), (1100, 300), (600, 2100), (5000, 24), (700, 9000)])
def test_norm_backward(m, d, coded, dtype):
    check_norm_backward(m, d, dtype, True, coded, True, True, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dres,affine,pad", [(False, True, 0), (True, False, 1), (False, False, 8)])
def test_norm_backward_forms(dres, affine, pad, center, dtype):
    for m, d in ((5, 77), (9, 4096)):
        check_norm_backward(m, d, dtype, center, pad == 1, dres, affine, pad)


def test_norm_backward_parts_in_place_and_without_rows():
    m, d = 40, 600
    g = gen(5)
    x, dy, r = (mat(g, m, d, "bf16") for _ in range(3))
    mean, rstd = torch.zeros((m,), device=DEV), torch.ones((m,), device=DEV)
    desc = fs.norm_desc(m, d, "bf16")
    ws, wp = workspace(fs.fs_layer_norm_workspace(desc))

    def run(dy, r, dx, dg, db, wp):
        fs.fs_layer_norm_backward(desc, dy, x, mean, rstd, None, r, dx, dg, db, wp)
        return dx

    dg, db = torch.empty((d,), device=DEV), torch.empty((d,), device=DEV)
    want = run(dy, r, torch.empty_like(dy), dg, db, wp)
    g1, b1 = torch.empty_like(dg), torch.empty_like(db)
    assert torch.equal(run(dy, r, torch.empty_like(dy), None, None, None), want)
    run(dy, r, torch.empty_like(dy), g1, None, wp)
    run(dy, r, torch.empty_like(dy), None, b1, wp)
    assert torch.equal(g1, dg) and torch.equal(b1, db)
    y2, r2 = dy.clone(), r.clone()
    assert torch.equal(run(y2, r, y2, None, None, None), want)
    assert torch.equal(run(dy, r2, r2, None, None, None), want)
    none = fs.norm_desc(0, d, "bf16")
    fs.fs_layer_norm_backward(none, None, None, None, None, None, None, None, g1, b1, None)
    torch.cuda.synchronize()
    assert float(g1.abs().sum() + b1.abs().sum()) == 0.0


# -------------------------------------------------------------- checkpoints
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,d,pad", [(1, 1, 0), (3, 31, 0), (5, 32, 1), (7, 33, 0), (300, 70, 8), (9, 2500, 3)])
def test_checkpoint(m, d, pad, dtype):
    g = gen(m + d)
    x = mat(g, m, d, dtype, pad)
    x.mul_(torch.exp(6 * torch.randn((m, d), generator=g, device=DEV)))
    c, back = Codes(m, d), Out(m, d, dtype, pad)
    fs.fs_checkpoint_fp8(CODE[dtype], m, d, x, *c.pair)
    fs.fs_checkpoint_restore(CODE[dtype], m, d, *c.pair, back.view)
    torch.cuda.synchronize()
    assert all(np.array_equal(p, q) for p, q in zip(c.get(), O.checkpoint(f64(x))))
    assert np.array_equal(back.get(), O.restore(*c.get()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_checkpoint_edges(dtype):
    """Ties, the border of a scale, the smallest and largest values, zeros of
    both signs, infinities and NaNs."""
    big = float(torch.finfo(TORCH[dtype]).max)
    rows = [[448.0, 17.0, 19.0, -0.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9], [450.0, 17.0, 1.0], [0.0, -0.0],
            [big, -big, 1.0], [2.0 ** -126, 2.0 ** -117, -2.0 ** -120], [1e-38, 2e-38], [float("inf"), 1.0],
            [float("nan"), 5.0], [-float("inf")]]
    x = torch.zeros((len(rows), 64), dtype=TORCH[dtype], device=DEV)
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r, device=DEV).to(TORCH[dtype])
        x[i, 63] = 3.0
    c, back = Codes(len(rows), 64), torch.empty_like(x)
    fs.fs_checkpoint_fp8(CODE[dtype], len(rows), 64, x, *c.pair)
    fs.fs_checkpoint_restore(CODE[dtype], len(rows), 64, *c.pair, back)
    torch.cuda.synchronize()
    want = O.checkpoint(f64(x))
    assert all(np.array_equal(p, q) for p, q in zip(c.get(), want))
    assert np.array_equal(f64(back), O.restore(*want), equal_nan=True)


# ------------------------------------------- offsets that pass 32 bits
def test_offsets_past_32_bits():
    """The last rows of matrices of more than 2^32 elements are what the same
    rows give alone."""
    m, d, tail = (1 << 19) + 70, 8200, 37
    g = gen(8)
    x = torch.zeros((m, d), dtype=torch.bfloat16, device=DEV)
    x[-tail:] = torch.randn((tail, d), generator=g, device=DEV).bfloat16()
    assert x.numel() > 1 << 32
    # checkpoint and back
    c, small = fs.checkpoint_buffers(m, d), fs.checkpoint_buffers(tail, d)
    fs.fs_checkpoint_fp8(L.FS_BF16, m, d, x, *c)
    fs.fs_checkpoint_fp8(L.FS_BF16, tail, d, x[-tail:], *small)
    assert torch.equal(c[0][-tail:], small[0]) and torch.equal(c[1][-tail:], small[1])
    y = torch.empty_like(x)
    fs.fs_checkpoint_restore(L.FS_BF16, m, d, *c, y)
    part = torch.empty((tail, d), dtype=torch.bfloat16, device=DEV)
    fs.fs_checkpoint_restore(L.FS_BF16, tail, d, *small, part)
    assert torch.equal(y[-tail:], part)
    # norm and its backward pass
    mean, rstd = torch.empty((m,), device=DEV), torch.empty((m,), device=DEV)
    big, few = fs.norm_desc(m, d), fs.norm_desc(tail, d)
    fs.fs_layer_norm(big, x, None, None, None, None, y, mean, rstd)
    fs.fs_layer_norm(few, x[-tail:], None, None, None, None, part, None, None)
    assert torch.equal(y[-tail:], part)
    dg, dg2 = torch.empty((d,), device=DEV), torch.empty((d,), device=DEV)
    xr = torch.empty_like(part)
    fs.fs_checkpoint_restore(L.FS_BF16, tail, d, *small, xr)
    terms = (part.double() * (xr.double() - mean[-tail:, None]) * rstd[-tail:, None]).abs().sum(0)
    ws = torch.empty((fs.fs_layer_norm_workspace(big),), dtype=torch.uint8, device=DEV)
    fs.fs_layer_norm_backward(big, y, c, mean, rstd, None, x, y, dg, None, ws)
    fs.fs_layer_norm_backward(few, part, small, mean[-tail:], rstd[-tail:], None, x[-tail:], part, dg2, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(y[-tail:], part)
    # the same 37 terms in two orders (the rows before add exact zeros): each
    # order rounds at most 36 sums, and each term at most 3 times (a difference,
    # two products), by half a step (U / 2) of at most the terms' absolute sum
    assert ((dg - dg2).abs().double() <= 2 * (tail + 3) * U / 2 * terms).all()


@pytest.mark.parametrize("k", [40, 264])
def test_linear_offsets_past_32_bits(k):
    """As above, with more output elements than 2^32: tokens that are zeros
    but for the last rows."""
    m, n, tail = (1 << 19) + 70, 8200, 37
    g = gen(9)
    a = torch.zeros((m, k), dtype=torch.bfloat16, device=DEV)
    a[-tail:] = torch.randn((tail, k), generator=g, device=DEV).bfloat16()
    w = torch.randn((n, k), generator=g, device=DEV).bfloat16()
    desc = fs.linear_desc(m, n, k, "bf16", "relu")
    out = torch.empty((m, n), dtype=torch.bfloat16, device=DEV)
    z = fs.checkpoint_buffers(m, n)
    ws = torch.empty((max(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR), 256),), dtype=torch.uint8, device=DEV)
    fs.fs_linear(desc, a, w, None, None, out, ws, save_z=z)
    Z = f64(a[-tail:]) @ f64(w).T
    err = (k + 2) * U * (np.abs(f64(a[-tail:])) @ np.abs(f64(w)).T)
    near(f64(out[-tail:]), np.maximum(Z, 0), err + HALF["bf16"] * (np.abs(Z) + err))
    # the gradients of zero rows are zeros; of the last, the small call's
    ws = torch.empty((fs.fs_linear_workspace(desc, L.FS_OP_LINEAR_BACKWARD),), dtype=torch.uint8, device=DEV)
    da, dw = torch.empty_like(a), torch.empty_like(w)
    fs.fs_linear_backward(desc, out, a, w, z, da, dw, None, ws)
    torch.cuda.synchronize()
    zt = O.restore(*(t[-tail:].cpu().numpy() for t in z))
    G = f64(out[-tail:]) * (zt > 0)
    wa, ww = G @ f64(w), G.T @ f64(a[-tail:])
    near(f64(da[-tail:]), wa, (n + 2) * U * (np.abs(G) @ np.abs(f64(w))) + HALF["bf16"] * 1.01 * np.abs(wa))
    near(f64(dw), ww, (tail + 40) * U * (np.abs(G).T @ np.abs(f64(a[-tail:]))) + HALF["bf16"] * 1.01 * np.abs(ww))
    assert float(da[:-tail].abs().max()) == 0.0


# ------------------------------------------------------------ used together
def sublayer_oracle(x, dout, p, act, center, rounded, coded):
    """Forward and gradients of DenseSublayer with its roundings."""
    gam, bet, w1, b1, w2, b2 = p
    keep = (lambda t: O.restore(*O.checkpoint(t))) if coded else (lambda t: t)
    h, mean, rstd = O.layer_norm(x, gam, bet, center)
    h = rounded(h)
    z, u = O.linear(h, w1, b1, None, act)
    u = rounded(u)
    _, out = O.linear(u, w2, b2, x)
    z = rounded(z)
    du, dw2, db2, _ = O.linear_backward(dout, keep(u), w2)
    dh, dw1, db1, _ = O.linear_backward(rounded(du), keep(h), w1, keep(z), act)
    dx, dg, db = O.layer_norm_backward(rounded(dh), keep(x), mean, rstd, gam, dout, center)
    return out, dict(x=dx, gamma=dg, beta=db, w1=dw1, b1=db1, w2=dw2, b2=db2)


def make_sublayer(n, d, f, dtype, act, center, save, seed=0):
    g = gen(seed)
    t = TORCH[dtype]
    p = [1 + 0.2 * torch.randn((d,), generator=g, device=DEV), 0.2 * torch.randn((d,), generator=g, device=DEV),
         (torch.randn((f, d), generator=g, device=DEV) * d ** -0.5).to(t), 0.2 * torch.randn((f,), generator=g, device=DEV),
         (torch.randn((d, f), generator=g, device=DEV) * f ** -0.5).to(t), 0.2 * torch.randn((d,), generator=g, device=DEV)]
    layer = fs.DenseSublayer(n, *p, act=act, center=center, save=save)
    x, dout = (torch.randn((n, d), generator=g, device=DEV).to(t) for _ in range(2))
    grads = dict(x=torch.empty_like(x), w1=torch.empty_like(p[2]), w2=torch.empty_like(p[4]),
                 **{k: torch.empty((s,), device=DEV) for k, s in (("gamma", d), ("beta", d), ("b1", f), ("b2", d))})
    return p, layer, x, dout, grads


# With fp32 rows the sublayer's values and gradients differ from the oracle's
# by sums of at most 600 terms: 600 * 2^-23 of sums of absolute values, which
# are about sqrt(600) = 25 times the sums: 2e-3 of the rms at worst.  In bf16
# a stored h, u, du, dh and dz each err by half a step, 2^-9 on average; of
# five such in turn at most 5 * 2^-8 = 2e-2.  (relative norms)
@pytest.mark.parametrize("dtype,tol", [("f32", 2e-3), ("bf16", 2e-2)])
@pytest.mark.parametrize("save", ["rows", "codes"])
@pytest.mark.parametrize("n,d,f,act,center", [(70, 96, 264, "silu", True), (33, 130, 70, "gelu", False),
                                              (600, 128, 320, "relu", True)])
def test_sublayer(n, d, f, act, center, save, dtype, tol):
    p, layer, x, dout, grads = make_sublayer(n, d, f, dtype, act, center, save)
    out = layer.forward(x, torch.empty_like(x))
    layer.backward(dout, grads)
    torch.cuda.synchronize()

    def rounded(v):
        return f64(torch.tensor(v).to(TORCH[dtype]))

    want, wg = sublayer_oracle(f64(x), f64(dout), [f64(t) for t in p], act, center, rounded, save == "codes")

    def rel(a, b):
        return np.linalg.norm(f64(a) - b) / np.linalg.norm(b)

    assert rel(out, want) <= tol
    for k, v in grads.items():
        # codes: a value at a code's border may fall to the other side (two in
        # a thousand do in bf16, one step of 2^-3 each: 2^-3 sqrt(2e-3) = 6e-3)
        assert rel(v, wg[k]) <= tol + (6e-3 if save == "codes" else 0), k


def test_sublayer_serving_matches_training():
    p, layer, x, dout, grads = make_sublayer(40, 128, 256, "bf16", "silu", True, "codes")
    want = layer.forward(x, torch.empty_like(x))
    serve = fs.DenseSublayer(40, *p, act="silu")
    got = serve.forward(x, torch.empty_like(x))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    with pytest.raises(ValueError):
        serve.backward(dout, grads)


@pytest.mark.parametrize("n", [1, 64, 300])
def test_sublayer_in_a_graph_and_on_a_side_stream(n):
    """Forward and backward captured once and replayed on new inputs, with
    eager work between; and the same calls on another stream."""
    p, layer, x, dout, grads = make_sublayer(n, 256, 520, "bf16", "gelu", True, "codes")
    _, eager, _, _, egrads = make_sublayer(n, 256, 520, "bf16", "gelu", True, "codes")
    out, eout = torch.empty_like(x), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.forward(x, out)
        layer.backward(dout, grads)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, out)
        layer.backward(dout, grads)
    g = gen(77)
    for _ in range(4):
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        dout.copy_(torch.randn(x.shape, generator=g, device=DEV))
        eager.forward(x, eout)
        eager.backward(dout, egrads)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eout)
        for k in grads:
            assert torch.equal(grads[k], egrads[k]), k


def test_two_sublayers_at_once():
    """Two sublayers' passes on two streams, captured into two graphs that are
    replayed together, are what each gives alone."""
    runs = []
    for i, (n, d, f) in enumerate(((300, 256, 1032), (257, 520, 776))):
        p, layer, x, dout, grads = make_sublayer(n, d, f, "bf16", "silu", True, "codes", seed=i)
        out = torch.empty_like(x)

        def step(layer=layer, x=x, out=out, dout=dout, grads=grads):
            layer.forward(x, out)
            layer.backward(dout, grads)

        step()
        torch.cuda.synchronize()
        want = [out.clone(), *(grads[k].clone() for k in sorted(grads))]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        runs.append((graph, torch.cuda.Stream(), want, out, grads, step))
    for way in ("graphs", "streams"):
        for _ in range(4):
            for graph, stream, want, out, grads, step in runs:
                stream.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(stream):
                    graph.replay() if way == "graphs" else step()
            torch.cuda.synchronize()
            for _, _, want, out, grads, _ in runs:
                got = [out, *(grads[k] for k in sorted(grads))]
                assert all(torch.equal(a, b) for a, b in zip(got, want)), way
                for t in got:
                    t.zero_()


def test_sublayer_in_the_far_skip_window():
    """The sublayer as the next layer of a block: BEGIN, the sublayer on the
    partial input, FINISH into its output."""
    from workloads import CONFIGS, make_workload
    cfg = CONFIGS["tiny"]
    wl = make_workload(cfg, DEV)
    blk = fs.MoEBlock(cfg, wl.w_router, None, wl.w_gate_up, wl.w_down, device=DEV)
    d = cfg.hidden
    p, layer, _, _, _ = make_sublayer(cfg.n_tokens, d, 2 * d, "f32", "silu", False, None)
    comm = torch.cuda.Stream()
    partial, out = torch.empty_like(wl.x), torch.empty_like(wl.x)
    blk.begin(wl.x, partial, comm=comm)
    layer.forward(partial, out)
    nxt = out.clone()
    blk.finish(wl.x, out, comm=comm)
    routed = torch.empty_like(wl.x)
    L.fs_combine_unpack(blk.desc, blk.y_ret(), blk.t["slot_to_row"], blk.t["topk_w"], None, routed, None)
    torch.cuda.synchronize()
    gam, bet, w1, b1, w2, b2 = (f64(t) for t in p)
    h, _, _ = O.layer_norm(f64(partial), gam, bet, False)
    want = O.linear(O.linear(h, w1, b1, None, "silu")[1], w2, b2, f64(partial))[1]
    assert np.linalg.norm(f64(nxt) - want) <= 2e-3 * np.linalg.norm(want)
    # FINISH adds the routed output, one rounding
    both = f64(nxt) + f64(routed)
    near(f64(out), both, 4 * U * (np.abs(f64(nxt)) + np.abs(f64(routed))))
    blk.close()


# --------------------------------------------- arguments that are left alone
# (a size for each kernel that ends in the epilogue: few tokens, waves that
# split K, 64 x 64 tiles, 64 x 128 tiles with and without slices, 128 x 256 tiles)
@pytest.mark.parametrize("m,n,k", [(3, 96, 520), (64, 512, 512), (130, 72, 1000), (300, 1001, 1409), (128, 4096, 4096),
                                   (520, 2056, 2056), (4096, 2048, 256)])
def test_scales_without_codes_are_left_alone(m, n, k):
    """z saved as rows, in a struct whose scales are set: they stay as they
    were, and the call gives what it gives without them."""
    g = gen(m + n)
    a, w = mat(g, m, k, "bf16"), mat(g, n, k, "bf16", 0, k ** -0.5)
    desc = fs.linear_desc(m, n, k, "bf16", "silu")
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR))
    scales = torch.full((m, (n + 31) // 32), 0x5A, dtype=torch.uint8, device=DEV)
    got = []
    for extra in (None, scales.data_ptr()):
        out, z = Out(m, n, "bf16"), Out(m, n, "bf16")
        save_z = fs.fs_saved(z.view.data_ptr(), z.view.stride(0), None, extra)
        fs.fs_linear(desc, a, w, None, None, out.view, wp, save_z=save_z)
        torch.cuda.synchronize()
        got.append((out.get(), z.get()))
    assert bool((scales == 0x5A).all())
    assert all(np.array_equal(p, q) for p, q in zip(*got))


@pytest.mark.parametrize("save", [None, "codes"])
@pytest.mark.parametrize("n,d,f", [(3, 128, 256), (300, 520, 1032)])
def test_sublayer_in_place(n, d, f, save):
    """out is x itself, where the backward pass does not read x: the bits of
    the same pass into another tensor, forward and backward."""
    _, layer, x, dout, grads = make_sublayer(n, d, f, "bf16", "silu", True, save)
    want = layer.forward(x, torch.empty_like(x))
    if save:
        layer.backward(dout, grads)
        wg = {k: v.clone() for k, v in grads.items()}
    assert torch.equal(layer.forward(x, x), want)
    if save:
        layer.backward(dout, grads)
        assert all(torch.equal(grads[k], wg[k]) for k in wg)


@pytest.mark.parametrize("save", ["rows", "codes"])
def test_sublayer_backward_twice(save):
    """What the backward pass reads outlives it: a second one gives the same
    bits."""
    _, layer, x, dout, grads = make_sublayer(70, 128, 264, "bf16", "silu", True, save)
    layer.forward(x, torch.empty_like(x))
    layer.backward(dout, grads)
    once = {k: v.clone() for k, v in grads.items()}
    layer.backward(dout, grads)
    assert all(torch.equal(grads[k], once[k]) for k in once)


# ------------------------------------------------ fp32 results hold 32 bits
# Bounds on the error's norm (tests/_bounds.py); an oracle with fewer bits
# anywhere in these sizes is outside of them (tests/test_bounds.py).
@pytest.mark.parametrize("m,n,k,parts,pad,route", FORWARD)
def test_linear_holds_32_bits(m, n, k, parts, pad, route):
    if route != "few":
        assert R.route(R.FORWARD, m, n, k, "f32", k % 8 == 0 and pad == 0) == route
    g = gen(m + n + k)
    a, w = mat(g, m, k, "f32", pad), mat(g, n, k, "f32", pad)
    desc = fs.linear_desc(m, n, k, "f32")
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR))
    out = Out(m, n, "f32", pad)
    fs.fs_linear(desc, a, w, None, None, out.view, wp)
    torch.cuda.synchronize()
    guard(ws, wp)
    assert rel(out.get(), f64(a) @ f64(w).T) <= B.product(k, parts)


@pytest.mark.parametrize("m,n,k,act,routes", BACKWARD)
def test_linear_backward_holds_32_bits(m, n, k, act, routes):
    for kind, size, width, route in ((R.INPUT, (m, k, n), k, routes[0]), (R.WEIGHT, (n, k, m), k, routes[1])):
        assert R.route(kind, *size, "f32", n % 8 == 0 and width % 8 == 0) == route
    g = gen(m + n + k)
    a, z, dout, w = mat(g, m, k, "f32"), mat(g, m, n, "f32"), mat(g, m, n, "f32"), mat(g, n, k, "f32")
    desc = fs.linear_desc(m, n, k, "f32", act)
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR_BACKWARD))
    da, dw, db = Out(m, k, "f32"), Out(n, k, "f32"), torch.full((n,), float("nan"), device=DEV)
    fs.fs_linear_backward(desc, dout, a, w, None if act == "none" else z, da.view, dw.view, db, wp)
    torch.cuda.synchronize()
    guard(ws, wp)
    wa, ww, wb, _ = O.linear_backward(f64(dout), f64(a), f64(w), f64(z), act)
    slope = 0 if act in ("none", "relu") else 2 * ACT
    assert rel(da.get(), wa) <= B.product(n) + slope
    assert rel(dw.get(), ww) <= B.product(m) + slope
    assert rel(f64(db), wb) <= B.product(m) + slope


@pytest.mark.parametrize("n,d,f,act", SUBLAYER)
def test_sublayer_holds_32_bits(n, d, f, act):
    p, layer, x, dout, grads = make_sublayer(n, d, f, "f32", act, True, "rows")
    out = layer.forward(x, torch.empty_like(x))
    layer.backward(dout, grads)
    torch.cuda.synchronize()
    want, wg = sublayer_oracle(f64(x), f64(dout), [f64(t) for t in p], act, True, lambda t: t, False)
    assert rel(f64(out), want) <= B.sublayer_forward(d, f)
    for k, v in grads.items():
        assert rel(f64(v), wg[k]) <= B.sublayer_backward(n, d, f), k


# -------------------------------------- a checkpoint and the rows it stands for
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,d", [(9, 77), (300, 1000), (5, 5120), (40, 9000), (3, 20001)])
def test_norm_backward_of_restored_rows(m, d, dtype):
    """Codes and the restored rows give the same bits."""
    g = gen(m + d)
    x, dy = mat(g, m, d, dtype), mat(g, m, d, dtype)
    c, back = fs.checkpoint_buffers(m, d), torch.empty((m, d), dtype=TORCH[dtype], device=DEV)
    fs.fs_checkpoint_fp8(CODE[dtype], m, d, x, *c)
    fs.fs_checkpoint_restore(CODE[dtype], m, d, *c, back)
    mean, rstd = x.float().mean(1), 1 / x.float().std(1)
    desc = fs.norm_desc(m, d, dtype)
    ws, wp = workspace(fs.fs_layer_norm_workspace(desc))
    got = []
    for saved in (c, back):
        dx, dg, db = Out(m, d, dtype), torch.empty((d,), device=DEV), torch.empty((d,), device=DEV)
        fs.fs_layer_norm_backward(desc, dy, saved, mean, rstd, None, None, dx.view, dg, db, wp)
        got.append([dx.get(), f64(dg), f64(db)])
    assert all(np.array_equal(p, q) for p, q in zip(*got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(9, 64, 72), (130, 40, 2048), (300, 520, 1000), (3000, 1000, 2000)])
def test_linear_backward_of_restored_rows(m, n, k, dtype):
    """The same for the linear where widths are whole chunks."""
    g = gen(m + n + k)
    a, z, dout, w = mat(g, m, k, dtype), mat(g, m, n, dtype), mat(g, m, n, dtype), mat(g, n, k, dtype)
    saved = []
    for t, cols in ((a, k), (z, n)):
        c, back = fs.checkpoint_buffers(m, cols), torch.empty((m, cols), dtype=TORCH[dtype], device=DEV)
        fs.fs_checkpoint_fp8(CODE[dtype], m, cols, t, *c)
        fs.fs_checkpoint_restore(CODE[dtype], m, cols, *c, back)
        saved.append((c, back))
    desc = fs.linear_desc(m, n, k, dtype, "gelu")
    ws, wp = workspace(fs.fs_linear_workspace(desc, L.FS_OP_LINEAR_BACKWARD))
    got = []
    for i in (0, 1):
        da, dw, db = Out(m, k, dtype), Out(n, k, dtype), torch.empty((n,), device=DEV)
        fs.fs_linear_backward(desc, dout, saved[0][i], w, saved[1][i], da.view, dw.view, db, wp)
        got.append([da.get(), dw.get(), f64(db)])
    assert all(np.array_equal(p, q) for p, q in zip(*got))
