"""The dense sublayer's operators in fp64 (numpy): the linear with bias,
activation and residual, layer norm, their backward passes, and 8-bit
checkpoints of activations.

Section 4.1's far-skip window runs the next layer's dense computation; these are
its parts, from their definitions.
"""

import math

import numpy as np
import torch

BLOCK = 32
MIN_EXP, MAX_EXP = -117, 119


def phi(z):
    """The normal distribution function."""
    return 0.5 * torch.erfc(torch.from_numpy(np.ascontiguousarray(-z / math.sqrt(2.0)))).numpy()


def _logistic(z):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z))


def act(z, name):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "gelu":
        return z * phi(z)
    if name == "silu":
        return z * _logistic(z)
    return z


def act_slope(z, name):
    if name == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if name == "gelu":
        return phi(z) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = _logistic(z)
        return s + z * s * (1 - s)
    return np.ones_like(z)


def linear(a, w, bias=None, residual=None, name="none"):
    """(z, out) of z = a w^T + bias, out = act(z) + residual."""
    z = a @ w.T
    if bias is not None:
        z = z + bias
    out = act(z, name)
    return z, out if residual is None else out + residual


def linear_backward(dout, a, w, z=None, name="none"):
    """da, dw, dbias and dz (none of them rounded)."""
    dz = dout if name == "none" else dout * act_slope(z, name)
    return dz @ w, dz.T @ a, dz.sum(0), dz


def layer_norm(s, gamma=None, beta=None, center=True, eps=1e-5):
    """y, mean, rstd of the rows of s."""
    mean = s.mean(1, keepdims=True) if center else np.zeros((s.shape[0], 1))
    rstd = 1.0 / np.sqrt(((s - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (s - mean) * rstd
    if gamma is not None:
        y = y * gamma
    if beta is not None:
        y = y + beta
    return y, mean[:, 0], rstd[:, 0]


def layer_norm_backward(dy, s, mean, rstd, gamma=None, dres=None, center=True):
    """dx, dgamma, dbeta."""
    h = (s - mean[:, None]) * rstd[:, None]
    u = dy if gamma is None else dy * gamma
    dx = u - h * (u * h).mean(1, keepdims=True)
    if center:
        dx = dx - u.mean(1, keepdims=True)
    dx = dx * rstd[:, None]
    if dres is not None:
        dx = dx + dres
    return dx, (dy * h).sum(0), dy.sum(0)


def checkpoint(x):
    """Codes [rows, cols] and scale bytes [rows, ceil(cols / 32)] of a
    checkpoint, by search over the 127 finite E4M3 magnitudes."""
    rows, cols = x.shape
    nb = (cols + BLOCK - 1) // BLOCK
    grid = e4m3_values(np.arange(127))
    codes = np.zeros((rows, cols), np.uint8)
    scales = np.zeros((rows, nb), np.uint8)
    for b in range(nb):
        blk = x[:, b * BLOCK:(b + 1) * BLOCK]
        amax = np.abs(blk).max(1)
        for r in range(rows):
            if not np.isfinite(amax[r]):
                scales[r, b] = 255
                codes[r, b * BLOCK:(b + 1) * BLOCK] = 0x7F
                continue
            e = MIN_EXP
            while e < MAX_EXP and amax[r] > math.ldexp(448.0, e):
                e += 1
            v = np.minimum(np.abs(blk[r]) * math.ldexp(1.0, -e), 448.0)
            lo = np.clip(np.searchsorted(grid, v, side="right") - 1, 0, 126)
            hi = np.minimum(lo + 1, 126)
            dl, dh = v - grid[lo], grid[hi] - v
            pick = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
            codes[r, b * BLOCK:(b + 1) * BLOCK] = pick + np.where(np.signbit(blk[r]), 128, 0)
            scales[r, b] = e + 127
    return codes, scales


def e4m3_values(codes):
    """fp64 values of E4M3 codes (0x7F and 0xFF: NaN)."""
    c = np.asarray(codes).astype(np.int64)
    field, man = (c >> 3) & 15, c & 7
    mag = np.where(field == 0, man * 2.0 ** -9, (8 + man) * 2.0 ** (field - 10.0))
    mag = np.where((c & 127) == 127, np.nan, mag)
    return np.where(c >= 128, -mag, mag)


def restore(codes, scales):
    """The values a checkpoint stands for."""
    cols = codes.shape[1]
    e = np.repeat(scales.astype(np.int64), BLOCK, axis=1)[:, :cols] - 127
    return e4m3_values(codes) * 2.0 ** e.astype(np.float64)
