"""Bounds on the relative error (2-norm over all outputs) of fp32 results, from
the roundings that fp32 sums make, u = 2^-24 each at most.

A sum of K products of independent random signs: the partial sum after j of
them has sqrt(j / K) of the result's norm, each add errs by at most u of its
partial sum, and the errors' norms add up to at most (2 / 3) K u, whatever
their signs; the products' own errors, u / sqrt(K) of the norm each, to
sqrt(K) u.  With the terms dealt to p sums of their own, added at the end in a
tree, each add's partial sum is that of its part: K / sqrt(p) in place of K.
8 u more for that tree and the store."""

import math

import numpy as np

U = 2.0 ** -24

# ---- the sizes of the tests
# tokens, outputs, inputs, parts of the sum (the few-token kernel's lanes),
# row padding, kernel
FORWARD = [(1, 300, 4096, 64, 0, "few"), (2, 40, 2048, 64, 0, "few"), (130, 72, 1000, 1, 0, "mid1"),
           (512, 1408, 2048, 1, 0, "mid3"), (200, 300, 2048, 1, 0, "any+slices"), (512, 1408, 2048, 1, 1, "any+slices"),
           (1000, 1000, 2047, 1, 0, "any")]
# tokens, outputs, inputs, act, kernels of da and dw (one launch for two "any"
# of few tiles)
BACKWARD = [(512, 1408, 2048, "relu", ("any", "any")), (300, 1001, 1409, "none", ("any+slices", "any")),
            (1000, 1992, 520, "silu", ("any+slices", "any+slices")), (2047, 1999, 1024, "none", ("any", "any"))]
# tokens, hidden, ffn, act (smooth ones: a z next to 0 may have another sign in
# fp32, which relu's slope turns into an error of its whole gradient)
SUBLAYER = [(70, 96, 264, "silu"), (600, 128, 320, "gelu")]


def rel(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def product(K, parts=1):
    return (K / math.sqrt(parts) + math.sqrt(K) + 8) * U


def saved_z(d):
    """The norm (a mean and a variance of at most 54 adds in turn) and the
    product over d.  A matrix of random signs passes on an error's norm by at
    most twice its mean gain."""
    return 2 * 2 * (54 + 8) * U + product(d)


# (the activations err by at most 2^-20 of their values; silu's and gelu's
# values and slopes have at least 0.55 of the norm of a pre-activation of norm
# 1, slopes are at most 1.13, their own slopes 0.8)
def sublayer_forward(d, f):
    return 2 * (1.13 / 0.55 * saved_z(d) + 2.0 ** -20) + product(f)


def sublayer_backward(n, d, f):
    """The largest of the gradients' bounds: du from dout over d; dz with the
    slopes' errors; products over f or the n tokens; the norm's three terms."""
    dz = product(d) + 2.0 ** -20 + 0.8 / 0.55 * saved_z(d)
    return 3 * (2 * dz + product(max(f, n)) + 2 * (54 + 8) * U)
