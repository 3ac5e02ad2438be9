"""Inputs and bounds of the norm, rotary and int8 tests."""
from __future__ import annotations

import numpy as np

from oracle import layer as ol
from oracle import quant as oq

U = 2.0 ** -24        # half a step of fp32, relative
U_BF16 = 2.0 ** -8
# Roundings on the way from a row to a normed value: a thread adds up to 8 x 8 terms, 5 levels of shuffles and up to 16
# warps follow: a sum of n terms in that order is off by at most (64 + 5 + 16) U of the sum of their magnitudes.
# The root halves the square sum's share; division, root, products and additions take less than 16 more.
K_NORM = 64 + 5 + 16 + 16


def rows(seed, n, dim, offset=0.5):
    """Rows of a residual stream: an offset a row, some features far larger than the others."""
    g = np.random.default_rng(seed)
    big = 1.0 + 7.0 * (g.random(dim) > 0.97)
    return (g.standard_normal((n, dim)) * big + offset * g.standard_normal((n, 1))).astype(np.float32)


def norm_error(x, kind, eps, weight, bias):
    """Bound on |fp32 norm - exact norm| per element, before any rounding of the result."""
    x = np.asarray(x, np.float64)
    w = np.ones(x.shape[-1]) if weight is None else np.abs(np.asarray(weight, np.float64))
    b = np.zeros(x.shape[-1]) if bias is None else np.abs(np.asarray(bias, np.float64))
    if kind == ol.NONE:
        return K_NORM * U * (np.abs(x) * w + b)
    c = x - x.mean(-1, keepdims=True) if kind == ol.LAYER else x
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    # the mean is off by K U mean|x|; its square's share of the variance is second order
    size = (np.abs(c) + np.abs(x) + np.abs(x).mean(-1, keepdims=True)) * r
    return K_NORM * U * (size * w + b)


def modulate_error(err, n, scale, shift, rows_per_group):
    g = np.arange(n.shape[0]) // rows_per_group
    s = 1.0 + np.abs(np.asarray(scale, np.float64)[g]) if scale is not None else 1.0
    t = np.abs(np.asarray(shift, np.float64)[g]) if shift is not None else 0.0
    return err * s + 4 * U * (np.abs(n) * s + t)


def assert_within(got, want, bound, what=""):
    got = np.asarray(got, np.float64)
    assert np.isfinite(got).all(), what
    bad = np.abs(got - want) > bound
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / bound):.2f} bounds"


def check_codes(codes, scale, h, err, fmt):
    """Codes of the rows h (fp32 error err) in a format: the scale, then every value the codes stand for."""
    top = 448.0 if fmt == "e4m3" else 127.0
    amax = np.abs(h).max(-1)
    want = np.where(amax < 2.0 ** -117, 1.0, amax / top)
    # amax is off by at most the row's largest err; one division
    assert_within(scale, want, 2 * U * want + err.max(-1) / top + 1e-45, "scale")
    s = np.asarray(scale, np.float64)[:, None]
    if fmt == "e4m3":
        v = oq.decode(codes)
        half = np.maximum(2.0 ** -4 * np.abs(h), 2.0 ** -10 * s)
    else:
        v = np.asarray(codes, np.float64)
        half = 0.5 * s
    # the reciprocal and the product round before the code does: at most 4 U of the value
    assert_within(v * s, h, half * (1 + 8 * U) + err * (1 + 2.0 ** -4) + 8 * U * np.abs(h) + 1e-45, "codes")
