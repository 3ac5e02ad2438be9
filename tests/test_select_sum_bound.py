"""The bound on what the selection's query sums lose, against exact sums: a restatement of their order and roundings.

A thread adds 2^-7 of its rows as a pair (TwoSum, the residues added in fp32); the threads' pairs are added alike, and at
the end hi becomes the rounded sum.  Claimed: hi + lo is within 2^-32 of the largest |2^-7 q|, and |lo| at most half a
step of hi.
"""
from fractions import Fraction

import numpy as np
import pytest

F = np.float32


def _two_sum(hi, lo, x):
    s = hi + x
    t = s - hi
    return s, lo + ((hi - (s - t)) + (x - t))


def _pair_sum(q, rows):
    """q fp32 [n][columns], of bf16 values; `rows` threads side by side."""
    n = len(q)
    a = b = np.zeros(q.shape[1], F)
    parts = []
    for r in range(rows):
        hi = lo = np.zeros(q.shape[1], F)
        for i in range(r, n, rows):
            hi, lo = _two_sum(hi, lo, q[i] * F(2.0 ** -7))
        parts.append((hi, lo))
    for hi, lo in parts[:n]:
        a, b = _two_sum(a, b, hi)
        b = b + lo
    return _two_sum(a, np.zeros_like(a), b)


def _bf16(x):
    return (np.asarray(x, F).view(np.uint32) & np.uint32(0xffff0000)).view(F)


@pytest.mark.parametrize("rows", [16, 32])
@pytest.mark.parametrize("kind", ["normal", "cancel", "pairs", "spread", "one size", "tiny", "largest"])
def test_sums_of_pairs(kind, rows):
    g = np.random.default_rng(rows)
    q = g.standard_normal((128, 40))
    if kind == "cancel":
        q[:2] = 2.0 ** g.integers(0, 60, 40)
        q[1] *= -1
        q = q[g.permutation(128)]
    elif kind == "pairs":
        q *= 2.0 ** g.integers(0, 40, (128, 40))
        q[64:] = -q[:64]
        q[5] = 1.0
        q = q[g.permutation(128)]
    elif kind == "spread":
        q *= 2.0 ** g.integers(-40, 40, (128, 40))
    elif kind == "one size":
        q = 1 + np.abs(q) * 2.0 ** -8
    elif kind == "tiny":
        q *= 2.0 ** -120
    elif kind == "largest":
        q = np.sign(q) * 3.3895314e38
        q[::3] = g.standard_normal((43, 40))
    q = _bf16(q)
    hi, lo = _pair_sum(q, rows)
    assert np.isfinite(hi).all()
    assert (np.abs(lo) <= np.spacing(np.abs(hi)) / 2).all()
    for c in range(q.shape[1]):
        exact = sum(Fraction(float(x)) for x in q[:, c]) / 128
        most = Fraction(float(np.abs(q[:, c]).max())) / 128
        assert abs(Fraction(float(hi[c])) + Fraction(float(lo[c])) - exact) <= most / 2 ** 32
