"""What stands around the chunk attention in a DiT layer (oracle; test infrastructure only).

Paper basis: Sec. 2 takes the queries and keys of a layer as given (after their rotary positions) and Sec. 3.2
changes the output projection; the norms, the rotation and the residual between them are the transformer's own,
from their formulas:

  rms(v) = v / sqrt(mean(v^2) + eps) w + b;  layer(v) = (v - mean) / sqrt(var + eps) w + b
  h = norm(x) (1 + scale_g) + shift_g;       x <- x_scale x + y_scale gate_g post(y)
  rotary: pair (u, v) of a head -> f (u cos a - v sin a, u sin a + v cos a), a = 2 pi pos steps_i / 2^64

and a product of 8-bit integers with one scale per token and channel (Sec. 4 runs W8A8 linear layers):
  y[t, n] = (sum_k a[t, k] w[n, k]) a_scale[t] w_scale[n] + bias[n], the sum an exact integer.

All in float64 but the last, whose steps after the sum are the fp32 ones that the library documents.
"""
from __future__ import annotations

import numpy as np

NONE, RMS, LAYER = 0, 1, 2


def norm(x, kind, eps, weight=None, bias=None):
    x = np.asarray(x, np.float64)
    if kind == LAYER:
        x = x - x.mean(-1, keepdims=True)
    if kind != NONE:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if weight is not None:
        x = x * np.asarray(weight, np.float64)
    return x if bias is None else x + np.asarray(bias, np.float64)


def modulate(n, scale=None, shift=None, rows_per_group=1):
    """n [rows][dim]; scale, shift [groups][dim]."""
    g = np.arange(n.shape[0]) // rows_per_group
    if scale is not None:
        n = n * (1.0 + np.asarray(scale, np.float64)[g])
    return n if shift is None else n + np.asarray(shift, np.float64)[g]


def gate_residual(x, y, x_scale, y_scale, gate=None, rows_per_group=1):
    """y already normed."""
    y = np.asarray(y, np.float64)
    if gate is not None:
        y = y * np.asarray(gate, np.float64)[np.arange(y.shape[0]) // rows_per_group]
    return x_scale * np.asarray(x, np.float64) + y_scale * y


def angles(pos, pos0, axis_pairs, steps):
    """Radians [n][pairs] in [-pi, pi), the product reduced exactly: pos int [axes][n], steps a list of ints."""
    axis = [a for a, m in enumerate(axis_pairs) for _ in range(m)]
    out = np.empty((len(pos[0]), len(axis)))
    for i, a in enumerate(axis):
        for t, p in enumerate(pos[a]):
            f = (int(p) + (pos0 if a == 0 else 0)) * int(steps[i]) % (1 << 64)
            out[t, i] = 2 * np.pi * ((f - (1 << 64) if f >= 1 << 63 else f) / 2.0 ** 64)
    return out


def rope(x, angle, factor, half):
    """x [n][H][d] float64, angle [n][pairs]."""
    p = angle.shape[1]
    c, s = factor * np.cos(angle)[:, None], factor * np.sin(angle)[:, None]
    out = np.array(x, np.float64)
    u, v = (slice(0, p), slice(p, 2 * p)) if half else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    out[..., u] = x[..., u] * c - x[..., v] * s
    out[..., v] = x[..., u] * s + x[..., v] * c
    return out


def frequencies(n, base, scaling="none", scale=1.0, trained=1.0, low=1.0, high=32.0):
    """Radians per position of n pairs (float64)."""
    i = np.arange(n)
    if scaling == "linear" or (scaling == "base" and n == 1):
        return base ** (-i / n) / scale
    if scaling == "base":
        return (base * scale ** (n / (n - 1))) ** (-i / n)
    w = np.float64(base) ** (-i / n)
    if scaling == "parts":
        keep = np.clip((trained * w / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
        w = w * (keep + (1.0 - keep) / scale)
    return w


def quantize_i8(x):
    """fp32 rows -> (int8 codes, fp32 scales), each step in fp32; a row below 2^-117 counts as zeros."""
    x = np.asarray(x, np.float32)
    amax = np.abs(x).max(-1)
    zero = amax < 2.0 ** -117
    safe = np.where(zero, np.float32(1), amax).astype(np.float32)
    inv = np.where(zero, np.float32(1), np.float32(127) / safe).astype(np.float32)
    scale = np.where(zero, np.float32(1), safe / np.float32(127)).astype(np.float32)
    return np.rint(x * inv[:, None]).astype(np.int8), scale


def round_bf16(x):
    """fp32 -> nearest bf16 (ties to even), as fp32."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return r.astype(np.uint32).view(np.float32).reshape(np.shape(x))


def linear_i8(a, a_scale, w, w_scale, bias=None):
    """a int8 [T][D], w int8 [N][D] -> fp32 [T][N] holding the bf16 results."""
    # products and sums below 2^53 are exact in float64
    s = (np.asarray(a, np.float64) @ np.asarray(w, np.float64).T).astype(np.int64).astype(np.float32)
    y = (s * np.asarray(a_scale, np.float32)[:, None]).astype(np.float32)
    y = (y * np.asarray(w_scale, np.float32)).astype(np.float32)
    if bias is not None:
        y = (y + np.asarray(bias, np.float32)).astype(np.float32)
    return round_bf16(y)
