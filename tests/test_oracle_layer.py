"""Pins of the layer oracle (norms, rotation, int8 product): invariants and brute force on tiny inputs."""
import numpy as np
import pytest

from oracle import layer as ol


def test_norms_have_the_moments_they_should():
    x = np.random.default_rng(0).standard_normal((7, 40)) * 3 + 2
    n = ol.norm(x, ol.LAYER, 0.0)
    assert np.allclose(n.mean(1), 0, atol=1e-12) and np.allclose((n * n).mean(1), 1)
    assert np.allclose((ol.norm(x, ol.RMS, 0.0) ** 2).mean(1), 1)
    assert np.array_equal(ol.norm(x, ol.NONE, 1e-6), x)
    w, b = np.arange(40.0), np.ones(40)
    assert np.allclose(ol.norm(x, ol.LAYER, 0.0, w, b), n * w + 1)


def test_modulation_goes_by_groups_of_rows():
    n = np.ones((5, 3))
    scale, shift = np.array([[1.0] * 3, [2.0] * 3]), np.array([[10.0] * 3, [20.0] * 3])
    assert ol.modulate(n, scale, shift, 3)[:, 0].tolist() == [12, 12, 12, 23, 23]
    assert ol.gate_residual(n, n, 2.0, 3.0, scale, 3)[:, 0].tolist() == [5, 5, 5, 8, 8]


@pytest.mark.parametrize("half", [False, True])
def test_rotation_is_a_rotation(half):
    g = np.random.default_rng(1)
    x, y = g.standard_normal((2, 6, 2, 16))
    a = g.uniform(-np.pi, np.pi, (6, 6))
    z = ol.rope(x, a, 1.0, half)
    assert np.allclose((z ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.array_equal(z[..., 12:], x[..., 12:])
    assert np.allclose(ol.rope(z, -a, 1.0, half), x)
    # dot products go by the difference of the angles alone
    b = a + 0.7
    assert np.allclose((ol.rope(x, a, 1.0, half) * ol.rope(y, b, 1.0, half)).sum(-1),
                       (x * ol.rope(y, np.full_like(a, 0.7), 1.0, half)).sum(-1))


def test_angles_of_far_positions_lose_nothing():
    step = 2 ** 64 // 10 + 1                # 10 steps are a turn and 4 2^-64 of one
    a = ol.angles([[0, 1, 10, 10 ** 10, -3]], 0, [1], [step])[:, 0] / (2 * np.pi)
    assert np.allclose(a, [0, 0.1, 0, 0, -0.3], atol=1e-9)
    assert a[3] == pytest.approx(4e9 / 2.0 ** 64, rel=1e-12)
    assert np.allclose(ol.angles([[5]], 7, [1], [step]), ol.angles([[12]], 0, [1], [step]))


def test_int8_codes_and_product():
    x = np.array([[1.0, -2.0, 0.5], [0, 0, 0]], np.float32)
    q, s = ol.quantize_i8(x)
    assert q.tolist() == [[64, -127, 32], [0, 0, 0]] and s[1] == 1      # 63.5 goes to the even 64, 31.75 to 32
    a = np.array([[1, -128], [127, 3]], np.int8)
    w = np.array([[-128, 127], [0, 1], [2, 2]], np.int8)
    one = np.ones(3, np.float32)
    want = ol.round_bf16((a.astype(np.int64) @ w.astype(np.int64).T).astype(np.float32))
    assert np.array_equal(ol.linear_i8(a, one[:2], w, one), want)
    assert np.array_equal(ol.round_bf16(np.float32([1 + 2 ** -8, 1 + 3 * 2 ** -8])), [1.0, 1 + 2 ** -6])
