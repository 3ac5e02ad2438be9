"""Rotary positions with the q/k norm through the C-ABI against the float64 oracle.

Bound: half a step of bf16 (2^-8) of the result; the norm's fp32 roundings (layer_helpers.K_NORM); the angle: a fraction of a turn
cut to 2^-32 (2^-29.3 rad) and rounded to fp32 (pi 2^-24), the hardware sine and cosine (2^-21.19 on [-pi, pi]), the factor
and two products: less than 20 U of |u| + |v| in all.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_helpers as lh  # noqa: E402
from oracle import layer as ol  # noqa: E402
from paper_2607_00712_gb300 import abi, synth  # noqa: E402

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _steps(axis_pairs, **kw):
    steps, factor = [], 1.0
    for m in axis_pairs:
        if m:
            s, factor = abi.ispa_rope_steps(m, **kw)
            steps += s
    return steps, factor


def _device_steps(steps):
    return torch.from_numpy(np.array(steps, np.uint64).view(np.int64)).cuda()


def _weight(seed, heads, d, norm):
    if norm == abi.ISPA_QK_NORM_NONE:
        return None
    n = d if norm == abi.ISPA_QK_NORM_HEAD else heads * d
    return (1 + 0.2 * np.random.default_rng(seed).standard_normal(n)).astype(np.float32)


def _expected(x, heads, d, norm, w, angle, factor, half):
    """(result, bound) of one tensor, x [n][heads * d]."""
    n = x.shape[0]
    x = x.astype(np.float64)
    err = 0.0
    if norm == abi.ISPA_QK_NORM_TOKEN:
        v = ol.norm(x, ol.RMS, EPS, w)
        err = lh.norm_error(x, ol.RMS, EPS, w, None)
    elif norm == abi.ISPA_QK_NORM_HEAD:
        xh = x.reshape(n * heads, d)
        v, err = ol.norm(xh, ol.RMS, EPS, w), lh.norm_error(xh, ol.RMS, EPS, w, None)
    else:
        v = x
    v = v.reshape(n, heads, d)
    err = np.broadcast_to(np.asarray(err).reshape(v.shape) if np.ndim(err) else 0.0, v.shape)
    want = ol.rope(v, angle, factor, half)
    p = angle.shape[1]
    size = np.abs(v)
    both, eb = size.copy(), err.copy()
    a, b = (slice(0, p), slice(p, 2 * p)) if half else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    both[..., a] = both[..., b] = factor * (size[..., a] + size[..., b])
    eb[..., a] = eb[..., b] = factor * (err[..., a] + err[..., b])
    return want, lh.U_BF16 * np.abs(want) + (1 + lh.U_BF16) * (eb + 20 * lh.U * both) + 1e-45


def _case(n, heads, d, axis_pairs, layout, norm, pos0=0, pos=None, in_place=False, seed=0, **scaling):
    """heads: of q and k.  Both stand in rows of one fused projection."""
    g = np.random.default_rng(seed + n)
    width = (sum(heads) + heads[-1]) * d
    qkv = synth.bf16_round((g.standard_normal((n, width)) * (0.25 + np.abs(g.standard_normal(width)))).astype(np.float32))
    t = torch.from_numpy(qkv).cuda().to(torch.bfloat16)
    before = t.clone()
    steps, factor = _steps(axis_pairs, **scaling)
    st = _device_steps(steps)
    if pos is None:
        pos = g.integers(-50, 3000, (len(axis_pairs), n))
    pt = torch.from_numpy(np.asarray(pos).astype(np.int32)).cuda()
    rope = abi.rope(layout, d, axis_pairs, st, factor)
    rows, keep, at = [], [], 0
    for i, h in enumerate(heads):
        w = _weight(seed + i, h, d, norm)
        wt = None if w is None else torch.from_numpy(w).cuda()
        out = t[:, at:] if in_place else torch.full((n + 1, h, d), 7.0, dtype=torch.bfloat16, device="cuda")
        rows.append(abi.rope_rows(t[:, at:], out, h, width, width if in_place else h * d, norm, wt, EPS))
        keep.append((h, at, w, wt, out))
        at += h * d
    abi.ispa_rope_apply(rope, rows, pt, pos0, n)
    torch.cuda.synchronize()
    angle = ol.angles(pos, pos0, axis_pairs, steps)
    half = layout == abi.ISPA_ROPE_HALF
    for h, at, w, wt, out in keep:
        want, bound = _expected(qkv[:, at:at + h * d], h, d, norm, w, angle, factor, half)
        if in_place:
            got = t[:, at:at + h * d].reshape(n, h, d)
        else:
            got = out[:n]
            assert (out[n] == 7.0).all()   # a row behind the last
        lh.assert_within(got.float().cpu().numpy(), want, bound)
    rest = keep[-1][1] + keep[-1][0] * d
    assert torch.equal(t[:, rest:], before[:, rest:])     # the values of the fused rows
    if not in_place:
        assert torch.equal(t, before)


LAYOUTS = [abi.ISPA_ROPE_INTERLEAVED, abi.ISPA_ROPE_HALF]
NORMS = [abi.ISPA_QK_NORM_NONE, abi.ISPA_QK_NORM_HEAD, abi.ISPA_QK_NORM_TOKEN]


@pytest.mark.parametrize("norm", NORMS)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("n,heads,d", [(1, (12, 12), 128), (5, (3, 1), 64), (33, (8, 2), 96), (2, (40, 40), 128),
                                       (3, (7,), 256), (1300, (4, 4), 64), (700, (12, 3), 128), (2, (160, 40), 256),
                                       (1, (520, 8), 128), (3, (5, 5), 16)])
def test_shapes(n, heads, d, layout, norm):
    _case(n, heads, d, [d // 2], layout, norm)


# Many tokens: a team for each of an SM's tokens (one warp, several), rounds with one token a team in shared memory and with
# two, a last round that not all teams have, full heads and not; out of place and in place.
@pytest.mark.parametrize("norm", NORMS)
@pytest.mark.parametrize("n,heads,d,in_place", [(1820, (8, 8), 128, False), (1217, (24, 8), 128, True),
                                                (1001, (96, 24), 96, True), (460, (160, 40), 96, False),
                                                (6151, (6, 2), 64, True), (2129, (24, 24), 128, False)])
def test_many_tokens(n, heads, d, in_place, norm):
    _case(n, heads, d, [d // 2], LAYOUTS[n % 2], norm, in_place=in_place)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_part_of_the_head_passes(layout):
    for d, pairs in [(128, 32), (64, 8), (96, 24), (256, 8), (128, 20), (40, 4)]:
        _case(9, (4, 4), d, [pairs], layout, abi.ISPA_QK_NORM_HEAD)
        _case(9, (4, 4), d, [pairs], layout, abi.ISPA_QK_NORM_NONE)


def test_odd_numbers_of_pairs_side_by_side():
    for pairs in (1, 3, 21, 63):
        _case(6, (2, 2), 128, [pairs], abi.ISPA_ROPE_INTERLEAVED, abi.ISPA_QK_NORM_NONE)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_three_axes(layout):
    n = 200
    t = np.arange(n)
    _case(n, (12, 12), 128, [22, 21, 21], layout, abi.ISPA_QK_NORM_TOKEN, pos0=57, pos=[t // 60, t // 10 % 6, t % 10])
    _case(n, (2, 2), 64, [0, 16, 16], layout, abi.ISPA_QK_NORM_NONE, pos0=5, pos=[t, t // 10, t % 10])
    _case(n, (2, 2), 64, [16, 16], layout, abi.ISPA_QK_NORM_NONE, pos=[t // 10, t % 10])


def test_far_and_negative_positions():
    far = [[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1_000_003, 65_537]]
    for pos0 in (0, 2 ** 40 + 17, -(2 ** 45), 2 ** 63 - 1):
        _case(7, (2, 2), 128, [64], abi.ISPA_ROPE_INTERLEAVED, abi.ISPA_QK_NORM_NONE, pos0=pos0, pos=far)


@pytest.mark.parametrize("scaling", [1, 2, 3])
def test_scaled_frequencies(scaling):
    _case(40, (4, 4), 128, [64], abi.ISPA_ROPE_HALF, abi.ISPA_QK_NORM_HEAD, scaling=scaling, scale=8.0,
          trained_length=4096.0)


@pytest.mark.parametrize("norm", NORMS)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_in_place(layout, norm):
    _case(41, (12, 4), 128, [48], layout, norm, in_place=True)
    _case(1250, (6, 2), 64, [32], layout, norm, in_place=True)
    _case(2, (300, 4), 128, [64], layout, norm, in_place=True)


def test_turning_back():
    n, h, d = 50, 3, 128
    x = torch.randn(n, h, d, device="cuda").to(torch.bfloat16)
    st = _device_steps(_steps([64])[0])
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[None] * 977
    y, z = torch.empty_like(x), torch.empty_like(x)
    rope = abi.rope(abi.ISPA_ROPE_HALF, d, [64], st)
    abi.ispa_rope_apply(rope, [abi.rope_rows(x, y, h, h * d, h * d)], pos, 0, n)
    abi.ispa_rope_apply(rope, [abi.rope_rows(y, z, h, h * d, h * d)], -pos, 0, n)
    torch.cuda.synchronize()
    # two bf16 roundings, the first one's error turned back with the pair: of each of the pair's values half a step
    u, v = x[..., :64].float(), x[..., 64:].float()
    size = torch.hypot(u, v)
    bound = torch.cat([size, size], -1) * (2.0 ** -8 * 2.5)
    assert ((z.float() - x.float()).abs() <= bound + 1e-30).all()


def test_infinities_past_the_turned_features_pass_alone():
    n, h, d = 4, 2, 64
    for layout in LAYOUTS:
        x = torch.randn(n, h, d, device="cuda").to(torch.bfloat16)
        x[1, 0, 40] = float("inf")
        x[2, 1, 63] = float("-inf")
        y = torch.empty_like(x)
        rope = abi.rope(layout, d, [16], _device_steps(_steps([16])[0]))
        pos = torch.arange(n, dtype=torch.int32, device="cuda")[None]
        abi.ispa_rope_apply(rope, [abi.rope_rows(x, y, h, h * d, h * d)], pos, 0, n)
        torch.cuda.synchronize()
        assert torch.equal(y[..., 32:], x[..., 32:]) and torch.isfinite(y[..., :32].float()).all()


def test_a_non_finite_token_stays_its_own():
    n, h, d = 1250, 4, 64
    x = torch.randn(n, h, d, device="cuda").to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    rope = abi.rope(abi.ISPA_ROPE_INTERLEAVED, d, [32], _device_steps(_steps([32])[0]))
    want, got = torch.empty_like(x), torch.empty_like(x)
    for norm in NORMS:
        abi.ispa_rope_apply(rope, [abi.rope_rows(x, want, h, h * d, h * d, norm)], pos, 0, n)
        z = x.clone()
        z[17, 2, 5] = float("nan")
        abi.ispa_rope_apply(rope, [abi.rope_rows(z, got, h, h * d, h * d, norm)], pos, 0, n)
        torch.cuda.synchronize()
        keep = [t for t in range(n) if t != 17]
        assert torch.equal(got[keep], want[keep]) and torch.isnan(got[17].float()).any()


def test_captured_and_replayed_with_new_positions():
    n, h, d = 64, 4, 128
    x = torch.randn(n, h, d, device="cuda").to(torch.bfloat16)
    y, want = torch.empty_like(x), torch.empty_like(x)
    pos = torch.zeros(1, n, dtype=torch.int32, device="cuda")
    rope = abi.rope(abi.ISPA_ROPE_HALF, d, [64], _device_steps(_steps([64])[0]))
    rows = [abi.rope_rows(x, y, h, h * d, h * d)]
    abi.ispa_rope_apply(rope, rows, pos, 0, n)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        abi.ispa_rope_apply(rope, rows, pos, 0, n, torch.cuda.current_stream())
    for start in (3, 100_000):
        pos.copy_(torch.arange(start, start + n, dtype=torch.int32, device="cuda")[None])
        graph.replay()
        abi.ispa_rope_apply(rope, [abi.rope_rows(x, want, h, h * d, h * d)], pos, 0, n)
        torch.cuda.synchronize()
        assert torch.equal(y, want)
