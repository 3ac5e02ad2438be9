"""Norm + modulation and gate + residual + norm through the C-ABI against the float64 oracle.

The bounds (layer_helpers) count fp32 roundings up to each result's own rounding: half a step of bf16 (2^-8), of an
e4m3 code (2^-4) or of an int8 code (half a scale).
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_helpers as lh  # noqa: E402
from oracle import layer as ol  # noqa: E402
from oracle.quant import decode as ol_decode  # noqa: E402
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


def _cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _x(seed, rows, dim, fp32):
    x = lh.rows(seed, rows, dim)
    if fp32:
        return x, _cuda(x), abi.ISPA_FP32
    x = synth.bf16_round(x)
    return x, _cuda(x).to(torch.bfloat16), abi.ISPA_BF16


def _vectors(seed, rows, dim, per):
    """Six vectors a group, as one projection leaves them."""
    e = (0.3 * np.random.default_rng(seed).standard_normal((-(-rows // per), 6, dim))).astype(np.float32)
    return e, _cuda(e)


def _affine(seed, dim, on):
    if not on:
        return None, None
    g = np.random.default_rng(seed)
    return (1 + 0.1 * g.standard_normal(dim)).astype(np.float32), (0.1 * g.standard_normal(dim)).astype(np.float32)


def _out(rows, dim, fmt):
    """Buffers with a row behind the last that nothing may touch."""
    if fmt == "bf16":
        t = torch.full((rows + 1, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        return t, None, abi.rows_out(t)
    t = torch.full((rows + 1, dim), 77, dtype=torch.uint8 if fmt == "e4m3" else torch.int8, device="cuda")
    s = torch.full((rows + 1,), 7.0, device="cuda")
    return t, s, abi.rows_out(t, abi.ISPA_ROWS_E4M3 if fmt == "e4m3" else abi.ISPA_ROWS_I8, s)


def _check(t, s, rows, h, err, fmt):
    torch.cuda.synchronize()
    if fmt == "bf16":
        assert (t[rows] == 7.0).all()
        lh.assert_within(t[:rows].float().cpu().numpy(), h, (1 + lh.U_BF16) * err + lh.U_BF16 * np.abs(h) + 1e-45)
    else:
        assert (t[rows] == 77).all() and s[rows] == 7.0
        lh.check_codes(t[:rows].cpu().numpy(), s[:rows].cpu().numpy(), h, err, fmt)


# row lengths on both sides of every way a row is dealt to threads (a warp or a block a row, one to eight vectors a
# thread), and lengths that end inside a thread's vectors
DIMS = [8, 72, 256, 512, 520, 1024, 1536, 2048, 2056, 4096, 4104, 5120, 8192, 8200, 16384, 32768]


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("dim", DIMS)
def test_norm_modulate_row_lengths(dim, fp32):
    for rows, kind, fmt in [(3, ol.LAYER, "bf16"), (1, ol.RMS, "e4m3"), (5, ol.LAYER, "i8")]:
        _norm_case(rows, dim, fp32, kind, fmt, affine=rows != 1, per=2)


@pytest.mark.parametrize("dim", [8, 72, 512, 520, 1536, 2048])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "i8"])
def test_norm_modulate_many_rows(dim, fmt):
    for fp32, kind in [(False, ol.LAYER), (True, ol.RMS), (False, ol.NONE)]:
        _norm_case(1301, dim, fp32, kind, fmt, affine=True, per=97)


@pytest.mark.parametrize("vectors", ["none", "scale", "shift"])
def test_norm_modulate_without_some_vectors(vectors):
    _norm_case(33, 136, False, ol.LAYER, "bf16", affine=False, per=5, vectors=vectors)


def _norm_case(rows, dim, fp32, kind, fmt, affine, per, vectors="both"):
    x, xt, x_type = _x(rows + dim, rows, dim, fp32)
    w, b = _affine(1, dim, affine)
    e, et = _vectors(2, rows, dim, per)
    scale, shift = vectors in ("both", "scale"), vectors in ("both", "shift")
    t, s, out = _out(rows, dim, fmt)
    wt, bt = _cuda(w), _cuda(b)
    mod = None if vectors == "none" else abi.modulation(et[:, 1] if scale else None, et[:, 0] if shift else None, None,
                                                        6 * dim, per)
    abi.ispa_norm_modulate(xt, x_type, rows, dim, abi.norm(kind, EPS, wt, bt), mod, out)
    n = ol.norm(x, kind, EPS, w, b)
    sc, sh = e[:, 1] if scale else None, e[:, 0] if shift else None
    h = ol.modulate(n, sc, sh, per)
    _check(t, s, rows, h, lh.modulate_error(lh.norm_error(x, kind, EPS, w, b), n, sc, sh, per), fmt)


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("rows,dim", [(1, 8), (7, 264), (3, 1536), (1203, 1536), (640, 2048), (5, 5120), (2, 32768),
                                      (700, 2056), (613, 8192), (640, 4104)])
def test_gate_residual(rows, dim, fp32):
    for post, pre, fmt in [(ol.NONE, ol.LAYER, "bf16"), (ol.RMS, ol.RMS, "i8"), (ol.LAYER, ol.NONE, "bf16"),
                           (ol.RMS, None, None)]:
        _residual_case(rows, dim, fp32, post, pre, fmt, in_place=pre == ol.RMS)


# One to three rows of an SM and a team, a block's last row missing; few rows and one block an SM or two (2433 and more)
@pytest.mark.parametrize("rows,dim,fp32", [(153, 264, True), (305, 8192, True), (306, 5120, False), (457, 1536, False),
                                           (911, 1536, True), (2431, 512, False), (2443, 1024, True)])
def test_a_few_rows_an_sm(rows, dim, fp32):
    _norm_case(rows, dim, fp32, ol.LAYER, "i8", affine=True, per=59)
    _residual_case(rows, dim, fp32, ol.RMS, ol.LAYER, "bf16", in_place=True)


def test_gate_residual_without_norms_or_vectors():
    _residual_case(20, 128, True, None, None, None, in_place=True, gate=False)


def _residual_case(rows, dim, fp32, post, pre, fmt, in_place, gate=True):
    per = 13
    x, xt, x_type = _x(rows * 3 + dim, rows, dim, fp32)
    y = synth.bf16_round(lh.rows(rows + 9, rows, dim))
    yt = _cuda(y).to(torch.bfloat16)
    w, b = _affine(3, dim, post is not None)
    w2, b2 = _affine(4, dim, pre is not None)
    e, et = _vectors(5, rows, dim, per)
    wt, bt, w2t, b2t = _cuda(w), _cuda(b), _cuda(w2), _cuda(b2)
    xo = xt if in_place else torch.empty_like(xt)
    t = s = out = None
    if pre is not None:
        t, s, out = _out(rows, dim, fmt)
    abi.ispa_gate_residual(xt, x_type, yt, rows, dim, None if post is None else abi.norm(post, EPS, wt, bt), 0.75, -0.5,
                           abi.modulation(et[:, 4], et[:, 3], et[:, 2], 6 * dim, per) if gate else None, xo,
                           None if pre is None else abi.norm(pre, EPS, w2t, b2t), out)
    torch.cuda.synchronize()
    kind = ol.NONE if post is None else post
    n, g = ol.norm(y, kind, EPS, w, b), np.arange(rows) // per
    want = ol.gate_residual(x, n, 0.75, -0.5, e[:, 2] if gate else None, per)
    gv = np.abs(e[g, 2]) if gate else 1.0
    err = 0.5 * gv * lh.norm_error(y, kind, EPS, w, b) + 4 * lh.U * (np.abs(x) + 0.5 * gv * np.abs(n))
    half = lh.U if fp32 else lh.U_BF16
    got = xo.float().cpu().numpy()
    lh.assert_within(got, want, (1 + half) * err + half * np.abs(want) + 1e-45)
    if pre is not None:   # of x as it was stored
        n2 = ol.norm(got, pre, EPS, w2, b2)
        sc, sh = (e[:, 4], e[:, 3]) if gate else (None, None)      # without vectors there is no modulation either
        h = ol.modulate(n2, sc, sh, per)
        _check(t, s, rows, h, lh.modulate_error(lh.norm_error(got, pre, EPS, w2, b2), n2, sc, sh, per), fmt)


def test_one_pass_equals_the_two_calls():
    rows, dim = 1000, 1536
    x, xt, x_type = _x(1, rows, dim, False)
    yt = _cuda(lh.rows(2, rows, dim)).to(torch.bfloat16)
    et = _vectors(3, rows, dim, 100)[1]
    mod = abi.modulation(et[:, 1], et[:, 0], et[:, 2], 6 * dim, 100)
    xo, h, h2 = torch.empty_like(xt), torch.empty_like(xt), torch.empty_like(xt)
    pre = abi.norm(abi.ISPA_NORM_LAYER)
    abi.ispa_gate_residual(xt, x_type, yt, rows, dim, None, 1.0, 1.0, mod, xo, pre, abi.rows_out(h))
    abi.ispa_norm_modulate(xo, x_type, rows, dim, pre, mod, abi.rows_out(h2))
    torch.cuda.synchronize()
    # the same formula from the same stored x: a step of bf16 apart at most
    a, b = h.float(), h2.float()
    assert ((a - b).abs() <= 2.0 ** -7 * torch.maximum(a.abs(), b.abs()) + 1e-6).all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "i8"])
def test_rows_of_zeros(fmt):
    xt = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    t, s, out = _out(4, 64, fmt)
    for kind in (ol.NONE, ol.RMS, ol.LAYER):
        abi.ispa_norm_modulate(xt, abi.ISPA_BF16, 4, 64, abi.norm(kind), None, out)
        torch.cuda.synchronize()
        assert (t[:4] == 0).all() and (s is None or (s[:4] == 1).all())


# Codes of rows about 2^-117, below which a row counts as zeros; no norm, whose output is the row itself in fp32.
@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("rows,dim", [(8, 64), (8, 5120), (1304, 1536)])   # a block a row, and many rows
def test_rows_of_tiny_values(rows, dim, fmt):
    g = np.random.default_rng(dim)
    top = np.array([2.0 ** -116, 2.0 ** -117, 2.0 ** -117 * (1 - 2.0 ** -20), 2.0 ** -119, 2.0 ** -121, 2.0 ** -126,
                    2.0 ** -140, 0.0], np.float32)
    top = np.resize(top, rows)
    x = ((2 * g.random((rows, dim)) - 1) * 0.99 * top[:, None]).astype(np.float32)
    x[:, 5], x[:, 7], x[:, 9] = top, -top, 0
    t, s, out = _out(rows, dim, fmt)
    abi.ispa_norm_modulate(_cuda(x), abi.ISPA_FP32, rows, dim, abi.norm(ol.NONE), None, out)
    torch.cuda.synchronize()
    tiny = top < 2.0 ** -117
    largest = 448.0 if fmt == "e4m3" else 127.0
    want = np.where(tiny, np.float32(1), top / np.float32(largest)).astype(np.float32)
    assert np.array_equal(s[:rows].cpu().numpy(), want)
    codes = t[:rows].cpu().numpy()
    value = ol_decode(codes) if fmt == "e4m3" else codes.astype(np.float64)   # e4m3 has a negative zero
    assert not value[tiny].any()
    assert (value[~tiny, 5] == largest).all() and (value[~tiny, 7] == -largest).all() and not value[:, 9].any()


def test_constant_rows_and_a_large_offset():
    # variance 0: the norm is eps's alone; and an offset 2^12 times the spread leaves the spread as fp32 holds it
    rows, dim = 6, 1536
    g = np.random.default_rng(0)
    x = np.full((rows, dim), 3.0, np.float32)
    x[3:] = (4096.0 + g.standard_normal((3, dim))).astype(np.float32)
    t, s, out = _out(rows, dim, "bf16")
    abi.ispa_norm_modulate(_cuda(x), abi.ISPA_FP32, rows, dim, abi.norm(ol.LAYER, EPS), None, out)
    _check(t, s, rows, ol.norm(x, ol.LAYER, EPS), lh.norm_error(x, ol.LAYER, EPS, None, None), "bf16")


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "i8"])
def test_a_row_with_a_non_finite_value_stays_its_own(bad, fmt):
    rows, dim = 9, 264
    x, xt, x_type = _x(4, rows, dim, True)
    xt[4, 100] = bad
    t, s, out = _out(rows, dim, fmt)
    abi.ispa_norm_modulate(xt, x_type, rows, dim, abi.norm(ol.LAYER, EPS), None, out)
    torch.cuda.synchronize()
    keep = [r for r in range(rows) if r != 4]
    h, err = ol.norm(x, ol.LAYER, EPS), lh.norm_error(x, ol.LAYER, EPS, None, None)
    if fmt == "bf16":
        assert not torch.isfinite(t[4].float()).any()
        lh.assert_within(t[keep].float().cpu().numpy(), h[keep], (1 + lh.U_BF16) * err[keep] +
                         lh.U_BF16 * np.abs(h[keep]) + 1e-45)
    else:
        assert not torch.isfinite(s[4])
        lh.check_codes(t[keep].cpu().numpy(), s[keep].cpu().numpy(), h[keep], err[keep], fmt)


def test_one_vector_for_every_group():
    rows, dim = 40, 64
    x, xt, x_type = _x(11, rows, dim, True)
    v = (0.3 * np.random.default_rng(1).standard_normal((2, dim))).astype(np.float32)
    vt = _cuda(v)
    t, s, out = _out(rows, dim, "bf16")
    abi.ispa_norm_modulate(xt, x_type, rows, dim, abi.norm(ol.RMS, EPS), abi.modulation(vt[0], vt[1], None, 0, 7), out)
    n = ol.norm(x, ol.RMS, EPS)
    h = ol.modulate(n, v[:1], v[1:], rows)
    _check(t, s, rows, h, lh.modulate_error(lh.norm_error(x, ol.RMS, EPS, None, None), n, v[:1], v[1:], rows), "bf16")


def test_captured_and_on_a_side_stream():
    rows, dim = 500, 1536
    x, xt, x_type = _x(21, rows, dim, True)
    yt = _cuda(lh.rows(5, rows, dim)).to(torch.bfloat16)
    xo, h = torch.empty_like(xt), torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
    pre = abi.norm(abi.ISPA_NORM_RMS)

    def call(stream):
        abi.ispa_gate_residual(xt, x_type, yt, rows, dim, pre, 1.0, 1.0, None, xo, pre, abi.rows_out(h), stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    want = xo.clone(), h.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(torch.cuda.current_stream())
    for k in (1.0, 2.0):
        xt.copy_(_cuda(x) * k)
        xo.zero_()
        h.zero_()
        graph.replay()
        torch.cuda.synchronize()
        if k == 1.0:
            assert torch.equal(xo, want[0]) and torch.equal(h, want[1])
        else:
            assert not torch.equal(xo, want[0])
