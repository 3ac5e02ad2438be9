"""Every form of the int8 projection's, the norms' and the rotary kernels (form_cases.py) against plain 64-bit arithmetic.

The products are compared bit for bit.  The bounds of the others are layer_helpers' (fp32 roundings on the way to the
result's own), here in torch on the device, since the calls are large.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import form_cases  # noqa: E402
import layer_helpers as lh  # noqa: E402
import test_gpu_linear_i8 as ti  # noqa: E402
from oracle import layer as ol  # noqa: E402
from oracle import quant as oq  # noqa: E402
from paper_2607_00712_gb300 import abi  # noqa: E402

pytestmark = pytest.mark.gpu
EPS = 1e-6
F64 = torch.float64


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def _within(got, want, bound, what):
    got = got.to(F64)
    assert torch.isfinite(got).all(), what
    worst = ((got - want).abs() / bound.clamp_min(1e-300)).max().item()
    assert worst <= 1, f"{what}: {worst} bounds"


# ------------------------------------------------------------ int8 projection
@pytest.mark.parametrize("part", range(4))
def test_int8_projection(part):
    for T, D, N in form_cases.LINEAR[part::4]:
        ti._check(T, D, N, bias=T % 2 == 0, full=D % 32 == 0)


def test_pairs_give_the_same_bits_every_time():
    # both pair shapes, several waves, new codes each time; other calls run on a second stream meanwhile
    side = torch.cuda.Stream()
    for T, D, N in ((4680, 1536, 4608), (7519, 2432, 616), (105, 1168, 8)):
        g = _gen(T)
        a, w = (torch.randint(-128, 128, s, generator=g, device="cuda", dtype=torch.int8) for s in ((T, D), (N, D)))
        sa, sw = torch.rand(T, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
        out, want = (torch.empty(T, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        other = torch.empty_like(out)
        side.wait_stream(torch.cuda.current_stream())
        for turn in range(30):
            if turn % 10 == 0:
                a.copy_(a.roll(1, 0))
                abi.ispa_linear_i8(a, sa, w, sw, None, T, D, N, want)
            out.zero_()
            if turn % 3 == 0:
                abi.ispa_linear_i8(w, sw, w, sw, None, min(T, N), D, N, other, side)
            abi.ispa_linear_i8(a, sa, w, sw, None, T, D, N, out)
            assert torch.equal(out, want)
        # products of integers in fp64 are exact
        s = (a.to(F64) @ w.to(F64).t()).to(torch.float32)
        assert torch.equal(out, ((s * sa[:, None]) * sw).to(torch.bfloat16))
        torch.cuda.synchronize()
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


# ------------------------------------------------------------ norms
def _norm(x, kind, w, b):
    """(exact norm, bound on the fp32 one's error) of fp64 rows."""
    ones, zeros = torch.ones((), dtype=F64, device="cuda"), torch.zeros((), dtype=F64, device="cuda")
    wa, ba = ones if w is None else w.to(F64), zeros if b is None else b.to(F64)
    if kind == ol.NONE:
        return x * wa + ba, lh.K_NORM * lh.U * (x.abs() * wa.abs() + ba.abs())
    c = x - x.mean(1, keepdim=True) if kind == ol.LAYER else x
    r = 1.0 / ((c * c).mean(1, keepdim=True) + EPS).sqrt()
    size = (c.abs() + x.abs() + x.abs().mean(1, keepdim=True)) * r
    return c * r * wa + ba, lh.K_NORM * lh.U * (size * wa.abs() + ba.abs())


def _check_rows(t, s, h, err, fmt, what):
    """As layer_helpers.check_codes and the bf16 check of test_gpu_norm.py; the row behind the last is untouched."""
    n = h.shape[0]
    if fmt == "bf16":
        assert (t[n] == 7.0).all()
        _within(t[:n], h, (1 + lh.U_BF16) * err + lh.U_BF16 * h.abs() + 1e-45, what)
        return
    assert (t[n] == 77).all() and s[n] == 7.0
    top = 448.0 if fmt == "e4m3" else 127.0
    scale = h.abs().amax(1) / top
    _within(s[:n], scale, 2 * lh.U * scale + err.amax(1) / top + 1e-45, what + " scale")
    sc = s[:n].to(F64)[:, None]
    if fmt == "e4m3":
        value = torch.from_numpy(oq.DECODE_TABLE).cuda()[t[:n].long()]
        half = torch.maximum(2.0 ** -4 * h.abs(), 2.0 ** -10 * sc)
    else:
        value, half = t[:n].to(F64), 0.5 * sc
    _within(value * sc, h, half * (1 + 8 * lh.U) + err * (1 + 2.0 ** -4) + 8 * lh.U * h.abs() + 1e-45, what + " codes")


def _buffers(rows, dim, fmt):
    if fmt == "bf16":
        t = torch.full((rows + 1, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        return t, None, abi.rows_out(t)
    t = torch.full((rows + 1, dim), 77, dtype=torch.uint8 if fmt == "e4m3" else torch.int8, device="cuda")
    s = torch.full((rows + 1,), 7.0, device="cuda")
    return t, s, abi.rows_out(t, abi.ISPA_ROWS_E4M3 if fmt == "e4m3" else abi.ISPA_ROWS_I8, s)


def _norm_case(case, post, pre, fmt):
    rows, dim, fp32, residual, post_bias, modulated, per = case
    what = f"{case} {post} {pre} {fmt}"
    g = _gen(rows + dim)
    xt = torch.float32 if fp32 else torch.bfloat16
    x = (_normal(g, rows, dim) * (1 + 7 * (_normal(g, dim) > 2)) + _normal(g, rows, 1, std=0.5)).to(xt)
    e = _normal(g, -(-rows // per), 6, dim, std=0.3)
    group = torch.arange(rows, device="cuda") // per
    mod = abi.modulation(e[:, 1], e[:, 0], e[:, 2], 6 * dim, per) if modulated else None
    w, b = 1 + _normal(g, dim, std=0.1), _normal(g, dim, std=0.1)
    t, s, out = _buffers(rows, dim, fmt)
    x64 = x.to(F64)
    x_type = abi.ISPA_FP32 if fp32 else abi.ISPA_BF16
    if residual:
        y = _normal(g, rows, dim, dtype=torch.bfloat16)
        w2, b2 = 1 + _normal(g, dim, std=0.1), _normal(g, dim, std=0.1) if post_bias else None
        xo = torch.full((rows + 1, dim), 7.0, dtype=xt, device="cuda")
        abi.ispa_gate_residual(x, x_type, y, rows, dim, abi.norm(post, EPS, w2, b2), 0.75, -0.5, mod, xo,
                               abi.norm(pre, EPS, w, b), out)
        n, err = _norm(y.to(F64), post, w2, b2)
        gate = e[group, 2].to(F64) if modulated else 1.0
        want = 0.75 * x64 - 0.5 * gate * n
        size = np.abs(gate) if isinstance(gate, float) else gate.abs()
        err = 0.5 * size * err + 4 * lh.U * (x64.abs() + 0.5 * size * n.abs())
        half = lh.U if fp32 else lh.U_BF16
        assert (xo[rows] == 7.0).all()
        _within(xo[:rows], want, (1 + half) * err + half * want.abs() + 1e-45, what + " x")
        x64 = xo[:rows].to(F64)       # the next norm is of x as it is stored
    else:
        abi.ispa_norm_modulate(x, x_type, rows, dim, abi.norm(pre, EPS, w, b), mod, out)
    n, err = _norm(x64, pre, w, b)
    if modulated:
        scale, shift = e[group, 1].to(F64), e[group, 0].to(F64)
        err = err * (1 + scale.abs()) + 4 * lh.U * (n.abs() * (1 + scale.abs()) + shift.abs())
        n = n * (1 + scale) + shift
    _check_rows(t, s, n, err, fmt, what)


@pytest.mark.parametrize("part", range(6))
def test_norms(part):
    kinds, formats = [ol.LAYER, ol.RMS, ol.NONE], ["bf16", "i8", "e4m3"]
    for i, case in enumerate(form_cases.NORM[part::6]):
        _norm_case(case, kinds[(i + 1) % 3], kinds[i // 2 % 3], formats[(i + part) % 3])
        _norm_case(case, ol.LAYER, ol.LAYER, formats[(i + part + 1) % 3])
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


# ------------------------------------------------------------ rotary positions
def _rope_case(case, in_place):
    n, heads, norm, d, pairs, half = case
    g = _gen(n + d + pairs)
    width = (sum(heads) + heads[-1]) * d
    t = (_normal(g, n, width) * (0.25 + _normal(g, width).abs())).to(torch.bfloat16)
    before = t.clone()
    split = [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3] if pairs > 2 else [pairs]
    steps = [s for m in split for s in abi.ispa_rope_steps(m)[0]]
    st = torch.from_numpy(np.array(steps, np.uint64).view(np.int64)).cuda()
    pos = torch.randint(-50, 100_000, (len(split), n), generator=g, device="cuda", dtype=torch.int32)
    rope = abi.rope(abi.ISPA_ROPE_HALF if half else abi.ISPA_ROPE_INTERLEAVED, d, split, st, 1.25)
    rows, keep, at = [], [], 0
    for h in heads:
        w = None if norm == abi.ISPA_QK_NORM_NONE else \
            1 + _normal(g, d if norm == abi.ISPA_QK_NORM_HEAD else h * d, std=0.2)
        out = t[:, at:] if in_place else torch.full((n + 1, h, d), 7.0, dtype=torch.bfloat16, device="cuda")
        rows.append(abi.rope_rows(t[:, at:], out, h, width, width if in_place else h * d, norm, w, EPS))
        keep.append((h, at, w, out))
        at += h * d
    abi.ispa_rope_apply(rope, rows, pos, 57, n)
    # a fraction of a turn: 64-bit products, modulo 2^64
    axis = torch.tensor([a for a, m in enumerate(split) for _ in range(m)], device="cuda")
    at_pos = pos.to(torch.int64)[axis] + 57 * (axis == 0)[:, None]
    angle = ((at_pos * st[:, None]).to(F64) * (2 * np.pi / 2.0 ** 64)).t()[:, None]
    cos, sin = 1.25 * torch.cos(angle), 1.25 * torch.sin(angle)
    u, v = (slice(0, pairs), slice(pairs, 2 * pairs)) if half else (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2))
    for h, at, w, out in keep:
        x = before[:, at:at + h * d].to(F64)
        err = torch.zeros_like(x)
        if norm == abi.ISPA_QK_NORM_TOKEN:
            x, err = _norm(x, ol.RMS, w, None)
        elif norm == abi.ISPA_QK_NORM_HEAD:
            x, err = _norm(x.reshape(n * h, d), ol.RMS, w, None)
        x, err = x.reshape(n, h, d), err.reshape(n, h, d)
        want, size = x.clone(), x.abs()
        want[..., u], want[..., v] = x[..., u] * cos - x[..., v] * sin, x[..., u] * sin + x[..., v] * cos
        size[..., u] = size[..., v] = 1.25 * (x[..., u].abs() + x[..., v].abs())
        eb = err.clone()
        eb[..., u] = eb[..., v] = 1.25 * (err[..., u] + err[..., v])
        if in_place:
            got = t[:, at:at + h * d].reshape(n, h, d)
        else:
            got = out[:n]
            assert (out[n] == 7.0).all()
        _within(got, want, lh.U_BF16 * want.abs() + (1 + lh.U_BF16) * (eb + 20 * lh.U * size) + 1e-45, str(case))
    rest = sum(heads) * d
    assert torch.equal(t[:, rest:], before[:, rest:]) and (in_place or torch.equal(t, before))


@pytest.mark.parametrize("part", range(6))
def test_rotary_positions(part):
    for i, case in enumerate(form_cases.ROPE[part::6]):
        _rope_case(case, in_place=i % 2 == 1)
        if case[0] == 4680:
            _rope_case(case, in_place=i % 2 == 0)
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


# ------------------------------------------------------------ rows that are not like others, in every form of the norms
# a block a row; teams of one warp; of several; two blocks an SM
FORMS = [(9, 264), (700, 264), (700, 1536), (5000, 1536)]


def _special(rows, dim, seed, fp32):
    g = _gen(seed)
    x = _normal(g, rows, dim) + _normal(g, rows, 1, std=0.5)
    return x if fp32 else x.to(torch.bfloat16)


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("rows,dim", FORMS)
def test_zero_constant_and_offset_rows(rows, dim, fp32):
    x = _special(rows, dim, 1, fp32)
    x[0], x[2], x[rows - 1], x[rows // 2] = 0, 3.0, -0.3125, 0
    x[4] += 4096.0
    zeros = [r for r in (0, rows // 2) if not x[r].any()]      # of nine rows the middle one is the one with the offset
    for fmt in ("bf16", "e4m3", "i8"):
        for kind in (ol.LAYER, ol.RMS, ol.NONE):
            t, s, out = _buffers(rows, dim, fmt)
            abi.ispa_norm_modulate(x, abi.ISPA_FP32 if fp32 else abi.ISPA_BF16, rows, dim, abi.norm(kind, EPS), None,
                                   out)
            torch.cuda.synchronize()
            for z in zeros:
                assert not t[z].float().any() and (s is None or s[z] == 1)
            n, err = _norm(x.to(F64), kind, None, None)
            if fmt != "bf16":     # codes and scales of rows whose norm is zero are those of what rounding left
                live = (n.abs().amax(1) > 4 * err.amax(1)).nonzero()[:, 0]
                t, s, n, err = torch.cat([t[live], t[rows:]]), torch.cat([s[live], s[rows:]]), n[live], err[live]
            _check_rows(t, s, n, err, fmt, f"{kind}")


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf"), 3.0e38])
@pytest.mark.parametrize("rows,dim", FORMS)
def test_rows_that_are_not_finite_stay_their_own(rows, dim, bad):
    for fp32 in (False, True):
        x_type, xt = (abi.ISPA_FP32, torch.float32) if fp32 else (abi.ISPA_BF16, torch.bfloat16)
        x, y = _special(rows, dim, 2, fp32), _special(rows, dim, 3, False)
        row, yrow = rows // 2, rows - 2
        keep = torch.tensor([r for r in range(rows) if r not in (row, yrow)], device="cuda")
        got = []
        for clean in (True, False):
            xs, ys = x.clone(), y.clone()
            if not clean:
                xs[row, dim - 1] = bad
                ys[yrow, 5] = bad
            for fmt in ("bf16", "e4m3", "i8"):
                t, s, out = _buffers(rows, dim, fmt)
                abi.ispa_norm_modulate(xs, x_type, rows, dim, abi.norm(ol.LAYER, EPS), None, out)
                got.append((t, s, clean, fmt, (row,)))
                t, s, out = _buffers(rows, dim, fmt)
                xo = torch.empty(rows, dim, dtype=xt, device="cuda")
                abi.ispa_gate_residual(xs, x_type, ys, rows, dim, abi.norm(ol.LAYER, EPS), 1.0, 1.0, None, xo,
                                       abi.norm(ol.RMS, EPS), out)
                got.append((t, s, clean, fmt, (row, yrow)))
        torch.cuda.synchronize()
        for (t, s, *_), (tb, sb, _, fmt, rs) in zip(got[:6], got[6:]):
            assert torch.equal(t[keep], tb[keep]) and (s is None or torch.equal(s[keep], sb[keep]))
            if abs(bad) < float("inf"):
                continue          # finite: its squares are not, and the row is whatever fp32 makes of it
            for r in rs:
                assert not (torch.isfinite(tb[r].float()).all() if fmt == "bf16" else torch.isfinite(sb[r]))


@pytest.mark.parametrize("rows,dim", FORMS)
def test_one_vector_for_every_group(rows, dim):
    x = _special(rows, dim, 4, True)
    g = _gen(5)
    v = _normal(g, 3, dim, std=0.3)
    y = _special(rows, dim, 6, False)
    t, s, out = _buffers(rows, dim, "bf16")
    xo = torch.empty_like(x)
    abi.ispa_gate_residual(x, abi.ISPA_FP32, y, rows, dim, None, 1.0, 1.0, abi.modulation(v[0], v[1], v[2], 0, 11), xo,
                           abi.norm(ol.LAYER, EPS), out)
    want = x.to(F64) + v[2].to(F64) * y.to(F64)
    _within(xo, want, 8 * lh.U * (x.to(F64).abs() + (v[2].to(F64) * y.to(F64)).abs()), "x")
    n, err = _norm(xo.to(F64), ol.LAYER, None, None)
    err = err * (1 + v[0].to(F64).abs()) + 4 * lh.U * (n.abs() * (1 + v[0].to(F64).abs()) + v[1].to(F64).abs())
    _check_rows(t, s, n * (1 + v[0].to(F64)) + v[1].to(F64), err, "bf16", "h")
