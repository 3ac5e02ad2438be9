"""Norm, rotary and int8 entry points on the host (no GPU): struct layouts, refusals, frequencies."""
import ctypes
import math
import os
import subprocess
import tempfile

import numpy as np
import pytest

from oracle import layer as ol
from paper_2607_00712_gb300 import abi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_00712_gb300.build import build_library
    build_library()


def test_struct_layouts_match_the_header():
    structs = {"ispa_norm": abi.Norm, "ispa_modulation": abi.Modulation, "ispa_rows_out": abi.RowsOut,
               "ispa_rope": abi.Rope, "ispa_rope_rows": abi.RopeRows, "ispa_rope_frequencies": abi.RopeFrequencies}
    lines = []
    for name, t in structs.items():
        lines.append(f'printf("%zu ", sizeof({name}));')
        lines += [f'printf("%zu ", offsetof({name}, {f[0]}));' for f in t._fields_]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "ispa.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n"
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
        open(c, "w").write(src)
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), c, "-o", exe], check=True)
        got = list(map(int, subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()))
    want = []
    for t in structs.values():
        want += [ctypes.sizeof(t)] + [getattr(t, f[0]).offset for f in t._fields_]
    assert got == want


def _status(call):
    try:
        call()
    except abi.IspaError as e:
        return e.status
    return abi.ISPA_OK


BAD, UNSUP = abi.ISPA_ERR_INVALID_ARG, abi.ISPA_ERR_UNSUPPORTED


def test_norm_refusals():
    good = abi.norm(abi.ISPA_NORM_RMS)
    out = abi.rows_out(16)

    def call(x=16, x_type=0, rows=2, dim=64, norm=good, mod=None, out=out):
        return _status(lambda: abi.ispa_norm_modulate(x, x_type, rows, dim, norm, mod, out))

    assert call(x=None) == BAD and call(x=24) == BAD
    assert call(x_type=2) == BAD and call(x_type=-1) == BAD
    assert call(rows=0) == BAD and call(rows=-3) == BAD and call(dim=0) == BAD
    assert call(rows=2 ** 31) == UNSUP and call(dim=60) == UNSUP and call(dim=32776) == UNSUP
    assert call(norm=None) == BAD and call(out=None) == BAD
    assert call(norm=abi.norm(3)) == BAD and call(norm=abi.norm(-1)) == BAD
    for eps in (-1e-6, math.nan, math.inf):
        assert call(norm=abi.norm(1, eps)) == BAD
    assert call(norm=abi.norm(1, 1e-6, 24)) == BAD and call(norm=abi.norm(1, 1e-6, None, 20)) == BAD
    assert call(out=abi.rows_out(None)) == BAD and call(out=abi.rows_out(24)) == BAD
    assert call(out=abi.rows_out(16, 3, 16)) == BAD and call(out=abi.rows_out(16, abi.ISPA_ROWS_I8, 18)) == BAD
    assert call(out=abi.rows_out(16, abi.ISPA_ROWS_E4M3)) == BAD and call(out=abi.rows_out(16, abi.ISPA_ROWS_I8)) == BAD
    for mod in (abi.modulation(16, 16, None, 64, 0), abi.modulation(16, 16, None, -64, 1),
                abi.modulation(16, 16, None, 66, 1), abi.modulation(20, 16, None, 64, 1),
                abi.modulation(16, 20, None, 64, 1), abi.modulation(16, 16, 8, 64, 1)):
        assert call(mod=mod) == BAD


def test_residual_refusals():
    pre, out = abi.norm(abi.ISPA_NORM_LAYER), abi.rows_out(16)

    def call(x=16, y=16, rows=2, dim=64, post=None, a=1.0, b=1.0, x_out=16, pre=pre, out=out):
        return _status(lambda: abi.ispa_gate_residual(x, 0, y, rows, dim, post, a, b, None, x_out, pre, out))

    assert call(x=None) == BAD and call(y=None) == BAD and call(y=24) == BAD
    assert call(x_out=None) == BAD and call(x_out=24) == BAD
    assert call(pre=None) == BAD and call(out=None) == BAD        # both or neither
    assert call(a=math.nan) == BAD and call(b=math.inf) == BAD
    assert call(rows=0) == BAD and call(dim=4) == UNSUP
    assert call(post=abi.norm(7)) == BAD


def test_linear_i8_refusals():
    def call(a=16, sa=16, w=16, sw=16, bias=None, T=10, D=64, N=64, out=16):
        return _status(lambda: abi.ispa_linear_i8(a, sa, w, sw, bias, T, D, N, out))

    assert call(a=None) == BAD and call(a=24) == BAD and call(w=None) == BAD and call(w=8) == BAD
    assert call(sa=None) == BAD and call(sw=None) == BAD and call(out=None) == BAD and call(out=24) == BAD
    assert call(T=2 ** 31 - 1024) == BAD and call(N=2 ** 31 - 1024) == BAD
    assert call(T=0) == BAD and call(T=2 ** 31) == BAD and call(D=0) == BAD and call(N=0) == BAD
    assert call(D=72) == UNSUP and call(N=36) == UNSUP and call(D=131072) == UNSUP
    assert _status(lambda: abi.ispa_quantize_rows_i8(16, 10, 24, 16, 16)) == UNSUP
    assert _status(lambda: abi.ispa_quantize_rows_i8(None, 10, 32, 16, 16)) == BAD
    assert _status(lambda: abi.ispa_quantize_rows_i8(16, 0, 32, 16, 16)) == BAD
    assert _status(lambda: abi.ispa_quantize_weight_i8(16, None, 24, 32, 16, 16)) == UNSUP
    assert _status(lambda: abi.ispa_quantize_weight_i8(16, None, 32, 0, 16, 16)) == BAD
    assert _status(lambda: abi.ispa_quantize_weight_i8(16, None, 16, 2097121, 16, 16)) == UNSUP
    assert _status(lambda: abi.ispa_quantize_weight_i8(16, None, 131072, 16, 16, 16)) == UNSUP
    # fp32 arrays off their four bytes
    assert call(sa=18) == BAD and call(sw=17) == BAD and call(bias=22) == BAD
    assert _status(lambda: abi.ispa_quantize_rows_i8(16, 10, 32, 16, 18)) == BAD
    for W, dW, s in ((18, None, 16), (16, 18, 16), (16, None, 18)):
        assert _status(lambda: abi.ispa_quantize_weight_i8(W, dW, 32, 32, 16, s)) == BAD


def test_rope_refusals():
    rope = abi.rope(0, 64, [32], 16)
    rows = abi.rope_rows(16, 16, 2, 128, 128)

    def call(rope=rope, rows=(rows,), pos=16, n=3):
        return _status(lambda: abi.ispa_rope_apply(rope, list(rows), pos, 0, n))

    assert call(pos=None) == BAD and call(pos=18) == BAD and call(n=0) == BAD and call(n=2 ** 30) == UNSUP
    assert call(rows=()) == BAD and call(rows=(rows, rows, rows)) == BAD
    assert call(abi.rope(2, 64, [32], 16)) == BAD and call(abi.rope(0, 64, [32], None)) == BAD
    assert call(abi.rope(0, 64, [32], 20)) == BAD
    assert call(abi.rope(0, 64, [], 16)) == BAD and call(abi.rope(0, 64, [0, 0], 16)) == BAD
    assert call(abi.rope(0, 64, [33, -1], 16)) == BAD and call(abi.rope(0, 64, [33], 16)) == UNSUP
    four = abi.rope(0, 64, [8, 8, 8], 16)
    four.n_axes = 4
    assert call(four) == BAD
    assert call(abi.rope(0, 64, [32], 16, math.nan)) == BAD
    assert call(abi.rope(1, 64, [14], 16)) == UNSUP               # half layout: pairs a multiple of 4
    assert call(abi.rope(0, 60, [16], 16), [abi.rope_rows(16, 16, 2, 128, 128)]) == UNSUP
    assert call(abi.rope(0, 264, [16], 16), [abi.rope_rows(16, 16, 2, 528, 528)]) == UNSUP
    for r in (abi.rope_rows(None, 16, 2, 128, 128), abi.rope_rows(16, 24, 2, 128, 128), abi.rope_rows(16, 32, 0, 128, 128),
              abi.rope_rows(16, 32, 2, 120, 128), abi.rope_rows(16, 32, 2, 128, 120), abi.rope_rows(16, 32, 2, 132, 128),
              abi.rope_rows(16, 16, 2, 128, 136), abi.rope_rows(16, 32, 2, 128, 128, 3),
              abi.rope_rows(16, 32, 2, 128, 128, 1, 20), abi.rope_rows(16, 32, 2, 128, 128, 1, None, -1.0),
              abi.rope_rows(16, 32, 2, 128, 128, 2, None, math.nan)):
        assert call(rows=(r,)) == BAD
        assert call(rows=(rows, r)) == BAD


@pytest.mark.parametrize("n", [1, 2, 21, 22, 64, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_frequencies_match_the_oracle(n, scaling):
    kind = ["none", "linear", "base", "parts"].index(scaling)
    for base, scale in [(10000.0, 8.0), (1e6, 4.0), (1.0, 2.0), (500000.0, 1.0)]:
        steps, factor = abi.ispa_rope_steps(n, base, kind, scale, 8192.0)
        w = ol.frequencies(n, base, scaling, scale, 8192.0)
        got = np.array([s / 2.0 ** 64 * 2 * np.pi for s in steps])
        # pow, a few products and (parts) a difference of numbers near 1: some steps of fp64, and half a step of 2^-64 turns
        assert np.all(np.abs(got - w) <= 64 * 2.0 ** -53 * w + 2.0 ** -62)
        assert factor == pytest.approx(0.1 * math.log(scale) + 1.0 if scaling == "parts" else 1.0, rel=2.0 ** -23)


def test_base_scaling_stretches_the_slowest_pair_by_the_whole_scale():
    plain = abi.ispa_rope_steps(64, 10000.0)[0]
    scaled = abi.ispa_rope_steps(64, 10000.0, abi.ISPA_ROPE_SCALE_BASE, 8.0)[0]
    assert scaled[0] == plain[0] and scaled[-1] == pytest.approx(plain[-1] / 8.0, rel=1e-12)


def test_frequency_refusals():
    for kw in (dict(n_pairs=0), dict(base=0.5), dict(base=math.nan), dict(base=math.inf), dict(scaling=4),
               dict(scaling=-1), dict(scaling=1, scale=0.5), dict(scaling=1, scale=math.inf),
               dict(scaling=3, scale=2.0, trained_length=0.0), dict(scaling=3, scale=2.0, low=4.0, high=4.0),
               dict(scaling=3, scale=2.0, low=-1.0), dict(scaling=3, scale=2.0, high=math.inf),
               dict(scaling=2, base=1e300, scale=1e300)):
        args = dict(n_pairs=32, trained_length=4096.0) | kw
        assert _status(lambda: abi.ispa_rope_steps(**args)) == BAD, kw
