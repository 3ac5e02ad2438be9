"""The e4m3 quantisers on groups so small that fp32 does not hold 448 / amax (amax up to 7 * 2^-122, subnormal values too):
scale 1 and codes of zeros, no NaN; one step above, ordinary codes and scales.  Codes and scales bit for bit.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import quant as qt  # noqa: E402
from paper_2607_00712_gb300 import abi, synth  # noqa: E402

pytestmark = pytest.mark.gpu
EDGE = 7 * 2.0 ** -122          # 448 / EDGE = 2^128
STEP = 1 + 2.0 ** -7 / 1.75     # the next bf16 value
TOP = np.array([2.0 ** -116, 2.0 ** -118, EDGE * STEP, EDGE, 2.0 ** -121, 2.0 ** -126, 2.0 ** -133, 0.0], np.float32)
SMALL = TOP <= np.float32(EDGE)


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _rows(cols, seed):
    """A row of every TOP: that value, its negative, a zero and bf16 values between."""
    g = np.random.default_rng(seed)
    x = synth.bf16_round(((2 * g.random((len(TOP), cols)) - 1) * 0.99 * TOP[:, None]).astype(np.float32))
    x[:, 5], x[:, 7], x[:, 9] = TOP, -TOP, 0
    return x


def _check(codes, scale, want_codes, want_scale):
    assert np.array_equal(scale, want_scale) and np.array_equal(codes, want_codes)
    assert (scale[SMALL] == 1).all() and (scale[~SMALL] < 2.0 ** -120).all()
    value = qt.decode(codes)
    assert not value[SMALL].any()
    assert (value[~SMALL, 5] == 448).all() and (value[~SMALL, 7] == -448).all() and not value[:, 9].any()


# every number of values that a lane keeps, and rows that run past them
@pytest.mark.parametrize("cols", [16, 1024, 1536, 2048, 5120])
def test_rows(cols):
    x = _rows(cols, cols)
    T = len(TOP)
    q, s = torch.empty(T, cols, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
    abi.ispa_quantize_rows_e4m3(torch.from_numpy(x).cuda().to(torch.bfloat16), T, cols, q, s)
    _check(q.cpu().numpy(), s.cpu().numpy(), *qt.quantize_rows(x))


@pytest.mark.parametrize("D", [16, 272])
def test_weight_channels(D):
    x = _rows(D, D + 1)
    N = len(TOP)
    q, s = torch.empty(N, D, dtype=torch.uint8, device="cuda"), torch.empty(N, device="cuda")
    abi.ispa_quantize_weight_e4m3(torch.from_numpy(np.ascontiguousarray(x.T)).cuda(), None, D, N, q, s)
    _check(q.cpu().numpy(), s.cpu().numpy(), *qt.quantize_weight(np.ascontiguousarray(x.T)))


def test_a_product_with_small_rows_and_channels_is_finite():
    T, D, N = 256, 128, 128
    g = np.random.default_rng(0)
    x = synth.bf16_round(g.standard_normal((T, D)).astype(np.float32))
    W = g.standard_normal((D, N)).astype(np.float32)
    x[3] = _rows(D, 1)[3]
    W[:, 6] = _rows(D, 2)[4]
    q, s = torch.empty(T, D, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
    wq, ws = torch.empty(N, D, dtype=torch.uint8, device="cuda"), torch.empty(N, device="cuda")
    y = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    abi.ispa_quantize_rows_e4m3(torch.from_numpy(x).cuda().to(torch.bfloat16), T, D, q, s)
    abi.ispa_quantize_weight_e4m3(torch.from_numpy(W).cuda(), None, D, N, wq, ws)
    abi.ispa_linear_w8a8(q, s, wq, ws, T, D, N, y)
    torch.cuda.synchronize()
    y = y.float()
    assert torch.isfinite(y).all() and not y[3].any() and not y[:, 6].any()


# heads of keys and blocks of queries, whose codes go by 1 / scale
def test_heads_and_query_blocks():
    H, d, n = len(TOP), 128, 130
    g = np.random.default_rng(5)
    x = synth.bf16_round(((2 * g.random((n, H, d)) - 1) * 0.99 * TOP[None, :, None]).astype(np.float32))
    x[0, :, 5], x[1, :, 7], x[129, :, 5], x[128, :, 7] = TOP, -TOP, TOP, -TOP
    x[:, :, 9] = 0
    xt = torch.from_numpy(x).cuda().to(torch.bfloat16)
    q, s = torch.empty(n, H, d, dtype=torch.uint8, device="cuda"), torch.empty(H, device="cuda")
    abi.ispa_quantize_heads_e4m3(xt, n, H, d, q, s)
    qb, sb = torch.empty(n, H, d, dtype=torch.uint8, device="cuda"), torch.empty(H, 2, device="cuda")
    abi.ispa_quantize_q_e4m3(xt, n, H, d, qb, sb)
    codes, scale = qt.quantize_heads(x)
    assert (scale[SMALL] == 1).all() and (scale[~SMALL] < 2.0 ** -120).all()
    assert np.array_equal(s.cpu().numpy(), scale) and np.array_equal(q.cpu().numpy(), codes)
    codes, scale = qt.quantize_query_blocks(x)
    assert np.array_equal(sb.cpu().numpy(), scale) and np.array_equal(qb.cpu().numpy(), codes)
    for c in (q, qb):
        value = qt.decode(c.cpu().numpy())
        assert not value[:, SMALL].any() and (value[0, ~SMALL, 5] == 448).all() and (value[1, ~SMALL, 7] == -448).all()
