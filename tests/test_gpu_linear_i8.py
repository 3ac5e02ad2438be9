"""The projection in 8-bit integers through the C-ABI: every step is specified, so results equal the oracle's bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import layer as ol  # noqa: E402
from paper_2607_00712_gb300 import abi, synth  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _inputs(seed, T, D, N, full=False):
    g = np.random.default_rng(seed)
    if full:      # all codes, -128 too
        a, w = (g.integers(-128, 128, s, dtype=np.int8) for s in ((T, D), (N, D)))
    else:
        a, w = (np.clip(np.rint(36 * g.standard_normal(s)), -127, 127).astype(np.int8) for s in ((T, D), (N, D)))
    return a, w, *((0.01 * (0.2 + g.random(n))).astype(np.float32) for n in (T, N)), \
        g.standard_normal(N).astype(np.float32)


def _run(a, w, sa, sw, bias, stream=None):
    T, D = a.shape
    N = w.shape[0]
    t = [torch.from_numpy(x).cuda() for x in (a, sa, w, sw)]
    b = None if bias is None else torch.from_numpy(bias).cuda()
    out = torch.full((T + 1, N), 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    abi.ispa_linear_i8(*t, b, T, D, N, out, stream)
    torch.cuda.synchronize()
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK
    assert (out[T] == 7.0).all()
    return out[:T].float().cpu().numpy()


def _check(T, D, N, bias=True, full=False, seed=0):
    a, w, sa, sw, b = _inputs(seed + T + D + N, T, D, N, full)
    got = _run(a, w, sa, sw, b if bias else None)
    assert np.array_equal(got, ol.linear_i8(a, sa, w, sw, b if bias else None))


# few tokens, on both sides of every number of tokens that a warp takes
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("D,N", [(16, 8), (48, 24), (512, 40), (528, 1000), (1536, 1536), (5120, 72)])
def test_few_tokens(T, D, N):
    _check(T, D, N, bias=T % 2 == 1, full=D == 48)


# clusters of CTAs that share a contraction: shares of one block and of more than 1024 codes, odd ones
@pytest.mark.parametrize("T,D,N", [(9, 128, 8), (16, 256, 64), (17, 272, 136), (61, 5120, 640), (128, 1536, 128),
                                   (129, 1040, 392), (64, 13824, 256), (200, 4112, 200), (33, 20480, 8)])
def test_split_contraction(T, D, N):
    _check(T, D, N, full=T == 17)


# whole tiles: one, many, ragged in every direction; a contraction that ends inside a block, and of 1, 2, 3 ... exact runs
@pytest.mark.parametrize("T,D,N", [(9, 16, 8), (130, 64, 128), (300, 80, 264), (1000, 1024, 1000), (1536, 1040, 1544),
                                   (2048, 48, 2048)])
def test_tiles(T, D, N):
    _check(T, D, N, bias=T != 1000)


# pairs of CTAs, several waves, ragged
@pytest.mark.parametrize("T,D,N", [(4680, 512, 1536), (2500, 1104, 2056), (5000, 64, 2568), (4680, 1536, 4608),
                                   (2305, 3136, 3848)])
def test_large(T, D, N):
    _check(T, D, N, full=T == 2500)


@pytest.mark.parametrize("T", [1, 8, 40, 1200, 2600])
def test_the_largest_sums_are_exact(T):
    # 1024 products of 2^14 fill the accumulator's 24 bits to the last; every sum of one sign, and one that cancels
    D, N = 4096 + 16, 264 if T < 2600 else 2056
    a = np.full((T, D), -128, np.int8)
    w = np.full((N, D), -128, np.int8)
    w[1::2] = 127
    w[2::4, D // 2:] = 127
    w[3::8, 5] = 126
    sa, sw = np.ones(T, np.float32), np.full(N, 2.0 ** -20, np.float32)
    got = _run(a, w, sa, sw, None)
    assert np.array_equal(got, ol.linear_i8(a, sa, w, sw))


def test_the_sum_itself_comes_out_with_a_scale_of_one():
    # sums below 2^8 survive the rounding to bf16: cancelling products of large codes leave a small integer
    T, D, N = 300, 2048, 256
    g = np.random.default_rng(3)
    h = g.integers(-127, 128, (T, D // 2), dtype=np.int8)
    a = np.concatenate([h, -h], 1)
    w = np.concatenate([np.full((N, D // 2), 127, np.int8)] * 2, 1)
    a[:, 0] = (h[:, 0].astype(np.int32) // 2).astype(np.int8)
    w[:, 0] = 1
    w[:, D // 2] = 1
    one = np.ones(max(T, N), np.float32)
    want = (a.astype(np.int64) @ w.astype(np.int64).T)
    assert np.abs(want).max() <= 256
    assert np.array_equal(_run(a, w, one[:T], one[:N], None), want.astype(np.float32))


def test_the_longest_contraction():
    D = 131056
    for T in (1, 12):
        a, w, sa, sw, b = _inputs(T, T, D, 16)
        a[0], w[0] = -128, -128      # 2147221504, below 2^31
        got = _run(a, w, sa, sw, b)
        assert np.array_equal(got, ol.linear_i8(a, sa, w, sw, b))


def test_scales_that_are_not_finite_reach_their_row_and_channel_alone():
    for T in (5, 60, 3000):
        a, w, sa, sw, b = _inputs(1, T, 128, 2056)
        a[a == 0] = 1
        sa[3], sw[7] = np.nan, np.inf
        got = _run(a, w, sa, sw, b)
        with np.errstate(invalid="ignore"):
            want = ol.linear_i8(a, sa, w, sw, b)
        assert np.isnan(got[3]).all() and not np.isfinite(got[:, 7]).any()
        keep = np.ones(want.shape, bool)
        keep[3], keep[:, 7] = False, False
        assert np.array_equal(got[keep], want[keep])


@pytest.mark.parametrize("T,D", [(1, 16), (3, 48), (77, 1536), (900, 1024), (33, 5120), (700, 2064)])
def test_quantized_rows(T, D):
    x = synth.bf16_round((np.random.default_rng(T + D).standard_normal((T, D)) * 3).astype(np.float32))
    if T > 2:
        x[1] = 0
        x[2] *= 2.0 ** -100
    xt = torch.from_numpy(x).cuda().to(torch.bfloat16)
    q = torch.full((T + 1, D), 77, dtype=torch.int8, device="cuda")
    s = torch.full((T + 1,), 7.0, device="cuda")
    abi.ispa_quantize_rows_i8(xt, T, D, q, s)
    torch.cuda.synchronize()
    codes, scale = ol.quantize_i8(x)
    assert np.array_equal(q[:T].cpu().numpy(), codes) and np.array_equal(s[:T].cpu().numpy(), scale)
    assert (q[T] == 77).all() and s[T] == 7.0


# a row shared by two or eight warps of a block, a block's last row missing, rows that run past what the block holds
@pytest.mark.parametrize("T,D", [(1, 3216), (2, 4096), (3, 5120), (5, 5136), (1, 10240), (3, 10256), (2, 16400),
                                 (301, 8960)])
def test_quantized_long_rows(T, D):
    test_quantized_rows(T, D)


# 2^-117 and what is below it (subnormal values too), on both sides of the quotients that fp32 holds
@pytest.mark.parametrize("D", [64, 1536, 5120])
def test_groups_of_tiny_values(D):
    g = np.random.default_rng(D)
    top = np.array([2.0 ** -116, 2.0 ** -117, 2.0 ** -117 * (1 - 2.0 ** -8), 2.0 ** -119, 2.0 ** -121, 2.0 ** -126,
                    2.0 ** -133, 0.0], np.float32)
    x = synth.bf16_round(((2 * g.random((len(top), D)) - 1) * 0.99 * top[:, None]).astype(np.float32))
    x[:, 5], x[:, 7], x[:, 9] = top, -top, 0
    codes, scale = ol.quantize_i8(x)
    assert (scale[:2] != 1).all() and (scale[2:] == 1).all() and not codes[2:].any() and codes[1, 5] == 127
    T = len(top)
    q, s = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    abi.ispa_quantize_rows_i8(torch.from_numpy(x).cuda().to(torch.bfloat16), T, D, q, s)
    qw, sw = torch.empty(T, D, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    abi.ispa_quantize_weight_i8(torch.from_numpy(np.ascontiguousarray(x.T)).cuda(), None, D, T, qw, sw)
    torch.cuda.synchronize()
    for codes_of, scale_of in ((q, s), (qw, sw)):
        assert np.array_equal(codes_of.cpu().numpy(), codes) and np.array_equal(scale_of.cpu().numpy(), scale)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_non_finite_row_is_no_finite_result(bad):
    T, D, N = 20, 2064, 64
    x = torch.randn(T, D, device="cuda").to(torch.bfloat16)
    x[4, 2050] = bad
    x[9, 3] = bad
    q = torch.empty(T, D, dtype=torch.int8, device="cuda")
    s = torch.empty(T, device="cuda")
    abi.ispa_quantize_rows_i8(x, T, D, q, s)
    w = torch.ones(N, D, dtype=torch.int8, device="cuda")
    out = torch.empty(T, N, dtype=torch.bfloat16, device="cuda")
    abi.ispa_linear_i8(q, s, w, torch.ones(N, device="cuda"), None, T, D, N, out)
    torch.cuda.synchronize()
    fine = torch.isfinite(out.float()).all(1)
    assert [t for t in range(T) if not fine[t]] == [4, 9]


@pytest.mark.parametrize("D,N", [(16, 8), (272, 100), (1536, 512)])
@pytest.mark.parametrize("with_dw", [False, True])
def test_quantized_weight(D, N, with_dw):
    W = synth.make_weight(D, D, N)
    dW = (0.1 * synth.make_weight(D + 1, D, N)).astype(np.float32) if with_dw else None
    W[:, 3] = 0
    if with_dw:
        dW[:, 3] = 0
    q = torch.empty(N, D, dtype=torch.int8, device="cuda")
    s = torch.empty(N, device="cuda")
    abi.ispa_quantize_weight_i8(torch.from_numpy(W).cuda(), None if dW is None else torch.from_numpy(dW).cuda(), D, N, q, s)
    torch.cuda.synchronize()
    codes, scale = ol.quantize_i8((W + dW if with_dw else W).T)
    assert np.array_equal(q.cpu().numpy(), codes) and np.array_equal(s.cpu().numpy(), scale)


def test_captured_side_stream_and_two_at_once():
    sizes = [(4, 1536, 512), (60, 2048, 256), (4680, 256, 1536)]
    for T, D, N in sizes:
        a, w, sa, sw, b = _inputs(T, T, D, N)
        want = ol.linear_i8(a, sa, w, sw, b)
        t = [torch.from_numpy(x).cuda() for x in (a, sa, w, sw, b)]
        outs = [torch.zeros(T, N, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            abi.ispa_linear_i8(*t, T, D, N, outs[0], torch.cuda.current_stream())
        for _ in range(2):
            outs[0].zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert np.array_equal(outs[0].float().cpu().numpy(), want)
        streams = [torch.cuda.Stream() for _ in range(2)]
        for _ in range(4):
            for st, o in zip(streams, outs[1:]):
                abi.ispa_linear_i8(*t, T, D, N, o, st)
        torch.cuda.synchronize()
        for o in outs[1:]:
            assert np.array_equal(o.float().cpu().numpy(), want)
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK
