"""Selection in one launch, for one query block (up to 128 queries) or few candidates, and its borders to the two and
three launches.  Exact, as in tests/test_gpu_blocks.py.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks as ob  # noqa: E402
from oracle import keysets as ks  # noqa: E402
from paper_2607_00712_gb300 import abi, synth  # noqa: E402
from paper_2607_00712_gb300.device import Window, bf16_tensor  # noqa: E402
from test_gpu_blocks import Cache, _bf16, _ok, _select  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _candidates(P, cap, sinks, written, win):
    nb = ob.per_frame(P, 64)
    local = ks.local_past_frames(written, *win)
    slots = sorted(ks.ring_slot(f, cap, sinks) for f in ks.resident_frames(written, cap, sinks) if f not in local)
    return [s * nb + b for s in slots for b in range(nb)]


# candidates at the borders of the instances (256, 1280, 2560, 5120) and of the CTAs' shares (64, 192 a CTA)
@pytest.mark.parametrize("n,H,d,cap,top_k", [
    (1, 1, 128, 63, 8), (1, 2, 64, 64, 63), (7, 1, 128, 65, 9), (128, 3, 64, 255, 100), (127, 2, 128, 257, 256),
    (1, 1, 128, 1280, 64), (33, 7, 64, 1281, 64), (2, 1, 128, 1536, 30), (2, 1, 128, 1537, 30), (1, 7, 128, 2560, 1),
    (17, 8, 128, 2561, 500), (1, 12, 64, 5120, 64), (16, 12, 128, 5121, 64), (3, 2, 64, 5121, 2000),
    (1, 40, 128, 700, 64), (100, 60, 64, 300, 5), (1, 160, 128, 400, 50), (128, 9, 128, 9000, 77)])
def test_selection(n, H, d, cap, top_k):
    c = Cache(1, H, d, 1, 1)
    ring = abi.KVRing(H, d, 64, cap, 0, 0, cap, 16, 16)     # no key is read
    g = np.random.default_rng(n + cap)
    means = g.standard_normal((H, cap, d)).astype(np.float32)
    q = _bf16(g, n, H, d)
    got = _select(c, (0, 0), 64, torch.from_numpy(means).cuda(), bf16_tensor(q), top_k, ring)
    assert np.array_equal(got, ob.select(ob.scores(q, means), list(range(cap)), top_k))


# an SM's share of the candidates below and above 450 (64 features: 200), lists of each instance, 2 to 74 query blocks
@pytest.mark.parametrize("n,H,d,cap,top_k", [
    (1100, 12, 128, 50, 7), (1100, 12, 128, 1500, 64), (2200, 12, 128, 1300, 64), (5000, 40, 64, 70, 5),
    (5000, 40, 128, 130, 30), (1000, 3, 64, 1281, 64), (140, 2, 64, 1600, 100), (140, 2, 64, 1601, 100),
    (256, 1, 128, 3600, 64), (256, 1, 128, 3601, 64), (9400, 2, 128, 460, 100), (9400, 2, 128, 900, 100),
    (9400, 2, 64, 205, 3), (9400, 2, 64, 201, 3), (4680, 3, 128, 100, 99), (4680, 3, 128, 601, 64),
    (300, 40, 128, 451, 33), (300, 50, 128, 456, 33), (520, 3, 128, 2561, 40), (1025, 2, 128, 5121, 40),
    (700, 160, 64, 9, 4),
    # 32, 25, 24 and 74 query blocks in three launches
    (4000, 12, 128, 1300, 64), (3200, 12, 64, 700, 30), (3000, 3, 128, 1400, 70), (9400, 12, 128, 1300, 128)])
def test_selection_of_more_query_blocks(n, H, d, cap, top_k):
    test_selection(n, H, d, cap, top_k)


@pytest.mark.parametrize("n", [1, 90])
@pytest.mark.parametrize("P,cap,written,sinks,win", [(700, 20, 20, 0, (0, 3)), (333, 31, 77, 2, (1, 4)),
                                                     (1000, 9, 100, 1, (1, 1)), (64, 700, 5000, 3, (3, 100))])
def test_selection_around_a_window(P, cap, written, sinks, win, n):
    H, d = 5, 128
    c = Cache(1, H, d, 1, 1)
    ring = abi.KVRing(H, d, P, cap, sinks, 0, written, 16, 16)
    g = np.random.default_rng(P)
    means = g.standard_normal((H, cap * ob.per_frame(P, 64), d)).astype(np.float32)
    cand = _candidates(P, cap, sinks, written, win)
    outside = np.setdiff1d(np.arange(means.shape[1]), cand)
    means[:, outside] = np.nan                               # not read
    q = _bf16(g, n, H, d)
    got = _select(c, win, 64, torch.from_numpy(means).cuda(), bf16_tensor(q), 40, ring)
    assert np.array_equal(got, ob.select(ob.scores(q, np.nan_to_num(means)), cand, 40))


@pytest.mark.parametrize("cap", [80, 1000, 6000])
@pytest.mark.parametrize("values,top_k", [("same", 10), ("zero", 10), ("few", 33), ("pairs", 7), ("nan", 30),
                                          ("inf", 30), ("nan", 75), ("huge", 40), ("tiny", 40), ("close", 50)])
def test_equal_close_and_extreme_scores(values, top_k, cap, n=100):
    """Small whole numbers, whose scores are exact in any order, and values at the ends of the range."""
    H, d = 7, 128
    c = Cache(9, H, d, 1, 1)
    ring = abi.KVRing(H, d, 64, cap, 0, 0, cap, 16, 16)
    g = np.random.default_rng(4)
    m = g.integers(-3, 4, (H, cap, d)).astype(np.float32)
    q = g.integers(-3, 4, (n, H, d)).astype(np.float32)
    if values == "same":
        m[:] = m[:, :1]
    elif values == "zero":
        q[:] = 0
    elif values == "few":
        m[:] = m[:, :1] * g.integers(0, 3, (1, cap, 1))
    elif values == "pairs":
        m[:, 1::2] = m[:, ::2]
    elif values == "nan":
        m[:, ::3, 5] = np.nan
    elif values == "inf":
        m[:, ::7, 5] = np.inf
    elif values == "huge":
        q, m = synth.bf16_round(q * np.float32(1e38)), m * np.float32(2.0 ** 125)
    elif values == "tiny":
        q, m = synth.bf16_round(q * np.float32(2.0 ** -130)), m * np.float32(2.0 ** -140)
    elif values == "close":      # one part in 2^23 apart: not to be told apart by a sum in 32 bits
        m[:] = 1 + g.permutation(cap)[None, :, None] * 2.0 ** -23
        q[:] = np.abs(q) + 1
    with np.errstate(invalid="ignore"):
        score = ob.scores(q, m)
    got = _select(c, (0, 0), 64, torch.from_numpy(m).cuda(), bf16_tensor(q), top_k, ring)
    assert np.array_equal(got, ob.select(score, list(range(cap)), top_k))


@pytest.mark.parametrize("cap,n", [(80, 300), (1000, 1100), (6000, 300)])   # one launch, three, three
@pytest.mark.parametrize("values,top_k", [("same", 10), ("few", 33), ("nan", 75), ("inf", 30), ("huge", 40),
                                          ("close", 50)])
def test_the_same_of_more_query_blocks(values, top_k, cap, n):
    test_equal_close_and_extreme_scores(values, top_k, cap, n)


def test_calls_in_a_row_over_one_workspace_and_replayed():
    """Calls that share a workspace, one behind the other in one graph, with new queries and means at every replay."""
    H, d, cap, top_k = 12, 128, 900, 20
    ring = abi.KVRing(H, d, 64, cap, 0, 0, cap, 16, 16)
    g = np.random.default_rng(3)
    sizes = [1, 128, 5, 300]
    means = torch.empty(H, cap, d, device="cuda")
    q = [torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda") for n in sizes]
    out = [torch.empty(H, -(-n // 128), top_k, dtype=torch.int32, device="cuda") for n in sizes]
    size = max(abi.ispa_select_blocks_workspace_size(ring, 64, n) for n in sizes)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def calls():
        for a, b in zip(q, out):
            abi.ispa_select_blocks(ring, Window(0, 0), 64, means, a, a.shape[0], top_k, b, ws, size,
                                   torch.cuda.current_stream())
    for a in q:
        a.zero_()
    means.zero_()
    torch.cuda.synchronize()
    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        hm = g.standard_normal((H, cap, d)).astype(np.float32)
        hq = [_bf16(g, n, H, d) for n in sizes]
        means.copy_(torch.from_numpy(hm))
        for a, b in zip(q, hq):
            a.copy_(bf16_tensor(b))
        torch.cuda.synchronize()
        for _ in range(4):
            graph.replay()
        _ok()
        for b, got in zip(hq, out):
            assert np.array_equal(got.cpu().numpy(), ob.select(ob.scores(b, hm), list(range(cap)), top_k))
