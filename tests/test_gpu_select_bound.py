"""Selections whose scores in 32 bits are far off: queries that cancel in their sum, and values whose squares leave
fp32's range at its lower end.  Exact against the oracle: the queries are whole multiples of a power of two and their
sums have less than 53 bits, so the oracle's sums are exact in any order.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks as ob  # noqa: E402
from paper_2607_00712_gb300 import abi, synth  # noqa: E402
from paper_2607_00712_gb300.device import bf16_tensor  # noqa: E402
from test_gpu_blocks import Cache, _bf16, _select  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _check(q, means, top_k):
    H, cap, d = means.shape
    c = Cache(1, H, d, 1, 1)
    ring = abi.KVRing(H, d, 64, cap, 0, 0, cap, 16, 16)     # no key is read
    got = _select(c, (0, 0), 64, torch.from_numpy(means).cuda(), bf16_tensor(q), top_k, ring)
    assert np.array_equal(got, ob.select(ob.scores(q, means), list(range(cap)), top_k))


# queries, heads, head size, candidates, top_k: one launch (one query block; few candidates), two, three
FORMS = [(100, 7, 128, 1000, 90), (128, 5, 64, 700, 50), (300, 9, 128, 80, 30), (90, 1, 128, 6000, 500),
         (300, 12, 128, 1300, 128), (1100, 5, 64, 900, 64)]


def _queries(g, n, H, d, std, bits):
    """Normal values, whole multiples of std 2^-bits that bf16 holds."""
    q = _bf16(g, n, H, d, std=std)
    unit = 2.0 ** (np.round(np.log2(std)) - bits)
    q = (np.trunc(q / unit) * unit).astype(np.float32)
    assert np.array_equal(q, synth.bf16_round(q))
    return q


@pytest.mark.parametrize("n,H,d,cap,top_k", FORMS)
@pytest.mark.parametrize("x,std", [(2.0 ** 16, 0.01), (2.0 ** 13, 0.001), (1e6, 1.0), (1e8, 1.0), (2.0 ** 36, 1.0)])
def test_queries_that_cancel(x, std, n, H, d, cap, top_k):
    """Two rows of every query block are x and -x (different ones a feature, about as large)."""
    g = np.random.default_rng(n + cap)
    q = _queries(g, n, H, d, std, 14)
    large = synth.bf16_round((x * (1 + g.random((-(-n // 128), H, d)))).astype(np.float32) / 2)
    for i in range(-(-n // 128)):
        rows = g.permutation(min(128, n - 128 * i))[:2] + 128 * i
        q[rows[0]], q[rows[1]] = large[i], -large[i]
    means = g.standard_normal((H, cap, d)).astype(np.float32)
    _check(q, means, top_k)


@pytest.mark.parametrize("n,H,d,cap,top_k", FORMS)
@pytest.mark.parametrize("x", [1.0, 2.0 ** 20])
def test_all_queries_but_one_cancel(x, n, H, d, cap, top_k):
    g = np.random.default_rng(n)
    q = np.zeros((n, H, d), np.float32)
    for i in range(0, n, 128):
        rows = g.permutation(min(128, n - i)) + i
        half = (len(rows) - 1) // 2
        large = _queries(g, half, H, d, x, 14)
        q[rows[1:1 + half]], q[rows[1 + half:1 + 2 * half]] = large, -large
        q[rows[0]] = _queries(g, 1, H, d, x * 2.0 ** -12, 14)[0]
    means = g.standard_normal((H, cap, d)).astype(np.float32)
    _check(q, means, top_k)


@pytest.mark.parametrize("n,H,d,cap,top_k", FORMS)
@pytest.mark.parametrize("q_bits,m_bits", [(-80, 0), (-110, 0), (0, -80), (0, -100), (-75, -30), (-30, -75), (-120, 30),
                                           (60, -100)])
def test_values_whose_squares_underflow(q_bits, m_bits, n, H, d, cap, top_k):
    """Means of random signs that differ by some units of their last place."""
    g = np.random.default_rng(n + d)
    q = _queries(g, n, H, d, 1.0, 14) * np.float32(2.0 ** q_bits)
    means = g.choice([-1.0, 1.0], (H, 1, d)) * (1 + g.integers(0, 256, (H, cap, d)) * 2.0 ** -23)
    _check(q, (means * 2.0 ** m_bits).astype(np.float32), top_k)
