"""Random sizes, layouts and options of the norm, residual, rotary and int8 entry points against the oracle, by the checks of
their own test files; sizes on both sides of every choice of kernel."""
import random

import pytest

torch = pytest.importorskip("torch")

import test_gpu_linear_i8 as ti  # noqa: E402
import test_gpu_norm as tn  # noqa: E402
import test_gpu_rope as tr  # noqa: E402
from oracle import layer as ol  # noqa: E402
from paper_2607_00712_gb300 import abi  # noqa: E402

pytestmark = pytest.mark.gpu
MOST = 3_000_000      # values of a case


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _rows_and_dim(r):
    while True:
        rows, dim = round(2 ** r.uniform(0, 12)), 8 * round(2 ** r.uniform(0, 11))
        if rows * dim <= MOST:
            return rows, dim


@pytest.mark.parametrize("seed", range(24))
def test_norms(seed):
    r = random.Random(seed)
    rows, dim = _rows_and_dim(r)
    kinds = [ol.NONE, ol.RMS, ol.LAYER]
    tn._norm_case(rows, dim, r.random() < 0.5, r.choice(kinds), r.choice(["bf16", "e4m3", "i8"]), r.random() < 0.5,
                  round(2 ** r.uniform(0, 11)), r.choice(["none", "scale", "shift", "both", "both"]))
    rows, dim = _rows_and_dim(r)
    tn._residual_case(rows, dim, r.random() < 0.5, r.choice([None, *kinds]), r.choice(kinds),
                      r.choice(["bf16", "e4m3", "i8"]), r.random() < 0.5, r.random() < 0.8)


@pytest.mark.parametrize("seed", range(32))
def test_rotary(seed):
    r = random.Random(100 + seed)
    layout = r.choice(tr.LAYOUTS)
    while True:
        d = 8 * r.randint(1, 32) if r.random() < 0.4 else r.choice([64, 128, 256])
        k = r.choice([1, 2, 3, 5, 8, 12, 40])
        heads = r.choice([(k,), (k, k), (k * r.choice([2, 4]), k)])
        n = round(2 ** r.uniform(0, 12))
        unit = 4 if layout == abi.ISPA_ROPE_HALF else 1
        if n * sum(heads) * d <= MOST and d // 2 >= unit:
            break
    pairs = unit * r.randint(1, d // 2 // unit)
    if r.random() < 0.4:
        pairs = d // 2 // unit * unit
    cut = sorted(r.randint(0, pairs) for _ in range(2))
    split = r.choice([[pairs], [cut[0], pairs - cut[0]], [cut[0], cut[1] - cut[0], pairs - cut[1]]])
    tr._case(n, heads, d, split, layout, r.choice(tr.NORMS), pos0=r.choice([0, 57, -3]), in_place=r.random() < 0.3,
             seed=seed)


@pytest.mark.parametrize("seed", range(32))
def test_int8_products(seed):
    r = random.Random(200 + seed)
    while True:
        T, D, N = round(2 ** r.uniform(0, 12)), 16 * round(2 ** r.uniform(0, 8.5)), 8 * round(2 ** r.uniform(0, 9.5))
        if T * D + D * N + T * N <= MOST and T * D * N <= 4e9:
            break
    ti._check(T, D, N, bias=r.random() < 0.5, full=r.random() < 0.3, seed=seed)
