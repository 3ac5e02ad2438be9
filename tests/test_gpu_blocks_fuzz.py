"""Random sizes, windows, lists and formats of the operators around selected blocks, some rows of each on the oracle."""
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_helpers as lh  # noqa: E402
from oracle import blocks as ob  # noqa: E402
from paper_2607_00712_gb300 import abi  # noqa: E402
from paper_2607_00712_gb300.device import to_f32  # noqa: E402
from test_gpu_append_rope import Call  # noqa: E402
from test_gpu_blocks import Cache, Step, _lists, _ok, _select  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _log(r, lo, hi):
    return int(round(lo * (hi / lo) ** r.random()))


@pytest.mark.parametrize("seed", range(24))
def test_attention_of_a_selection(seed):
    r = random.Random(seed)
    e4m3 = r.random() < 0.4
    H, d = r.choice([1, 2, 5, 40]), 128 if e4m3 else r.choice([64, 128])
    P, block = _log(r, 1, 700), 64 * r.choice([1, 1, 2, 3, 20])
    cap, sinks = r.randint(2, 12), r.choice([0, 0, 1])
    written = r.choice([1, cap - 1, cap, 3 * cap + 1])
    recent = r.randint(0, min(2, cap - sinks))
    win = (r.randint(0, sinks), recent)
    chunk = r.random() < 0.7
    causal = chunk and not e4m3 and r.random() < 0.3
    n = P * r.randint(1, 2) if causal else _log(r, 1, 900)
    top_k = _log(r, 1, 60)
    c = Cache(seed, H, d, P, cap, written, sinks, e4m3)
    s = Step(seed + 100, c, n, chunk)
    nb = ob.per_frame(P, block)
    means = torch.zeros(H, cap * nb, d, device="cuda")
    scale = c.ks_t if e4m3 else None
    if c.resident()[0] == 0 and len(c.resident()) > 1:      # the sinks, then the rest
        abi.ispa_key_means(c.ring.c, scale, 0, 1, block, means)
    rest = [f for f in c.resident() if f >= max(1, written - (cap - sinks))] or [0]
    abi.ispa_key_means(c.ring.c, scale, rest[0], len(rest), block, means)
    q16 = torch.from_numpy(np.asarray(s.q, np.float32)).cuda().to(torch.bfloat16)
    got = _select(c, win, block, means, q16, top_k)
    cand = [x * nb + b for x in c.history(win) for b in range(nb)]
    m = means.cpu().numpy()
    want_m, size = ob.key_means(c.k, P, block), ob.key_means(np.abs(c.k), P, block)
    known = [x * nb + b for x in c.slots(c.resident()) for b in range(nb)]
    lh.assert_within(m[:, known], want_m[:, known], (min(P, block) + 8) * lh.U * size[:, known] + 1e-40, "means")
    assert np.array_equal(got, ob.select(ob.scores(to_f32(q16), m), cand, top_k))
    lists = got if seed % 2 else _lists(seed, c, win, block, n, top_k, True)
    out, lse = s.run(c, win, block, lists, causal)
    _ok()
    rows = sorted({0, n - 1, n // 2, min(n - 1, 127), min(n - 1, 128)})
    want = ob.attend(s.q, c.k, c.v, c.window(win), lists, P, block, s.kc if chunk else None, s.vc if chunk else None,
                     None, causal, min(written, cap) * nb, queries=rows)
    b_out, b_lse = ob.bounds(*want, d)
    lh.assert_within(to_f32(out[:n])[rows], want[0][rows], b_out[rows], "out")
    g, w = lse[:-1].view(H, n).cpu().numpy()[:, rows], want[1][:, rows]
    none = np.isneginf(w)
    assert (np.isneginf(g) == none).all()
    lh.assert_within(np.where(none, 0, g), np.where(none, 0, w), np.where(none, 1, b_lse[:, rows]), "lse")


@pytest.mark.parametrize("seed", range(24))
def test_append(seed):
    r = random.Random(seed)
    fmt = r.choice([0, 0, 1, 2])
    d = 128 if fmt else r.choice([64, 128])
    H, layout = r.choice([1, 2, 7, 12, 33]), r.choice([abi.ISPA_ROPE_INTERLEAVED, abi.ISPA_ROPE_HALF])
    P = 4 * _log(r, 1, 150) if fmt == 2 else _log(r, 1, 600)
    pairs = 4 * r.randint(1, d // 8)
    axes = [pairs] if r.random() < 0.5 else [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]
    norms = [r.choice([abi.ISPA_QK_NORM_NONE, abi.ISPA_QK_NORM_HEAD, abi.ISPA_QK_NORM_TOKEN])] * 2
    if r.random() < 0.2:
        norms[0] = abi.ISPA_QK_NORM_NONE
    frames = r.randint(1, 4)
    sinks = r.choice([0, 0, 2])
    cap = frames + sinks + r.randint(0, 3)
    Call(P, frames, H * r.choice([0, 1, 1, 3]), H, d, axes, layout, tuple(norms), fmt, cap, sinks,
         r.choice([0, 1, 5, 100]), r.randint(0, 10 ** 9), r.random() < 0.2, seed).run().check()
