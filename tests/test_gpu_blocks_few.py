"""Attention of one and two queries over the window, the chunk and selected blocks: the kernel without tensor cores, and
its border to the kernel with them at three.  The oracle and its bounds are those of tests/test_gpu_blocks.py.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import blocks as ob  # noqa: E402
from paper_2607_00712_gb300 import abi  # noqa: E402
from paper_2607_00712_gb300.device import to_f32  # noqa: E402
from test_gpu_blocks import Cache, Step, _lists, _ok  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


SHAPES = [  # chunk, H, d, P, cap, written, sinks, win, block, top_k
    (False, 1, 128, 16, 1, 1, 0, (0, 1), 64, 1),       # one unit of keys
    (True, 1, 128, 17, 3, 3, 0, (0, 1), 64, 2),        # a key behind it
    (True, 3, 128, 15, 4, 9, 1, (1, 1), 64, 2),
    (True, 5, 128, 333, 6, 6, 0, (0, 0), 64, 9),
    (True, 12, 128, 100, 9, 9, 1, (1, 3), 128, 5),     # blocks larger than a frame
    (False, 12, 128, 1000, 5, 5, 0, (0, 1), 512, 3),
    (True, 20, 128, 200, 7, 30, 2, (1, 1), 192, 4),    # clusters of seven
    (True, 40, 128, 90, 7, 7, 0, (0, 2), 64, 6),       # of three
    (False, 100, 128, 700, 8, 8, 0, (0, 8), 64, 3),    # a CTA a head; more than 32 units a warp
    (True, 160, 128, 65, 3, 3, 0, (0, 1), 64, 3),      # more heads than SMs
]


@pytest.mark.parametrize("n", [1, 2, 3])
@pytest.mark.parametrize("d,e4m3", [(64, False), (128, False), (128, True)])
@pytest.mark.parametrize("shape", SHAPES)
def test_few_queries(shape, d, e4m3, n):
    chunk, H, _, P, cap, written, sinks, win, block, top_k = shape
    c = Cache(P + n, H, d, P, cap, written, sinks, e4m3=e4m3)
    Step(n, c, n, chunk).check(c, win, block, _lists(P, c, win, block, n, top_k, H % 2 == 0))


@pytest.mark.parametrize("n", [1, 2])
@pytest.mark.parametrize("d,e4m3", [(64, False), (128, True)])
def test_heads_without_keys(n, d, e4m3):
    c = Cache(1, 3, d, 40, 4, e4m3=e4m3)
    lists = np.full((3, 1, 5), -1, np.int32)
    lists[1, 0, 4] = 2
    Step(2, c, n, False).check(c, (0, 0), 64, lists)
    nothing = np.full((3, 1, 5), -1, np.int32)
    Step(2, c, n, False).check(c, (0, 0), 64, nothing)
    Step(2, c, n, True).check(c, (0, 0), 64, nothing)    # the chunk alone


@pytest.mark.parametrize("n", [1, 2])
def test_numbers_of_no_resident_block_and_rows_behind_a_frame(n):
    """Numbers past the resident blocks are passed over, and rows next to a block, not a number among them, not used."""
    H, d, P, cap, block = 2, 128, 70, 4, 64
    c = Cache(3, H, d, P, cap, written=3)
    c.ring.k[:, 3 * P:], c.ring.v[:, 3 * P:] = float("nan"), float("nan")
    c.ring.k[:, P:2 * P], c.ring.v[:, P:2 * P] = float("nan"), float("inf")    # the frame after block 1's
    lists = np.array([[[1, 6, 7, 2 ** 31 - 1]], [[-5, 1, 4, -2 ** 31]]], np.int32)
    s = Step(4, c, n)
    out, lse = s.run(c, (0, 0), block, lists)
    _ok()
    kept = np.array([[[1, -1, -1, -1]], [[-1, 1, 4, -1]]], np.int32)
    want = ob.attend(s.q, c.k, c.v, [], kept, P, block, s.kc, s.vc, residents=6)
    b_out, b_lse = ob.bounds(*want, d)
    assert (np.abs(to_f32(out[:n]) - want[0]) <= b_out).all()
    assert (np.abs(lse[:-1].view(H, n).cpu().numpy() - want[1]) <= b_lse).all()


@pytest.mark.parametrize("n", [1, 2])
@pytest.mark.parametrize("e4m3", [False, True])
def test_large_scores(n, e4m3):
    """Scores some hundred apart: all weight on one key, wherever among warps and CTAs it is, and none lost."""
    c = Cache(5, 3, 128, 300, 5, e4m3=e4m3)
    for seed in (1, 2, 3):
        s = Step(seed, c, n)
        s.check(c, (0, 2), 64, _lists(seed, c, (0, 2), 64, n, 7), scale=16.0)


def test_the_same_bits_without_lse_and_again():
    c = Cache(6, 12, 128, 400, 6)
    s = Step(7, c, 2)
    lists = _lists(1, c, (0, 1), 64, 2, 20)
    out, lse = s.run(c, (0, 1), 64, lists)
    bare, _ = s.run(c, (0, 1), 64, lists, lse=False)
    again, lse2 = s.run(c, (0, 1), 64, lists)
    _ok()
    assert torch.equal(out, bare) and torch.equal(out, again) and torch.equal(lse, lse2)


def test_captured_beside_other_streams():
    """Two graphs of the same ring on two streams with other lists, replayed at once with lists changed in between."""
    H, d, P = 12, 128, 400
    c = Cache(8, H, d, P, 6)
    steps, graphs, outs, lists = [], [], [], []
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        s = Step(10 + i, c, 1 + i)
        t = torch.from_numpy(_lists(20 + i, c, (0, 1), 64, 1, 12)).cuda()
        s.run(c, (0, 1), 64, t)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[i]):
            o = s.run(c, (0, 1), 64, t, stream=streams[i])
        steps.append(s), graphs.append(g), outs.append(o), lists.append(t)
    for seed in (30, 40):
        for i in range(2):
            lists[i].copy_(torch.from_numpy(_lists(seed + i, c, (0, 1), 64, 1, 12)))
        torch.cuda.synchronize()
        for _ in range(5):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            steps[i].check(c, (0, 1), 64, lists[i], got=outs[i])
