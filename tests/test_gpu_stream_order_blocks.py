"""The append with rotary positions, the means, the selection and the attention back to back: launches that start while
the one before still runs must not read what it has not written, nor write what it still reads.  The same calls with a
wait behind each of them are the reference, bit for bit; then from four threads, and replayed from a graph."""
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_00712_gb300 import abi  # noqa: E402
from paper_2607_00712_gb300.device import Ring, Window  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


class Layer:
    """A layer's ring and buffers; step() runs a chunk through it, `wait` behind every call."""

    def __init__(self, seed, H, P, chunk, fmt=0, norm=abi.ISPA_QK_NORM_TOKEN, block=64, top_k=9, cap=8):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.H, self.P, self.chunk, self.fmt, self.norm, self.block, self.top_k = H, P, chunk, fmt, norm, block, top_k
        self.n, self.d, self.W = P * chunk, 128, 3 * H * 128
        self.ring = Ring(H, 128, P, cap, 1, k_e4m3=fmt == 1)
        self.nb, n_qt = -(-P // block), -(-self.n // 128)
        self.means = torch.zeros(H, cap * self.nb, 128, device="cuda")
        self.src = [torch.randn(self.n, self.W, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3)]
        self.x = torch.empty_like(self.src[0])
        self.q = torch.empty(self.n, H, 128, dtype=torch.bfloat16, device="cuda")
        self.k, self.v = torch.empty_like(self.q), torch.empty_like(self.q)
        self.q8, self.k8 = torch.empty(2, self.n, H, 128, dtype=torch.uint8, device="cuda")
        self.qs = torch.empty(H, n_qt, device="cuda")
        self.ks = torch.full((H,), 4.0 / 448, device="cuda")
        self.w = 1 + 0.1 * torch.randn(H * 128, generator=g, device="cuda")
        steps = abi.ispa_rope_steps(64)[0]
        self.steps = torch.from_numpy(np.array(steps, np.uint64).view(np.int64)).cuda()
        self.rope = abi.rope(abi.ISPA_ROPE_HALF, 128, [64], self.steps)
        self.pos = torch.arange(self.n, device="cuda", dtype=torch.int32)
        self.blocks = torch.zeros(H, n_qt, top_k, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(abi.ispa_select_blocks_workspace_size(self.ring.c, block, self.n), dtype=torch.uint8,
                              device="cuda")
        self.out = torch.empty(self.n, H * 128, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.empty(H, self.n, device="cuda")
        torch.cuda.synchronize()

    def step(self, i, stream, wait):
        H, W, n, c = self.H, self.W, self.n, self.ring.c
        rows = abi.rope_rows
        with torch.cuda.stream(stream):
            self.x.copy_(self.src[i % 3])
            wait()
            q, k = (rows(x, out, H, W, H * 128, self.norm, self.w)
                    for x, out in ((self.x, self.q), (self.x[:, H * 128:], self.k)))
            abi.ispa_rope_apply(self.rope, [q, k], self.pos, i * n, n, stream)
            wait()
            self.v.copy_(self.x[:, 2 * H * 128:].view(n, H, 128))
            wait()
            abi.ispa_select_blocks(c, Window(1, 2), self.block, self.means, self.q, n, self.top_k, self.blocks, self.ws,
                                   self.ws.numel(), stream)
            wait()
            if self.fmt:
                abi.ispa_quantize_q_e4m3(self.q, n, H, 128, self.q8, self.qs, stream)
                wait()
                abi.ispa_quantize_k_e4m3(self.k, n, H, 128, self.ks, self.k8, stream)
                wait()
                abi.ispa_attn_blocks_qk8(c, self.ks, Window(1, 2), self.block, self.blocks, self.top_k, self.q8,
                                         self.qs, self.k8, self.ks, self.v, n, 0.0, self.out, self.lse, stream)
            else:
                abi.ispa_attn_blocks(c, Window(1, 2), self.block, self.blocks, self.top_k, self.q, self.k, self.v, n,
                                     0.0, 0, self.out, self.lse, stream)
            wait()
            abi.ispa_kv_append_rope(c, self.rope, rows(self.x[:, H * 128:], None, H, W, 0, self.norm, self.w),
                                    rows(self.x, self.q, H, W, H * 128, self.norm, self.w), self.x[:, 2 * H * 128:], W,
                                    self.pos, i * n, self.chunk, self.ks if self.fmt else None, None, stream)
            wait()
            abi.ispa_key_means(c, self.ks if self.fmt else None, c.frames_written - self.chunk, self.chunk, self.block,
                               self.means, stream)
            wait()

    def results(self):
        return [t.clone() for t in (self.q, self.ring.k, self.ring.v, self.means, self.blocks, self.out, self.lse)]


CASES = [dict(seed=1, H=12, P=1560, chunk=1), dict(seed=2, H=12, P=900, chunk=2, norm=abi.ISPA_QK_NORM_HEAD),
         dict(seed=3, H=40, P=700, chunk=1, fmt=1), dict(seed=4, H=3, P=10, chunk=1, top_k=3),
         dict(seed=5, H=2, P=130, chunk=3, norm=abi.ISPA_QK_NORM_NONE, fmt=1, top_k=300)]


def _waited(case, steps=5):
    a = Layer(**case)
    stream = torch.cuda.Stream()
    out = []
    for i in range(steps):
        a.step(i, stream, torch.cuda.synchronize)
        out.append(a.results())
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("case", CASES)
def test_back_to_back(case):
    want = _waited(case)
    for _ in range(3):
        b = Layer(**case)
        stream = torch.cuda.Stream()
        got = []
        with torch.cuda.stream(stream):
            for i in range(5):
                b.step(i, stream, lambda: None)
                got.append(b.results())
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert all(torch.equal(s, t) for s, t in zip(x, y))
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


def test_from_four_threads():
    cases = CASES[:4]
    want = [_waited(c)[-1] for c in cases]
    got, errors = [None] * 4, []

    def work(j):
        try:
            layer, stream = Layer(**cases[j]), torch.cuda.Stream()
            for i in range(5):
                layer.step(i, stream, lambda: None)
            stream.synchronize()
            got[j] = layer.results()
        except Exception as e:      # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(j,)) for j in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    torch.cuda.synchronize()
    assert not errors
    for x, y in zip(got, want):
        assert all(torch.equal(s, t) for s, t in zip(x, y))


@pytest.mark.parametrize("case", CASES[:3])
def test_a_chunk_from_a_graph(case):
    """Two chunks eager, the third captured and replayed twice: a replay writes the frames of the capture again."""
    want = _waited(case, 3)[-1]
    b, stream, graph = Layer(**case), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for i in range(2):
        b.step(i, stream, lambda: None)
    torch.cuda.synchronize()
    before = b.results()
    with torch.cuda.graph(graph, stream=stream):
        b.step(2, torch.cuda.current_stream(), lambda: None)
    for _ in range(2):
        for t, s in zip((b.ring.k, b.ring.v, b.means), (before[1], before[2], before[3])):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(b.results(), want))
