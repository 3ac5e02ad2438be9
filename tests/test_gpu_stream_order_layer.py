"""The calls around the attention back to back, each launched while the one before it finishes, over the same buffers again
and again, on the default stream, on two streams at once and in a replayed graph: the same bits as one at a time.  One token
and a few (dp4a, a block a row), some hundred and some thousand (teams over runs of rows, all tensor-core forms)."""
import pytest

torch = pytest.importorskip("torch")

import numpy as np  # noqa: E402

from paper_2607_00712_gb300 import abi  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


class Chain:
    """Norm to int8 codes, q and k in one projection, rotary positions in place, row codes, output projection, gate and
    residual in place with the next norm."""

    def __init__(self, n, H, d, norm):
        g = torch.Generator(device="cuda").manual_seed(n)
        self.n, self.H, self.d, self.D = n, H, d, H * d
        D = self.D
        self.start = torch.randn(n, D, generator=g, device="cuda")
        self.x = self.start.clone()
        self.codes, self.scale = torch.empty(n, D, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        self.qk = torch.empty(n, 2 * D, dtype=torch.bfloat16, device="cuda")
        self.a8, self.sa = torch.empty(n, 2 * D, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        self.y, self.h = (torch.empty(n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.w = []
        for rows, cols in ((D, 2 * D), (2 * D, D)):
            W = torch.randn(rows, cols, generator=g, device="cuda") / rows ** 0.5
            q, s = torch.empty(cols, rows, dtype=torch.int8, device="cuda"), torch.empty(cols, device="cuda")
            abi.ispa_quantize_weight_i8(W, None, rows, cols, q, s)
            self.w += [q, s]
        self.e = 0.3 * torch.randn(-(-n // 60), 6, D, generator=g, device="cuda")
        steps = torch.from_numpy(np.array(abi.ispa_rope_steps(d // 2)[0], np.uint64).view(np.int64)).cuda()
        self.rope = abi.rope(abi.ISPA_ROPE_INTERLEAVED, d, [d // 2], steps)
        self.pos = torch.arange(n, dtype=torch.int32, device="cuda")[None]
        self.norm = norm
        torch.cuda.synchronize()

    def step(self, i, stream, sync):
        n, D, H, e = self.n, self.D, self.H, self.e
        layer, after = abi.norm(abi.ISPA_NORM_LAYER), abi.norm(abi.ISPA_NORM_RMS)
        mod = abi.modulation(e[:, 1], e[:, 0], e[:, 2], 6 * D, 60)
        rows = [abi.rope_rows(t, t, H, 2 * D, 2 * D, self.norm) for t in (self.qk, self.qk[:, D:])]
        for call in (
                lambda: abi.ispa_norm_modulate(self.x, abi.ISPA_FP32, n, D, layer, mod,
                                               abi.rows_out(self.codes, abi.ISPA_ROWS_I8, self.scale), stream),
                lambda: abi.ispa_linear_i8(self.codes, self.scale, self.w[0], self.w[1], None, n, D, 2 * D, self.qk,
                                           stream),
                lambda: abi.ispa_rope_apply(self.rope, rows, self.pos, i, n, stream),
                lambda: abi.ispa_quantize_rows_i8(self.qk, n, 2 * D, self.a8, self.sa, stream),
                lambda: abi.ispa_linear_i8(self.a8, self.sa, self.w[2], self.w[3], None, n, 2 * D, D, self.y, stream),
                lambda: abi.ispa_gate_residual(self.x, abi.ISPA_FP32, self.y, n, D, after, 0.9, 0.5, mod, self.x, layer,
                                               abi.rows_out(self.h), stream)):
            call()
            if sync:
                torch.cuda.synchronize()

    def run(self, steps, stream=None, sync=False):
        for i in range(steps):
            self.step(i, stream, sync)

    def reset(self):
        self.x.copy_(self.start)

    def seen(self):
        return [t.clone() for t in (self.x, self.h, self.qk, self.y, self.codes, self.a8, self.scale, self.sa)]


NONE, HEAD, TOKEN = abi.ISPA_QK_NORM_NONE, abi.ISPA_QK_NORM_HEAD, abi.ISPA_QK_NORM_TOKEN


@pytest.mark.parametrize("n,H,d,norm", [(1, 12, 128, HEAD), (4, 2, 64, NONE), (7, 12, 128, TOKEN), (24, 4, 128, TOKEN),
                                        (180, 2, 128, TOKEN), (700, 12, 128, HEAD), (1560, 12, 128, TOKEN),
                                        (4680, 12, 128, TOKEN), (2500, 4, 64, HEAD)])
def test_back_to_back_calls_equal_synchronised_ones(n, H, d, norm):
    steps = 12
    a, b = Chain(n, H, d, norm), Chain(n, H, d, norm)
    a.run(steps, sync=True)
    want = a.seen()
    assert torch.isfinite(want[0]).all() and want[0].abs().max() > 0
    for _ in range(3):
        a.reset()
        a.run(steps)
        for x, y in zip(want, a.seen()):
            assert torch.equal(x, y)
    # two streams at once
    streams = [torch.cuda.Stream() for _ in range(2)]
    for c in (a, b):
        c.reset()
    torch.cuda.synchronize()
    for i in range(steps):
        for c, s in zip((a, b), streams):
            c.step(i, s, False)
    torch.cuda.synchronize()
    for c in (a, b):
        for x, y in zip(want, c.seen()):
            assert torch.equal(x, y)
    # captured, and replayed twice
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run(steps, torch.cuda.current_stream())
    for _ in range(2):
        a.reset()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, a.seen()):
            assert torch.equal(x, y)
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


def test_four_host_threads():
    import threading
    chains = [Chain(n, 12, 128, m) for n, m in ((3, HEAD), (200, TOKEN), (1560, HEAD), (2600, TOKEN))]
    want = []
    for c in chains:
        c.run(6, sync=True)
        want.append(c.seen())
        c.reset()
    torch.cuda.synchronize()
    streams, failed = [torch.cuda.Stream() for _ in chains], []

    def work(c, s):
        try:
            c.run(6, s)
        except Exception as e:   # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=x) for x in zip(chains, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for c, w in zip(chains, want):
        for x, y in zip(w, c.seen()):
            assert torch.equal(x, y)
