"""A layer's attention block through the C-ABI, as a program runs it: norm and modulation to int8 codes, the int8
projection, q/k norm and rotary positions, the chunk attention over the ring and the append, the int8 output projection,
gate, residual and the next norm.  Each step is held against the float64 oracle on the step before's own output, over
two chunks; then the whole is captured into a graph and replayed.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_helpers as lh  # noqa: E402
from gpu_helpers import assert_close_attn  # noqa: E402
from oracle import attention as oat  # noqa: E402
from oracle import layer as ol  # noqa: E402
from paper_2607_00712_gb300 import abi  # noqa: E402
from paper_2607_00712_gb300.device import Ring, to_f32  # noqa: E402

pytestmark = pytest.mark.gpu
EPS = 1e-6
P, H, d, CHUNK = 60, 2, 128, 3      # tokens per frame (6 x 10), heads, head_dim, frames of a chunk
D, N = H * d, 3 * P


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


class Layer:
    def __init__(self, seed):
        g = np.random.default_rng(seed)
        dev = dict(device="cuda")
        self.ring = Ring(H, d, P, capacity_frames=6)
        self.np = dict(wqk=(g.standard_normal((D, 2 * D)) / 16).astype(np.float32),
                       wv=(g.standard_normal((D, D)) / 16).astype(np.float32),
                       wo=(g.standard_normal((D, D)) / 16).astype(np.float32),
                       bqk=(0.1 * g.standard_normal(2 * D)).astype(np.float32),
                       gq=(1 + 0.1 * g.standard_normal(D)).astype(np.float32),
                       gk=(1 + 0.1 * g.standard_normal(D)).astype(np.float32),
                       e=(0.3 * g.standard_normal((CHUNK, 6, D))).astype(np.float32))
        self.t = {k: torch.from_numpy(v).cuda() for k, v in self.np.items()}
        for k, n in (("wqk", 2 * D), ("wv", D), ("wo", D)):
            q, s = torch.empty(n, D, dtype=torch.int8, **dev), torch.empty(n, **dev)
            abi.ispa_quantize_weight_i8(self.t[k], None, D, n, q, s)
            self.t[k + "_q"], self.t[k + "_s"] = q, s
        self.pairs = [22, 21, 21]
        self.steps = [s for m in self.pairs for s in abi.ispa_rope_steps(m)[0]]
        steps = torch.from_numpy(np.array(self.steps, np.uint64).view(np.int64)).cuda()
        self.rope = abi.rope(abi.ISPA_ROPE_INTERLEAVED, d, self.pairs, steps)
        t = np.arange(N)
        self.pos = np.stack([t // P, t // 10 % 6, t % 10])
        self.pos_t = torch.from_numpy(self.pos.astype(np.int32)).cuda()
        bf = dict(dtype=torch.bfloat16, device="cuda")
        i8 = dict(dtype=torch.int8, device="cuda")
        self.o = dict(x=torch.zeros(N, D, **dev), codes=torch.empty(N, D, **i8), scale=torch.empty(N, **dev),
                      qk=torch.empty(N, 2 * D, **bf), v=torch.empty(N, H, d, **bf), q=torch.empty(N, H, d, **bf),
                      k=torch.empty(N, H, d, **bf), a=torch.empty(N, D, **bf), a_codes=torch.empty(N, D, **i8),
                      a_scale=torch.empty(N, **dev), y=torch.empty(N, D, **bf), x2=torch.empty(N, D, **dev),
                      h=torch.empty(N, D, **bf))

    def run(self, frame0, stream=None, append=True):
        o, t, e = self.o, self.t, self.t["e"]
        mod = abi.modulation(e[:, 1], e[:, 0], e[:, 2], 6 * D, P)
        after = abi.modulation(e[:, 4], e[:, 3], e[:, 2], 6 * D, P)
        pre = abi.norm(abi.ISPA_NORM_LAYER, EPS)
        abi.ispa_norm_modulate(o["x"], abi.ISPA_FP32, N, D, pre, mod, abi.rows_out(o["codes"], abi.ISPA_ROWS_I8, o["scale"]),
                               stream)
        abi.ispa_linear_i8(o["codes"], o["scale"], t["wqk_q"], t["wqk_s"], t["bqk"], N, D, 2 * D, o["qk"], stream)
        abi.ispa_linear_i8(o["codes"], o["scale"], t["wv_q"], t["wv_s"], None, N, D, D, o["v"], stream)
        rows = [abi.rope_rows(o["qk"], o["q"], H, 2 * D, D, abi.ISPA_QK_NORM_TOKEN, t["gq"], EPS),
                abi.rope_rows(o["qk"][:, D:], o["k"], H, 2 * D, D, abi.ISPA_QK_NORM_TOKEN, t["gk"], EPS)]
        abi.ispa_rope_apply(self.rope, rows, self.pos_t, frame0, N, stream)
        abi.ispa_attn_full(self.ring.c, o["q"], o["k"], o["v"], N, 0.0, o["a"], None, stream)
        if append:
            abi.ispa_kv_append(self.ring.c, o["k"], o["v"], CHUNK, stream)
        abi.ispa_quantize_rows_i8(o["a"], N, D, o["a_codes"], o["a_scale"], stream)
        abi.ispa_linear_i8(o["a_codes"], o["a_scale"], t["wo_q"], t["wo_s"], None, N, D, D, o["y"], stream)
        abi.ispa_gate_residual(o["x"], abi.ISPA_FP32, o["y"], N, D, None, 1.0, 1.0, after, o["x2"], pre,
                               abi.rows_out(o["h"]), stream)

    def check(self, x, frame0, hist):
        """Every step against the oracle on its own input; hist: the (k, v) of the chunks before."""
        o = {k: v.cpu().numpy() if v.dtype != torch.bfloat16 else to_f32(v) for k, v in self.o.items()}
        w, e = self.np, self.np["e"]
        n = ol.norm(x, ol.LAYER, EPS)
        h = ol.modulate(n, e[:, 1], e[:, 0], P)
        err = lh.modulate_error(lh.norm_error(x, ol.LAYER, EPS, None, None), n, e[:, 1], e[:, 0], P)
        lh.check_codes(o["codes"], o["scale"], h, err, "i8")
        wq = {k: ol.quantize_i8(w[k].T) for k in ("wqk", "wv", "wo")}
        assert np.array_equal(o["qk"], ol.linear_i8(o["codes"], o["scale"], *wq["wqk"], w["bqk"]))
        assert np.array_equal(o["v"].reshape(N, D), ol.linear_i8(o["codes"], o["scale"], *wq["wv"]))
        angle = ol.angles(self.pos, frame0, self.pairs, self.steps)
        for name, at, g in (("q", 0, w["gq"]), ("k", D, w["gk"])):
            r = o["qk"][:, at:at + D].astype(np.float64)
            v, ve = ol.norm(r, ol.RMS, EPS, g), lh.norm_error(r, ol.RMS, EPS, g, None)
            want = ol.rope(v.reshape(N, H, d), angle, 1.0, False)
            pair = (np.abs(v) * 20 * lh.U + ve).reshape(N, H, d // 2, 2).sum(-1, keepdims=True).repeat(2, -1)
            lh.assert_within(o[name], want, lh.U_BF16 * np.abs(want) + 1.01 * pair.reshape(want.shape))
        kh = np.concatenate([k for k, _ in hist]) if hist else o["k"][:0]
        vh = np.concatenate([v for _, v in hist]) if hist else o["v"][:0]
        ref, _ = oat.attn_full(o["q"], kh, vh, o["k"], o["v"], P)
        assert_close_attn(o["a"].reshape(ref.shape), ref, "attention")
        codes, scale = ol.quantize_i8(o["a"])
        assert np.array_equal(o["a_codes"], codes) and np.array_equal(o["a_scale"], scale)
        assert np.array_equal(o["y"], ol.linear_i8(codes, scale, *wq["wo"]))
        want = ol.gate_residual(x, o["y"], 1.0, 1.0, e[:, 2], P)
        lh.assert_within(o["x2"], want, 8 * lh.U * (np.abs(x) + np.abs(want - x)) + 1e-45)
        n = ol.norm(o["x2"], ol.LAYER, EPS)
        h = ol.modulate(n, e[:, 4], e[:, 3], P)
        err = lh.modulate_error(lh.norm_error(o["x2"], ol.LAYER, EPS, None, None), n, e[:, 4], e[:, 3], P)
        lh.assert_within(o["h"], h, (1 + lh.U_BF16) * err + lh.U_BF16 * np.abs(h))
        return o["k"], o["v"]


def test_two_chunks_step_by_step():
    layer, hist = Layer(0), []
    for chunk in range(2):
        x = lh.rows(chunk, N, D)
        layer.o["x"].copy_(torch.from_numpy(x))
        torch.cuda.synchronize()
        layer.run(chunk * CHUNK)
        torch.cuda.synchronize()
        assert abi.ispa_last_device_error()[0] == abi.ISPA_OK
        hist.append(layer.check(x, chunk * CHUNK, hist))
    assert layer.ring.frames_written == 2 * CHUNK


def test_captured_layer_gives_what_the_eager_one_gives():
    layer = Layer(1)
    x = [torch.from_numpy(lh.rows(10 + i, N, D)).cuda() for i in range(3)]
    layer.o["x"].copy_(x[0])
    layer.run(0)                       # the history of what follows
    want = []
    for v in x[1:]:
        layer.o["x"].copy_(v)
        layer.run(CHUNK, append=False)
        torch.cuda.synchronize()
        want.append([layer.o[k].clone() for k in ("q", "k", "a", "x2", "h")])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.run(CHUNK, torch.cuda.current_stream(), append=False)
    for v, w in zip(x[1:] * 2, want * 2):
        layer.o["x"].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for k, t in zip(("q", "k", "a", "x2", "h"), w):
            assert torch.equal(layer.o[k], t), k
