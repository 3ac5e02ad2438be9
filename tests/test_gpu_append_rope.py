"""Keys and values from the projection into the ring with norm and rotary positions, against the float64 oracle.

Bounds: as in test_gpu_rope; keys that become e4m3 codes instead of bf16 are off by half a step of e4m3 (2^-4 of the
value, 2^-10 of the scale where it is subnormal) after the same fp32 arithmetic, the reciprocal and one product, and
saturate at 448 scales.  Values and everything that the call must leave alone are exact.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_helpers as lh  # noqa: E402
from oracle import keysets as ks  # noqa: E402
from oracle import layer as ol  # noqa: E402
from oracle import quant as oq  # noqa: E402
from paper_2607_00712_gb300 import abi, synth  # noqa: E402
from paper_2607_00712_gb300.device import Ring  # noqa: E402
from test_gpu_rope import EPS, _device_steps, _expected, _steps, _weight  # noqa: E402

pytestmark = pytest.mark.gpu
NONE, HEAD, TOKEN = abi.ISPA_QK_NORM_NONE, abi.ISPA_QK_NORM_HEAD, abi.ISPA_QK_NORM_TOKEN


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


class Call:
    """A fused projection's rows, a ring with older frames in it, and what an append makes of them."""

    def __init__(self, P, frames, hq, H, d, axis_pairs, layout, norms, fmt=0, cap=None, sinks=0, written=None, pos0=0,
                 in_place=False, seed=0, pos=None, **scaling):
        g = np.random.default_rng(1000 * P + 10 * frames + seed)
        n = self.n = P * frames
        self.P, self.frames, self.hq, self.H, self.d, self.fmt, self.norms = P, frames, hq, H, d, fmt, norms
        self.cap = cap or frames + 1
        self.width = (hq + 2 * H) * d + 24                       # 24 columns that belong to nobody
        size = 0.25 + np.abs(g.standard_normal(self.width))
        self.host = synth.bf16_round((g.standard_normal((n, self.width)) * size).astype(np.float32))
        self.x = torch.from_numpy(self.host).cuda().to(torch.bfloat16)
        self.ring = Ring(H, d, P, self.cap, sinks, k_e4m3=fmt == 1, kv_e4m3=fmt == 2)
        for t in (self.ring.k, self.ring.v):
            t.copy_(torch.from_numpy(g.integers(0, 120, tuple(t.shape)).astype(np.uint8)).cuda().to(t.dtype))
        self.ring.c.frames_written = self.written = self.cap + 1 if written is None else written
        steps, factor = _steps(axis_pairs, **scaling)
        self.pos = g.integers(-50, 3000, (len(axis_pairs), n)) if pos is None else pos
        self.pos_t = torch.from_numpy(np.asarray(self.pos).astype(np.int32)).cuda()
        self.pos0 = pos0
        self.steps_t = _device_steps(steps)
        self.rope = abi.rope(layout, d, axis_pairs, self.steps_t, factor)
        self.angle, self.factor = ol.angles(self.pos, pos0, axis_pairs, steps), factor
        self.half = layout == abi.ISPA_ROPE_HALF
        self.w = [_weight(seed + i, h, d, m) for i, (h, m) in enumerate(zip((hq, H), norms))]
        self.wt = [None if w is None else torch.from_numpy(w).cuda() for w in self.w]
        self.ks = ((0.5 + g.random(H)) * 0.02).astype(np.float32)      # some keys are cut off
        self.vs = ((0.5 + g.random(H)) * 0.02).astype(np.float32)
        self.ks_t, self.vs_t = torch.from_numpy(self.ks).cuda(), torch.from_numpy(self.vs).cuda()
        self.in_place = in_place
        self.q_out = torch.full((n + 1, max(hq, 1), d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.before = [t.clone() for t in (self.x, self.ring.k, self.ring.v)]

    def run(self, stream=None):
        hq, H, d, W = self.hq, self.H, self.d, self.width
        k = abi.rope_rows(self.x[:, hq * d:], None, H, W, 0, self.norms[1], self.wt[1], EPS)
        q = None
        if hq:
            q = abi.rope_rows(self.x, self.x if self.in_place else self.q_out, hq, W, W if self.in_place else hq * d,
                              self.norms[0], self.wt[0], EPS)
        abi.ispa_kv_append_rope(self.ring.c, self.rope, k, q, self.x[:, (hq + H) * d:], W, self.pos_t, self.pos0,
                                self.frames, self.ks_t if self.fmt else None, self.vs_t if self.fmt == 2 else None,
                                stream)
        return self

    def check(self):
        torch.cuda.synchronize()
        hq, H, d, P, n = self.hq, self.H, self.d, self.P, self.n
        assert self.ring.c.frames_written == self.written + self.frames
        x0, k0, v0 = self.before
        at = np.concatenate([np.arange(P) + P * ks.ring_slot(self.written + i, self.cap, self.ring.c.n_sink_frames)
                             for i in range(self.frames)])
        at = torch.from_numpy(at).cuda()
        # queries
        if hq:
            want, bound = _expected(self.host[:, :hq * d], hq, d, self.norms[0], self.w[0], self.angle, self.factor,
                                    self.half)
            got = self.x[:, :hq * d].reshape(n, hq, d) if self.in_place else self.q_out[:n]
            lh.assert_within(got.float().cpu().numpy(), want, bound, "q")
            assert (self.q_out[n] == 7.0).all()
        keep = hq * d if self.in_place else 0
        assert torch.equal(self.x[:, keep:], x0[:, keep:])
        # keys
        want, bound = _expected(self.host[:, hq * d:(hq + H) * d], H, d, self.norms[1], self.w[1], self.angle,
                                self.factor, self.half)
        want, bound = want.transpose(1, 0, 2), bound.transpose(1, 0, 2)
        got = self.ring.k[:, at]
        if self.fmt:
            s = self.ks.astype(np.float64)[:, None, None]
            err = bound - lh.U_BF16 * np.abs(want)        # of the fp32 value
            cut = np.clip(want, -448 * s, 448 * s)
            half = np.maximum(2.0 ** -4 * np.abs(cut), 2.0 ** -10 * s)
            lh.assert_within(oq.decode(got.cpu().numpy()) * s, cut,
                             half * (1 + 8 * lh.U) + err * (1 + 2.0 ** -4) + 8 * lh.U * np.abs(cut), "k codes")
        else:
            lh.assert_within(got.float().cpu().numpy(), want, bound, "k")
        # values
        v = self.host[:, (hq + H) * d:(hq + 2 * H) * d].reshape(n, H, d)
        if self.fmt == 2:
            codes = oq.quantize_heads_with_scale(v, self.vs)
            assert np.array_equal(self.ring.v[:, :, at].cpu().numpy(), codes.transpose(1, 2, 0))
        else:
            assert np.array_equal(self.ring.v[:, at].float().cpu().numpy(), v.transpose(1, 0, 2))
        # the other frames
        others = torch.ones(self.cap * P, dtype=torch.bool, device="cuda")
        others[at] = False
        assert torch.equal(self.ring.k[:, others], k0[:, others])
        if self.fmt == 2:
            behind = torch.ones(self.ring.v.shape[2], dtype=torch.bool, device="cuda")
            behind[at] = False
            assert torch.equal(self.ring.v[:, :, behind], v0[:, :, behind])
        else:
            assert torch.equal(self.ring.v[:, others], v0[:, others])
        assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("norms", [(NONE, NONE), (HEAD, HEAD), (TOKEN, TOKEN), (TOKEN, NONE), (HEAD, TOKEN)])
@pytest.mark.parametrize("P,frames", [(4, 1), (52, 3), (1560, 1)])
def test_formats_norms_and_sizes(fmt, norms, P, frames):
    Call(P, frames, 3, 3, 128, [22, 21, 21], abi.ISPA_ROPE_INTERLEAVED, norms, fmt).run().check()


@pytest.mark.parametrize("layout", [abi.ISPA_ROPE_INTERLEAVED, abi.ISPA_ROPE_HALF])
@pytest.mark.parametrize("hq,H,d,pairs", [(0, 1, 64, [32]), (1, 1, 64, [16]), (8, 2, 128, [24, 20, 20]),
                                          (0, 12, 128, [32]),
                                          (5, 5, 128, [4]), (24, 8, 64, [32]), (40, 40, 128, [24, 20, 20])])
@pytest.mark.parametrize("P", [1, 333])
def test_shapes(layout, hq, H, d, pairs, P):
    for norm in (TOKEN, HEAD, NONE):
        Call(P, 2, hq, H, d, pairs, layout, (norm, norm), 0).run().check()


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("cap,sinks,written,frames", [(3, 0, 0, 1), (3, 0, 2, 3), (5, 1, 4, 4), (17, 0, 40, 16),
                                                      (4, 2, 1, 2),
                                                      (2, 0, 10 ** 12 + 1, 1)])
def test_ring_positions(fmt, cap, sinks, written, frames):
    Call(20, frames, 2, 2, 128, [64], abi.ISPA_ROPE_HALF, (HEAD, HEAD), fmt, cap, sinks, written).run().check()


def test_far_positions_and_scaling():
    pos = np.array([[2 ** 31 - 1 - i for i in range(40)]])
    Call(40, 1, 2, 2, 128, [64], abi.ISPA_ROPE_HALF, (NONE, NONE), pos=pos, pos0=2 ** 40,
         scaling=abi.ISPA_ROPE_SCALE_PARTS, scale=8.0, trained_length=32768.0).run().check()


def test_queries_in_place():
    Call(300, 2, 4, 2, 128, [64], abi.ISPA_ROPE_INTERLEAVED, (TOKEN, TOKEN), in_place=True).run().check()


def test_same_keys_as_the_two_calls():
    """ispa_rope_apply and ispa_kv_append give the same bits: one arithmetic, one rounding."""
    for P, norm in ((5, HEAD), (700, TOKEN), (700, NONE)):
        c = Call(P, 2, 4, 4, 128, [64], abi.ISPA_ROPE_HALF, (norm, norm))
        k = torch.empty(c.n, 4, 128, dtype=torch.bfloat16, device="cuda")
        q = torch.empty_like(k)
        two = Ring(4, 128, P, c.cap)
        two.c.frames_written = c.written
        two.k.copy_(c.ring.k), two.v.copy_(c.ring.v)
        W = c.width
        abi.ispa_rope_apply(c.rope, [abi.rope_rows(c.x, q, 4, W, 512, norm, c.wt[0], EPS),
                                     abi.rope_rows(c.x[:, 512:], k, 4, W, 512, norm, c.wt[1], EPS)], c.pos_t, 0, c.n)
        abi.ispa_kv_append(two.c, k, c.x[:, 1024:1536].contiguous(), 2)
        c.run().check()
        assert torch.equal(two.k, c.ring.k) and torch.equal(two.v, c.ring.v) and torch.equal(q, c.q_out[:c.n])


def test_infinite_and_nan_rows_stay_their_own():
    c = Call(64, 2, 2, 2, 128, [32], abi.ISPA_ROPE_HALF, (TOKEN, TOKEN))
    c.run().check()
    good_k, good_q = c.ring.k.clone(), c.q_out.clone()
    d = Call(64, 2, 2, 2, 128, [32], abi.ISPA_ROPE_HALF, (TOKEN, TOKEN))
    d.x[5, 300] = float("nan")      # a key of token 5
    d.x[77, 10] = float("inf")      # a query of token 77
    d.run()
    torch.cuda.synchronize()
    slot = ks.ring_slot(d.written, d.cap, 0) * 64
    bad = torch.zeros(d.cap * 64, dtype=torch.bool, device="cuda")
    bad[slot + 5] = True
    assert torch.equal(d.ring.k[:, ~bad], good_k[:, ~bad]) and d.ring.k[:, bad].isnan().all()
    assert torch.equal(d.q_out[:77], good_q[:77]) and torch.equal(d.q_out[78:], good_q[78:])
    assert not torch.isfinite(d.q_out[77]).all()


def test_ring_past_2_31_bytes():
    """Head 1 of a ring whose heads take over 2 GiB each."""
    P, H, d, cap = 1560, 2, 128, 5400
    ring = Ring(H, d, P, cap)
    ring.c.frames_written = cap * 2 - 1
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(2 * P, 2 * H * d, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.zeros(1, 2 * P, dtype=torch.int32, device="cuda")
    steps = _device_steps(_steps([64])[0])
    abi.ispa_kv_append_rope(ring.c, abi.rope(0, d, [64], steps), abi.rope_rows(x, None, H, 2 * H * d, 0), None,
                            x[:, H * d:], 2 * H * d, pos, 0, 2)
    torch.cuda.synchronize()
    for f, slot in ((0, cap - 1), (1, 0)):
        rows = x[f * P:(f + 1) * P].view(P, 2, H, d)
        for h in range(H):      # position 0 turns nothing
            assert torch.equal(ring.k[h, slot * P:(slot + 1) * P], rows[:, 0, h])
            assert torch.equal(ring.v[h, slot * P:(slot + 1) * P], rows[:, 1, h])


@pytest.mark.parametrize("fmt", [0, 2])
def test_captured_and_on_another_stream(fmt):
    c = Call(260, 2, 3, 3, 128, [64], abi.ISPA_ROPE_HALF, (TOKEN, TOKEN), fmt)
    eager = Call(260, 2, 3, 3, 128, [64], abi.ISPA_ROPE_HALF, (TOKEN, TOKEN), fmt)
    eager.run().check()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        c.run(s)
    for t, b in zip((c.x, c.ring.k, c.ring.v), c.before):
        assert torch.equal(t, b)            # capture alone does nothing
    for _ in range(2):
        c.q_out.fill_(7.0)
        graph.replay()
        c.check()
        assert torch.equal(c.ring.k, eager.ring.k) and torch.equal(c.ring.v, eager.ring.v)
